// Losses over classes of fp32 layers and their gradients where the products are short: what the tiles of fc_xent.hip lay out, split and join before and after
// them would take longer than they do.
//
// The scores are kept here, in fp32 (4096 x 2048 at the most), and dz after them in fp32 too.  Products are those of the fp32
// matrix unit, 32 x 32 of C to one wave or to 2, 4 or 8 of them that share the contraction and add up in LDS; operands come straight from
// where they are: a lane has a row (or column) of its own, and of the contraction half, in whichever order, as long as
// both operands take the same.  Forward: scores, rows; backward: scores, dz with db, then da and dw in one launch.
#include "common.h"
#include "exp_of.h"
#include "xent.h"

namespace vgg {

namespace {

constexpr int kWaves = 8;

// One product C[i][j] = sum_c A[i][c] B[j][c].
struct Small {
    const float *a, *b;
    size_t lda, ldb;               // elements from row to row, of i and j, or of c
    int rows, cols, length;        // i, j, c
    int waves;                     // of a tile
    float *out;                    // [i][ld]
    size_t ld;
    const float *relu_of;          // where given ([i][cols]): 0 where that is not above 0
    const int *open;               // of c: 0 where B's row counts as zeros whatever it holds
};

// The wave's share of a tile's products: runs of 8 contraction indices, every waves-th of them, eight runs at once and the next eight on their
// way.  Operands whose contraction index is their rows' place (TR): value by value, neighbouring lanes in neighbouring columns.
template <bool A_TR, bool B_TR> __device__ __forceinline__ f32x16 tile_share(const Small &p, int i0, int j0, int share, int lane)
{
    constexpr int U = 8;
    const int half = lane >> 5, step = 8 * p.waves;
    const int i = i0 + (lane & 31) < p.rows ? i0 + (lane & 31) : p.rows - 1, j = j0 + (lane & 31) < p.cols ? j0 + (lane & 31) : p.cols - 1;
    const float *a = p.a + (A_TR ? (size_t)i : (size_t)i * p.lda), *b = p.b + (B_TR ? (size_t)j : (size_t)j * p.ldb);
    auto fetch = [&](int c0, f32x4 (&va)[U], f32x4 (&vb)[U]) __attribute__((always_inline)) {
        // (whole runs, for all lanes alike, without a branch between loads: what hangs on one is waited for by itself)
        if (c0 + (U - 1) * step + 8 <= p.length) {
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const int c = c0 + u * step + 4 * half;
                if constexpr (A_TR) {
#pragma unroll
                    for (int k = 0; k < 4; ++k) va[u][k] = a[(size_t)(c + k) * p.lda];
                } else
                    __builtin_memcpy(&va[u], a + c, 16);
                if constexpr (B_TR) {
#pragma unroll
                    for (int k = 0; k < 4; ++k) vb[u][k] = b[(size_t)(c + k) * p.ldb];
                } else
                    __builtin_memcpy(&vb[u], b + c, 16);
            }
            if (p.open) {
#pragma unroll
                for (int u = 0; u < U; ++u)
#pragma unroll
                    for (int k = 0; k < 4; ++k) vb[u][k] = p.open[c0 + u * step + 4 * half + k] ? vb[u][k] : 0.f;
            }
        } else {
#pragma unroll
            for (int u = 0; u < U; ++u)
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    const int c = c0 + u * step + 4 * half + k, at = c < p.length ? c : p.length - 1;
                    const float x = a[A_TR ? (size_t)at * p.lda : at], y = b[B_TR ? (size_t)at * p.ldb : at];
                    va[u][k] = c < p.length ? x : 0.f;
                    vb[u][k] = c < p.length && (!p.open || p.open[at]) ? y : 0.f;
                }
        }
    };
    f32x16 acc = {}, other = {};      // (two sums: a product waits for the one before the last)
    auto multiply = [&](const f32x4 (&va)[U], const f32x4 (&vb)[U]) __attribute__((always_inline)) {
#pragma unroll
        for (int u = 0; u < U; ++u)
#pragma unroll
            for (int k = 0; k < 4; k += 2) {
                acc = __builtin_amdgcn_mfma_f32_32x32x2f32(va[u][k], vb[u][k], acc, 0, 0, 0);
                other = __builtin_amdgcn_mfma_f32_32x32x2f32(va[u][k + 1], vb[u][k + 1], other, 0, 0, 0);
            }
    };
    f32x4 va[2][U], vb[2][U];
    int c = 8 * share;
    if (c < p.length) fetch(c, va[0], vb[0]);
    while (c < p.length) {
        const int next = c + U * step, after = next + U * step;
        if (next < p.length) fetch(next, va[1], vb[1]);
        multiply(va[0], vb[0]);
        if (next >= p.length) break;
        if (after < p.length) fetch(after, va[0], vb[0]);
        multiply(va[1], vb[1]);
        c = after;
    }
    return acc + other;
}

template <bool A_TR, bool B_TR> __device__ __forceinline__ void small_tiles(const Small &p, int block, float *lds)
{
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, tile = block * (kWaves / p.waves) + wave / p.waves, share = wave % p.waves;
    const int across = (p.cols + 31) / 32, i0 = tile / across * 32, j0 = tile % across * 32;
    const bool there = i0 < p.rows;
    f32x16 acc = {};
    if (there) acc = tile_share<A_TR, B_TR>(p, i0, j0, share, lane);
    // value v of a lane: row 8 (v / 4) + 4 (lane / 32) + v % 4, column lane % 32; a tile's waves add up in order, each its part of the rows
    float *mine = lds + wave * 1024;
#pragma unroll
    for (int v = 0; v < 16; ++v) mine[(8 * (v >> 2) + 4 * (lane >> 5) + (v & 3)) * 32 + (lane & 31)] = acc[v];
    __syncthreads();
    if (!there) return;
    const float *all = lds + (wave - share) * 1024;
    for (int at = share * 64 + lane; at < 1024; at += 64 * p.waves) {
        float s = 0.f;
        for (int w = 0; w < p.waves; ++w) s += all[w * 1024 + at];
        const int i = i0 + (at >> 5), j = j0 + (at & 31);
        if (i >= p.rows || j >= p.cols) continue;
        if (p.relu_of && !(p.relu_of[(size_t)i * p.cols + j] > 0.f)) s = 0.f;
        p.out[(size_t)i * p.ld + j] = s;
    }
}

__global__ __launch_bounds__(512) void small_scores_kernel(Small p)
{
    __shared__ float lds[kWaves * 1024];
    small_tiles<false, false>(p, blockIdx.x, lds);
}

// da in the first workgroups, dw in those after them, db of the last ones: 512 classes each.
__global__ __launch_bounds__(512) void small_gradients_kernel(Small da, Small dw, int da_blocks, int dw_blocks, const float *__restrict__ db_part, int db_parts, int classes, float *db)
{
    __shared__ float lds[kWaves * 1024];
    const int block = blockIdx.x;
    if (block < da_blocks) return small_tiles<false, true>(da, block, lds);
    if (block < da_blocks + dw_blocks) return small_tiles<true, true>(dw, block - da_blocks, lds);
    const int k = (block - da_blocks - dw_blocks) * 512 + threadIdx.x;
    if (k >= classes) return;
    float s = 0.f;
    for (int q = 0; q < db_parts; ++q) s += db_part[(size_t)q * classes + k];
    db[k] = s;
}

// Scores z [N][ld] become dz; db of a range of rows; whether a row counts.  A workgroup: 2^quads times four classes, and as many rows at a time as it
// has threads for.
__global__ __launch_bounds__(256) void small_dz_kernel(float *z, int N, int classes, size_t ld, const float *__restrict__ bias, const int32_t *__restrict__ labels,
                                                       const float *__restrict__ stats, const float *__restrict__ g, int quads, float *db_part, int *open)
{
    __shared__ f32x4 sums[256];
    const int k = (blockIdx.x << quads | (threadIdx.x & ((1 << quads) - 1))) * 4, r = threadIdx.x >> quads, at_once = 256 >> quads;
    const int r0 = (int)((long)N * blockIdx.y / gridDim.y), r1 = (int)((long)N * (blockIdx.y + 1) / gridDim.y);
    f32x4 sum = {};
    if (k < classes)
        for (int row = r0 + r; row < r1; row += at_once) {
            const int y = labels[row];
            const float w = y >= 0 && y < classes ? g[row] : 0.f, m = stats[2 * (size_t)row], log_s = stats[2 * (size_t)row + 1];
            f32x4 *here = reinterpret_cast<f32x4 *>(z + (size_t)row * ld + k), out = {};
            if (w != 0.f && log_s != -INFINITY) {
                const f32x4 v = *here;
#pragma unroll
                for (int j = 0; j < 4; ++j)
                    if (k + j < classes) {
                        const float s = v[j] + (bias ? bias[k + j] : 0.f), d = (s - m) - log_s;
                        out[j] = w * (k + j != y ? exp_of(below(d)) : s == -INFINITY ? 0.f : expm1f(d));
                    }
            }
            *here = out;
            sum += out;
            if (k == 0) open[row] = w != 0.f;
        }
    sums[threadIdx.x] = sum;
    __syncthreads();
    if (r || !db_part) return;
    for (int q = 1; q < at_once; ++q) sum += sums[(q << quads) + threadIdx.x];
#pragma unroll
    for (int j = 0; j < 4; ++j)
        if (k + j < classes) db_part[(size_t)blockIdx.y * classes + k + j] = sum[j];
}

inline long tiles_of(int rows, int cols) { return (long)((rows + 31) / 32) * ((cols + 31) / 32); }
// Waves of a tile: enough to fill the chip, each with at least 64 indices of the contraction.
inline int waves_of(long tiles, int length)
{
    int w = 1;
    while (w < kWaves && tiles * w < 2048 && length >= 64 * 2 * w) w *= 2;
    return w;
}
inline int blocks_of(const Small &p) { return (int)((tiles_of(p.rows, p.cols) * p.waves + kWaves - 1) / kWaves); }

struct Places { size_t z, open, db, bytes, ld; int db_parts, quads; };
Places places(int N, int K)
{
    Places p;
    p.ld = (K + 3) / 4 * 4;
    p.quads = 0;
    while (p.quads < 6 && (4 << p.quads) < K) ++p.quads;
    const long down = 256 >> p.quads, want = (N + 8 * down - 1) / (8 * down);
    p.db_parts = (int)(want < 64 ? want : 64);
    p.z = 0;
    p.open = round_up((size_t)N * p.ld * 4, 256);
    p.db = p.open + round_up((size_t)N * 4, 256);
    p.bytes = p.db + round_up((size_t)p.db_parts * K * 4, 256);
    return p;
}

int scores(int N, int In, int K, const float *a, const float *w, float *z, size_t ld, hipStream_t s)
{
    Small p = {};
    p.a = a; p.b = w; p.lda = p.ldb = In;
    p.rows = N; p.cols = K; p.length = In;
    p.waves = waves_of(tiles_of(N, K), In);
    p.out = z; p.ld = ld;
    small_scores_kernel<<<blocks_of(p), 512, 0, s>>>(p);
    return launch_status();
}

}  // namespace

size_t fc_xent_small_workspace(int N, int K) { return places(N, K).bytes; }

int fc_xent_small(int N, int In, int K, const float *a, const float *w, const float *bias, const int32_t *labels, float *loss, float *stats, void *ws, hipStream_t s)
{
    const Places at = places(N, K);
    float *z = reinterpret_cast<float *>(static_cast<char *>(ws) + at.z);
    const int rc = scores(N, In, K, a, w, z, at.ld, s);
    return rc ? rc : xent_rows(Scores{z, 1, N, K, at.ld, bias}, labels, loss, stats, s);
}

int fc_xent_small_bwd(int N, int In, int K, const float *a, const float *w, const float *bias, const int32_t *labels, const float *stats, const float *g, float *da, float *dw,
                      float *db, int relu_mask, void *ws_, hipStream_t s)
{
    char *ws = static_cast<char *>(ws_);
    const Places at = places(N, K);
    float *z = reinterpret_cast<float *>(ws + at.z), *db_part = reinterpret_cast<float *>(ws + at.db);
    int *open = reinterpret_cast<int *>(ws + at.open);
    int rc = scores(N, In, K, a, w, z, at.ld, s);
    if (rc) return rc;
    float *db_to = !db ? nullptr : at.db_parts == 1 ? db : db_part;
    small_dz_kernel<<<dim3((unsigned)((K + (4 << at.quads) - 1) / (4 << at.quads)), (unsigned)at.db_parts), 256, 0, s>>>(z, N, K, at.ld, bias, labels, stats, g, at.quads, db_to, open);
    if ((rc = launch_status())) return rc;
    Small pa = {}, pw = {};
    pa.a = z; pa.lda = at.ld; pa.b = w; pa.ldb = In;
    pa.rows = N; pa.cols = In; pa.length = K;
    pa.waves = waves_of(tiles_of(N, In), K);
    pa.out = da; pa.ld = In;
    pa.relu_of = relu_mask ? a : nullptr;
    pw.a = z; pw.lda = at.ld; pw.b = a; pw.ldb = In;
    pw.rows = K; pw.cols = In; pw.length = N;
    pw.waves = waves_of(tiles_of(K, In), N);
    pw.out = dw; pw.ld = In;
    pw.open = open;
    const int da_blocks = da ? blocks_of(pa) : 0, dw_blocks = dw ? blocks_of(pw) : 0, db_blocks = db && at.db_parts > 1 ? (K + 511) / 512 : 0;
    if (da_blocks + dw_blocks + db_blocks == 0) return VGG_OK;
    small_gradients_kernel<<<da_blocks + dw_blocks + db_blocks, 512, 0, s>>>(pa, pw, da_blocks, dw_blocks, db_part, at.db_parts, K, db);
    return launch_status();
}

}  // namespace vgg
