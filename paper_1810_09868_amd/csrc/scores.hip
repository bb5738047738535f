// Class scores to log probabilities: of given classes, with every row's entropy and most likely alternatives, and the
// gradient of the first two with respect to the scores.
//
// One pass over a row keeps, with d = z - m and m the largest score so far, the sums S = sum exp(d) and T = sum d exp(d); a
// larger score rescales both (S' = r S, T' = r (T + (m - m') S), r = exp(m - m')).  Then
//     log p_j = (z_j - m) - log S,   entropy = log S - T / S.
// m and log S are kept apart (stats): their sum would round what the gradient takes the exponential of.
// All sums are fp32.  A score of -inf has d = -inf and exp(d) = 0; only its product d exp(d) has to be kept from NaN.
// A NaN, or a +inf (whose d is NaN), makes S and with it everything of its row NaN.
#include "common.h"

namespace vgg {

namespace {

constexpr float kLowest = -3.402823466e38f;
constexpr float kNothing = -1e4f;   // exp of it is 0, and no product with it overflows
constexpr int kMaxTop = 64;   // one alternative to a lane

struct Sums { float m, s, t; };   // of no scores: -inf, 0, 0

// The factor and shift that bring sums over to a larger maximum M.
__device__ __forceinline__ void rebase(Sums &a, float M)
{
    const float d = fmaxf(a.m - M, kNothing);
    const float r = a.m == M ? 1.f : expf(d);
    a.t = r * (a.t + (a.s > 0.f && a.m != M ? d * a.s : 0.f));
    a.s *= r;
    a.m = M;
}
__device__ __forceinline__ Sums joined(Sums a, Sums b)
{
    const float M = fmaxf(a.m, b.m);
    rebase(a, M);
    rebase(b, M);
    return {M, a.s + b.s, a.t + b.t};
}
__device__ __forceinline__ Sums wave_joined(Sums a)
{
    const float M = wave_max(a.m);
    rebase(a, M);
    return {M, wave_sum(a.s), wave_sum(a.t)};
}

// V scores into a thread's sums.
template <int V> __device__ __forceinline__ void add_scores(Sums &a, const float (&z)[V])
{
    float M = a.m;
#pragma unroll
    for (int j = 0; j < V; ++j) M = fmaxf(M, z[j]);
    if (M > a.m) rebase(a, M);
    const float base = M == -INFINITY ? 0.f : M;
#pragma unroll
    for (int j = 0; j < V; ++j) {
        const float d = z[j] - base, e = __expf(d);
        a.s += e;
        a.t = __builtin_fmaf(fmaxf(d, kLowest), e, a.t);
    }
}

// The best scores that a wave has seen, one to a lane, best first; empty places are -inf at class -1.  Equal scores: the lower
// class is better.
struct Best {
    float v;
    int id;
    float worst_v;   // of the last of `top` places
    int worst_id;
};
__device__ __forceinline__ float lane_of(float v, int lane) { return __int_as_float(__builtin_amdgcn_readlane(__float_as_int(v), lane)); }
__device__ __forceinline__ bool better(float v, int id, float w, int wid) { return v > w || (v == w && id < wid); }
// Takes what the lanes offer (one score each) into the list, best of the wave or not.
__device__ __forceinline__ void offer(Best &b, float v, int id, int top, int lane)
{
    unsigned long long rest = __ballot(better(v, id, b.worst_v, b.worst_id));
    while (rest) {
        const int l = __builtin_ctzll(rest);
        const float nv = lane_of(v, l);
        const int ni = __builtin_amdgcn_readlane(id, l);
        const int at = __builtin_popcountll(__ballot(better(b.v, b.id, nv, ni)));
        const float pv = __shfl_up(b.v, 1);
        const int pi = __shfl_up(b.id, 1);
        if (lane > at) { b.v = pv; b.id = pi; }
        else if (lane == at) { b.v = nv; b.id = ni; }
        b.worst_v = lane_of(b.v, top - 1);
        b.worst_id = __builtin_amdgcn_readlane(b.id, top - 1);
        rest &= rest - 1;
        rest &= __ballot(better(v, id, b.worst_v, b.worst_id));
    }
}

template <typename T> constexpr int kVec = 16 / (int)sizeof(T);   // scores of a 16-byte load
__device__ __forceinline__ void load_scores(const float *p, float (&z)[4])
{
    const f32x4 v = *reinterpret_cast<const f32x4 *>(p);
#pragma unroll
    for (int j = 0; j < 4; ++j) z[j] = v[j];
}
__device__ __forceinline__ void load_scores(const bf16_t *p, float (&z)[8])
{
    typedef unsigned u32x4 __attribute__((ext_vector_type(4)));
    const u32x4 v = *reinterpret_cast<const u32x4 *>(p);
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        z[2 * j] = __uint_as_float(v[j] << 16);
        z[2 * j + 1] = __uint_as_float(v[j] & 0xffff0000u);
    }
}

struct ScoreArgs {
    int N, K, top, parts, span;   // span: scores of a part
    size_t ldz;
    const int32_t *labels;
    float *logp, *entropy, *top_logp, *stats;
    int32_t *top_idx;
    float *part_sums;             // [N][parts][3]
    float *part_v;                // [N][parts][top]
    int *part_id;
};

// What a row's waves leave in LDS (or parts in the workspace) becomes the row's outputs: `count` list entries at v, id.
__device__ void finish_row(const ScoreArgs &a, const Sums &r, float z_label, int row, const float *v, const int *id, int count, int tid, int threads)
{
    const float log_s = r.m == -INFINITY && r.s == 0.f ? -INFINITY : logf(r.s);
    const bool empty = log_s == -INFINITY;
    if (tid == 0) {
        if (a.logp) {
            const int y = a.labels[row];
            a.logp[row] = y < 0 || y >= a.K ? 0.f : empty ? -INFINITY : (z_label - r.m) - log_s;
        }
        if (a.entropy) a.entropy[row] = empty ? 0.f : log_s - r.t / r.s;
        if (a.stats) { a.stats[2 * (size_t)row] = r.m; a.stats[2 * (size_t)row + 1] = log_s; }
    }
    if (!a.top) return;
    float *tv = a.top_logp + (size_t)row * a.top;
    int32_t *ti = a.top_idx + (size_t)row * a.top;
    const bool none = !(r.s > 0.f);   // no class left, or a NaN
    int real = 0;
    for (int i = 0; i < count; ++i) real += id[i] >= 0;
    for (int i = tid; i < count; i += threads) {
        if (id[i] < 0 || none) continue;
        int rank = 0;
        for (int j = 0; j < count; ++j) rank += id[j] >= 0 && better(v[j], id[j], v[i], id[i]);
        if (rank < a.top) { tv[rank] = (v[i] - r.m) - log_s; ti[rank] = id[i]; }
    }
    for (int i = tid; i < a.top; i += threads)
        if (none || i >= real) { tv[i] = empty ? -INFINITY : none ? r.s : -INFINITY; ti[i] = -1; }
}

// W waves to a row or to a part of one; W == 1: four rows to a workgroup.
template <typename T, int W, bool TOP>
__global__ __launch_bounds__(W == 1 ? 256 : W * 64) void log_probs_kernel(const T *__restrict__ z, ScoreArgs a)
{
    constexpr int V = kVec<T>;
    constexpr int R = W == 1 ? 4 : 1;    // rows of a workgroup
    __shared__ Sums sums[W];
    __shared__ float best_v[R * (W == 1 ? 1 : W) * kMaxTop];
    __shared__ int best_id[R * (W == 1 ? 1 : W) * kMaxTop];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int unit = W == 1 ? blockIdx.x * 4 + wave : blockIdx.x;
    const int row = unit / a.parts, part = unit - row * a.parts;
    if (row >= a.N) return;              // (W == 1 only: there is no barrier there)
    const T *zr = z + (size_t)row * a.ldz;
    const int k0 = part * a.span, k1 = a.K - k0 < a.span ? a.K : k0 + a.span;
    // whole 16-byte vectors between a head and a tail of fewer scores
    const int off = (int)((reinterpret_cast<uintptr_t>(zr + k0) & 15) / sizeof(T));
    int head = off ? V - off : 0;
    if (head > k1 - k0) head = k1 - k0;
    const int v0 = k0 + head, nvec = (k1 - v0) / V, tail0 = v0 + nvec * V;
    const int ti = W == 1 ? lane : threadIdx.x, tn = W == 1 ? 64 : W * 64;

    Sums mine = {-INFINITY, 0.f, 0.f};
    Best b = {-INFINITY, -1, -INFINITY, -1};
    for (int i0 = 0; i0 < nvec; i0 += tn) {
        const int i = i0 + ti;
        float x[V];
        if (i < nvec) load_scores(zr + v0 + (size_t)i * V, x);
        else
#pragma unroll
            for (int j = 0; j < V; ++j) x[j] = -INFINITY;
        add_scores<V>(mine, x);
        if constexpr (TOP) {
            float most = x[0];
#pragma unroll
            for (int j = 1; j < V; ++j) most = fmaxf(most, x[j]);
            if (__ballot(most >= b.worst_v && most > -INFINITY))
#pragma unroll
                for (int j = 0; j < V; ++j) offer(b, x[j], v0 + i * V + j, a.top, lane);
        }
    }
    if (W == 1 || wave == 0) {           // head and tail: fewer than 2 V scores, one to a lane
        const int k = lane < head ? k0 + lane : tail0 + lane - head;
        float x[1] = {lane < head || k < k1 ? Elem<T>::load(zr + k) : -INFINITY};
        add_scores<1>(mine, x);
        if constexpr (TOP) offer(b, x[0], k, a.top, lane);
    }
    mine = wave_joined(mine);

    const int y = a.logp ? a.labels[row] : -1;
    const float z_label = y >= 0 && y < a.K ? Elem<T>::load(zr + y) : 0.f;
    if constexpr (W == 1) {
        // the list is in order already
        if (a.parts == 1) {
            float *bv = best_v + wave * kMaxTop;
            int *bi = best_id + wave * kMaxTop;
            if (TOP && lane < a.top) { bv[lane] = b.v; bi[lane] = b.id; }
            __builtin_amdgcn_wave_barrier();
            finish_row(a, mine, z_label, row, bv, bi, TOP ? a.top : 0, lane, 64);
        }
    } else {
        if (lane == 0) sums[wave] = mine;
        if (TOP && lane < a.top) { best_v[wave * a.top + lane] = b.v; best_id[wave * a.top + lane] = b.id; }
        __syncthreads();
        mine = sums[0];
        for (int w = 1; w < W; ++w) mine = joined(mine, sums[w]);
        const int count = TOP ? W * a.top : 0;
        if (a.parts == 1) { finish_row(a, mine, z_label, row, best_v, best_id, count, threadIdx.x, W * 64); return; }
        const size_t at = (size_t)row * a.parts + part;
        if (threadIdx.x == 0) { a.part_sums[at * 3] = mine.m; a.part_sums[at * 3 + 1] = mine.s; a.part_sums[at * 3 + 2] = mine.t; }
        // the part's own best, in order
        int real = 0;
        for (int i = 0; i < count; ++i) real += best_id[i] >= 0;
        for (int i = threadIdx.x; i < count; i += W * 64) {
            if (best_id[i] < 0) continue;
            int rank = 0;
            for (int j = 0; j < count; ++j) rank += best_id[j] >= 0 && better(best_v[j], best_id[j], best_v[i], best_id[i]);
            if (rank < a.top) { a.part_v[at * a.top + rank] = best_v[i]; a.part_id[at * a.top + rank] = best_id[i]; }
        }
        for (int i = real + threadIdx.x; i < a.top && TOP; i += W * 64) { a.part_v[at * a.top + i] = -INFINITY; a.part_id[at * a.top + i] = -1; }
    }
}

// The parts of a row: a workgroup of four waves to each row.
template <typename T, bool TOP>
__global__ __launch_bounds__(256) void log_probs_join_kernel(const T *__restrict__ z, ScoreArgs a)
{
    __shared__ Sums sums[4];
    __shared__ float best_v[4 * kMaxTop];
    __shared__ int best_id[4 * kMaxTop];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, row = blockIdx.x;
    Sums mine = {-INFINITY, 0.f, 0.f};
    for (int p = threadIdx.x; p < a.parts; p += 256) {
        const float *s = a.part_sums + ((size_t)row * a.parts + p) * 3;
        mine = joined(mine, {s[0], s[1], s[2]});
    }
    mine = wave_joined(mine);
    if constexpr (TOP) {
        Best b = {-INFINITY, -1, -INFINITY, -1};
        const int n = a.parts * a.top;
        const size_t at = (size_t)row * n;
        for (int i0 = 0; i0 < n; i0 += 256) {
            const int i = i0 + threadIdx.x;
            offer(b, i < n ? a.part_v[at + i] : -INFINITY, i < n ? a.part_id[at + i] : 0, a.top, lane);
        }
        if (lane < a.top) { best_v[wave * a.top + lane] = b.v; best_id[wave * a.top + lane] = b.id; }
    }
    if (lane == 0) sums[wave] = mine;
    __syncthreads();
    mine = sums[0];
    for (int w = 1; w < 4; ++w) mine = joined(mine, sums[w]);
    const int y = a.logp ? a.labels[row] : -1;
    const float z_label = y >= 0 && y < a.K ? Elem<T>::load(z + (size_t)row * a.ldz + y) : 0.f;
    finish_row(a, mine, z_label, row, best_v, best_id, TOP ? 4 * a.top : 0, threadIdx.x, 256);
}

// dz_j = g (1[j = y] - p_j) - h p_j (log p_j + entropy).
struct GradArgs {
    int N, K, span, parts;
    size_t ldz, lddz;
    const int32_t *labels;
    const float *stats, *entropy, *g_logp, *g_entropy;
};
template <typename T>
__global__ __launch_bounds__(256) void log_probs_bwd_kernel(const T *z, T *dz, GradArgs a)
{
    constexpr int V = kVec<T>;
    const int row = blockIdx.x / a.parts, part = blockIdx.x - row * a.parts;
    const T *zr = z + (size_t)row * a.ldz;
    T *dr = dz + (size_t)row * a.lddz;
    const int k0 = part * a.span, k1 = a.K - k0 < a.span ? a.K : k0 + a.span;
    int y = a.g_logp ? a.labels[row] : -1;
    if (y < 0 || y >= a.K) y = -1;
    const float g = y >= 0 ? a.g_logp[row] : 0.f;
    const float h = a.g_entropy ? a.g_entropy[row] : 0.f, ent = a.g_entropy ? a.entropy[row] : 0.f;
    const float m = a.stats[2 * (size_t)row], log_s = a.stats[2 * (size_t)row + 1];
    const bool none = m == -INFINITY && log_s == -INFINITY;
    const bool zero = none || (g == 0.f && h == 0.f);
    auto grad = [&](float zj, int j) __attribute__((always_inline)) {
        const float lp = (zj - m) - log_s, p = expf(lp);
        float x = -p * __builtin_fmaf(h, fmaxf(lp, kNothing) + ent, g);
        if (j == y && zj > -INFINITY) x += g;
        return x;
    };
    const int off = (int)((reinterpret_cast<uintptr_t>(zr + k0) & 15) / sizeof(T));
    const bool together = ((reinterpret_cast<uintptr_t>(zr) ^ reinterpret_cast<uintptr_t>(dr)) & 15) == 0;
    int head = together ? (off ? V - off : 0) : k1 - k0;   // scores before the first 16-byte vector; all, where dz has none there
    if (head > k1 - k0) head = k1 - k0;
    const int v0 = k0 + head, nvec = (k1 - v0) / V, tail0 = v0 + nvec * V;
    for (int i = threadIdx.x; i < nvec; i += 256) {
        float x[V] = {};
        if (!zero) {
            load_scores(zr + v0 + (size_t)i * V, x);
#pragma unroll
            for (int j = 0; j < V; ++j) x[j] = grad(x[j], v0 + i * V + j);
        }
#pragma unroll
        for (int j = 0; j < V; j += 4) store4(dr + v0 + (size_t)i * V + j, x[j], x[j + 1], x[j + 2], x[j + 3]);
    }
    for (int i = threadIdx.x; i < head + (k1 - tail0); i += 256) {
        const int k = i < head ? k0 + i : tail0 + i - head;
        Elem<T>::store(dr + k, zero ? 0.f : grad(Elem<T>::load(zr + k), k));
    }
}

struct Split { int parts, span; };
// Rows that are too few to fill the chip are cut into parts of at least 4096 scores.
Split split_rows(int N, int K)
{
    const int most = (K + 4095) / 4096, want = (1024 + N - 1) / N;
    int parts = want < most ? want : most;
    if (parts < 1) parts = 1;
    const int span = ((K + parts - 1) / parts + 7) / 8 * 8;
    return {(K + span - 1) / span, span};
}

}  // namespace

size_t log_probs_workspace(int N, int K, int top)
{
    const Split s = split_rows(N, K);
    if (s.parts == 1) return 0;
    return round_up((size_t)N * s.parts * (3 + 2 * top) * 4, 256);
}

template <typename T>
static int log_probs_of(const T *z, ScoreArgs a, hipStream_t s)
{
    const dim3 one((unsigned)(((size_t)a.N + 3) / 4));
    const bool small = a.K <= 2048;
    if (small && a.top) hipLaunchKernelGGL((log_probs_kernel<T, 1, true>), one, dim3(256), 0, s, z, a);
    else if (small) hipLaunchKernelGGL((log_probs_kernel<T, 1, false>), one, dim3(256), 0, s, z, a);
    else if (a.top) hipLaunchKernelGGL((log_probs_kernel<T, 4, true>), dim3((unsigned)a.N * a.parts), dim3(256), 0, s, z, a);
    else hipLaunchKernelGGL((log_probs_kernel<T, 4, false>), dim3((unsigned)a.N * a.parts), dim3(256), 0, s, z, a);
    if (a.parts > 1) {
        if (a.top) hipLaunchKernelGGL((log_probs_join_kernel<T, true>), dim3(a.N), dim3(256), 0, s, z, a);
        else hipLaunchKernelGGL((log_probs_join_kernel<T, false>), dim3(a.N), dim3(256), 0, s, z, a);
    }
    return launch_status();
}

int log_probs(int dtype, int N, int K, size_t ldz, const void *z, const int32_t *labels, int top, float *logp, float *entropy,
              float *top_logp, int32_t *top_idx, float *stats, void *ws, hipStream_t s)
{
    const Split c = split_rows(N, K);
    ScoreArgs a = {N, K, top, c.parts, c.span, ldz, labels, logp, entropy, top_logp, stats, top_idx, nullptr, nullptr, nullptr};
    if (c.parts > 1) {
        const size_t n = (size_t)N * c.parts;
        a.part_sums = static_cast<float *>(ws);
        a.part_v = a.part_sums + n * 3;
        a.part_id = reinterpret_cast<int *>(a.part_v + n * top);
    }
    if (dtype == VGG_BF16) return log_probs_of(static_cast<const bf16_t *>(z), a, s);
    return log_probs_of(static_cast<const float *>(z), a, s);
}

int log_probs_bwd(int dtype, int N, int K, size_t ldz, const void *z, const int32_t *labels, const float *stats, const float *entropy,
                  const float *g_logp, const float *g_entropy, void *dz, size_t lddz, hipStream_t s)
{
    const Split c = split_rows(N, K);
    const GradArgs a = {N, K, c.span, c.parts, ldz, lddz, labels, stats, entropy, g_logp, g_entropy};
    const dim3 grid((unsigned)N * c.parts), block(256);
    if (dtype == VGG_BF16) hipLaunchKernelGGL(log_probs_bwd_kernel<bf16_t>, grid, block, 0, s, static_cast<const bf16_t *>(z), static_cast<bf16_t *>(dz), a);
    else hipLaunchKernelGGL(log_probs_bwd_kernel<float>, grid, block, 0, s, static_cast<const float *>(z), static_cast<float *>(dz), a);
    return launch_status();
}

}  // namespace vgg
