// Orthogonalised updates: Newton-Schulz products, and the optimiser step around them.
//
// X_0 = U / (|U| + eps), |U| the Frobenius norm; then, X of m x n with m <= n (a tall U is taken transposed),
//     G = X X^T,   X <- a X + (b G + c G G) X.
// The polynomial a s + b s^3 + c s^5 takes the singular values, all in [0, 1], towards 1, within [0, 1.21] throughout.
//
// Products are on the f16 matrix unit with fp32 sums.  X, G and P = b G + c G G are bounded (|X|, |G|, |P| <= 1.21, 1.47, 2.9), so
// that they are held times 2^14, below f16's largest, and need no other scale; f16 then keeps 11 bits of everything down to
// 2^-28.  PLANES = 2: a value is two f16 numbers, the nearest and what that leaves, 22 bits down to 2^-17 and 2^-39 below; hi hi + hi lo
// + lo hi leaves out 2^-22 of a product at most.  PLANES = 1 (updates that ask for VGG_BF16): operands are rounded to 11 bits.  The term a X takes an
// fp32 copy of X: a rounding to 11 bits there would grow 3.4-fold in every later step where X has no (or small) singular values, and where the
// matrix's norm is small beside eps all of X is small and a X nearly all of the result: f16 parts at a fixed scale lose it (130 x 514, a gradient
// times 2^-64: 73 % off).  In both the diagonals of G and P, which hold most of them, are kept apart in fp32 (zeros in the planes): with G = D + E,
//     (G G)_ij = (E E)_ij + (d_i + d_j) e_ij,   (G G)_ii = (E E)_ii + d_i^2,   (P X)_i = p_i X_i + (the rest of P) X.
// One plane is then, by an emulation of its roundings in 64 bits, 3.6e-4 to 6.5e-4 off for noise, 6e-5 to 5.6e-4 for few strong directions
// and 6e-4 to 1.6e-3 for singular values over six decades (64 x 576 to 1000 x 1003), against up to 2.4e-3 with the diagonals rounded.
//
// X, G and P lie in columns of 128 bytes to a row: [column][row][64 elements], or [32 elements of the first plane, 32 of the
// second], so that what a workgroup copies for a stage of its contraction is contiguous.  X's fp32 copy lies in columns of 32.
// G and G G contract along rows of both operands; P X takes X's columns, which LDS hands out transposed (ds_read_b64_tr_b16), so
// that X is kept once.  X is padded with zeros to whole tiles.  G and P are symmetric: the tiles on and below the diagonal are
// formed, over a few ranges of the contraction where they are too few to fill the chip, and a second kernel adds the ranges in
// order and mirrors them (in the product kernel's own end, where there is one range: no faster).
#include "common.h"
#include "plans.h"

#include <type_traits>

namespace vgg {

namespace {

typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 half_t;

constexpr float kA = 3.4445f, kB = -4.7750f, kC = 2.0315f, kEps = 1e-7f;
constexpr float kUp = 16384.f, kDown = 1.f / 16384.f;   // 2^14
constexpr int kParts = 1024;                            // partial sums of squares of a matrix

// Element k of a row of K-blocks of 32 with PL planes.
template <int PL> __device__ __forceinline__ size_t at_plane(int k, int plane) { return (size_t)(k >> 5) * (32 * PL) + plane * 32 + (k & 31); }
// The same in a matrix of `rows` (padded) rows, columns of 128 bytes.
template <int PL> __device__ __forceinline__ size_t at_column(int rows, int i, int k)
{
    constexpr int C = 64 / PL;
    return ((size_t)(k / C) * rows + i) * 64 + k % C;
}
__device__ __forceinline__ size_t at_x32(int rows, int i, int j) { return ((size_t)(j >> 5) * rows + i) * 32 + (j & 31); }

// ----------------------------------------------------------------------------------- momentum and the norm
// Squares are summed in 64 bits: they neither overflow nor vanish.  Bound by the read (7 x 512 x 4608, bf16: 13 to 16 us for 33 MB, from the launch on; with a
// step of the momentum, 4096 x 25088: 208 us for 1.2 GB, 5.9 TB/s).
__device__ __forceinline__ double block_sum(double v)
{
    __shared__ double red[4];
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) v += __shfl_xor(v, o, kWave);
    if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = v;
    __syncthreads();
    return red[0] + red[1] + red[2] + red[3];
}

// What a matrix is divided by, as a factor: in 64 bits, in which it is none of fp32's zeros for any norm; NaN for what is not finite.
__device__ __forceinline__ double scale_of(double norm2) { return norm2 < (double)INFINITY ? 1. / (sqrt(norm2) + (double)kEps) : (double)NAN; }

// momentum <- mu momentum + grad; U = grad + mu momentum (nesterov) or momentum.
struct Source {
    const void *x;         // the matrix itself (no momentum), or the gradient
    float *momentum;       // null: x is the matrix
    float mu;
    int nesterov;
};
template <typename T> __device__ __forceinline__ float source_at(const Source &s, size_t i)
{
    const float g = Elem<T>::load(static_cast<const T *>(s.x) + i);
    if (!s.momentum) return g;
    const float m = s.momentum[i];     // (stepped already)
    return s.nesterov ? __builtin_fmaf(s.mu, m, g) : m;
}

// 16 bytes from or to an address that is a multiple of an element's size only; a thread's V elements at a time, the first n of them.
template <typename T> struct __attribute__((packed, aligned(sizeof(T)))) Loose { T v[16 / sizeof(T)]; };
template <typename T, int V> __device__ __forceinline__ void load_some(const T *p, int n, float (&v)[V])
{
    constexpr int L = 16 / (int)sizeof(T);
    if (n >= V) {
#pragma unroll
        for (int h = 0; h < V / L; ++h) {
            const Loose<T> l = *reinterpret_cast<const Loose<T> *>(p + h * L);
#pragma unroll
            for (int k = 0; k < L; ++k) v[h * L + k] = Elem<T>::load(&l.v[k]);
        }
    } else
#pragma unroll
        for (int k = 0; k < V; ++k) v[k] = k < n ? Elem<T>::load(p + k) : 0.f;
}
template <typename T, int V> __device__ __forceinline__ void store_some(T *p, int n, const float (&v)[V])
{
    constexpr int L = 16 / (int)sizeof(T);
    if (n >= V) {
#pragma unroll
        for (int h = 0; h < V / L; ++h) {
            Loose<T> l;
#pragma unroll
            for (int k = 0; k < L; ++k) Elem<T>::store(&l.v[k], v[h * L + k]);
            *reinterpret_cast<Loose<T> *>(p + h * L) = l;
        }
    } else
#pragma unroll
        for (int k = 0; k < V; ++k)
            if (k < n) Elem<T>::store(p + k, v[k]);
}

constexpr int kNormLoads = 4;                           // of 16 bytes, in flight
template <typename T> constexpr int kNormLot = 256 * kNormLoads * 16 / (int)sizeof(T);   // elements of a workgroup at a time
inline int norm_parts(size_t count, size_t lot) { return (int)((count + lot - 1) / lot < (size_t)kParts ? (count + lot - 1) / lot : (size_t)kParts); }
template <typename T>
__global__ __launch_bounds__(256) void muon_norm_kernel(Source s, double *__restrict__ part, size_t count)
{
    constexpr int U = kNormLoads, V = 16 / (int)sizeof(T);
    const size_t base = (size_t)blockIdx.y * count, step = (size_t)gridDim.x * 256 * V;
    const T *x = static_cast<const T *>(s.x) + base;
    float *mom = s.momentum ? s.momentum + base : nullptr;
    double sum = 0;
    for (size_t i = ((size_t)blockIdx.x * 256 + threadIdx.x) * V; i < count; i += U * step) {
        float u[U][V];
        auto left = [&](int k) __attribute__((always_inline)) {
            const size_t at = i + k * step;
            return at >= count ? 0 : count - at < (size_t)V ? (int)(count - at) : V;
        };
#pragma unroll
        for (int k = 0; k < U; ++k) load_some<T, V>(x + i + k * step, left(k), u[k]);
        if (mom) {
            float m[U][V];
#pragma unroll
            for (int k = 0; k < U; ++k) load_some<float, V>(mom + i + k * step, left(k), m[k]);
#pragma unroll
            for (int k = 0; k < U; ++k) {
#pragma unroll
                for (int j = 0; j < V; ++j) {
                    m[k][j] = __builtin_fmaf(s.mu, m[k][j], u[k][j]);
                    u[k][j] = s.nesterov ? __builtin_fmaf(s.mu, m[k][j], u[k][j]) : m[k][j];
                }
                float *to = mom + i + k * step;
                store_some<float, V>(to, left(k), m[k]);
            }
        }
#pragma unroll
        for (int k = 0; k < U; ++k)
#pragma unroll
            for (int j = 0; j < V; ++j) sum = __builtin_fma((double)u[k][j], (double)u[k][j], sum);
    }
    sum = block_sum(sum);
    if (threadIdx.x == 0) part[blockIdx.y * kParts + blockIdx.x] = sum;
}

// What a call works on.
struct Layout {
    int rows, cols, m, n, mp, np, tall, tile, parts, batch;   // tile: of the products, 128 or 256, which mp and np are multiples of
    int splits[2];         // of the Gram matrix and its square
    float *x32;            // [batch][np / 32][mp][32]
    half_t *x[2];          // [batch][columns][mp][64], of mp x np
    half_t *g, *p;         // [batch][columns][mp][64], of mp x mp, zero diagonals
    float *gd, *pd;        // [batch][mp], the diagonals
    float *sums;           // [batch][tiles][splits][tile][tile]
    double *part;          // [batch][kParts]
};

// X_0 in all its forms, zeros where they are padded.  A workgroup: 64 x 64 of the padded X, eight consecutive elements to a thread.
// Bound by what it writes (7 x 512 x 4608, bf16: 34 us for 165 MB, read and written).
template <typename T, int PL>
__global__ __launch_bounds__(256) void muon_start_kernel(Source s, Layout L)
{
    __shared__ float tile[64][65];
    const int b = blockIdx.z, i0 = blockIdx.y * 64, j0 = blockIdx.x * 64, t8 = (threadIdx.x & 7) * 8, ty = threadIdx.x >> 3;
    const size_t base = (size_t)b * L.rows * L.cols;
    // the source is read along its own rows
    float v[2][8];
#pragma unroll
    for (int k = 0; k < 2; ++k) {
        const int r = (L.tall ? j0 : i0) + ty + 32 * k, c = (L.tall ? i0 : j0) + t8, n = r < L.rows ? L.cols - c : 0;
        const size_t at = base + (size_t)r * L.cols + c;
        load_some<T, 8>(static_cast<const T *>(s.x) + at, n, v[k]);
        if (s.momentum) {                              // (stepped already)
            float m[8];
            load_some<float, 8>(s.momentum + at, n, m);
#pragma unroll
            for (int j = 0; j < 8; ++j) v[k][j] = s.nesterov ? __builtin_fmaf(s.mu, m[j], v[k][j]) : m[j];
        }
    }
    double norm2 = 0;
    for (int k = threadIdx.x; k < L.parts; k += 256) norm2 += L.part[b * kParts + k];
    norm2 = block_sum(norm2);
    const double by = scale_of(norm2);
    if (L.tall) {
#pragma unroll
        for (int k = 0; k < 2; ++k)
#pragma unroll
            for (int j = 0; j < 8; ++j) tile[t8 + j][ty + 32 * k] = v[k][j];
        __syncthreads();
#pragma unroll
        for (int k = 0; k < 2; ++k)
#pragma unroll
            for (int j = 0; j < 8; ++j) v[k][j] = tile[ty + 32 * k][t8 + j];
    }
    const size_t mn = (size_t)L.mp * L.np;
    half_t *x = L.x[0] + b * mn * PL;
#pragma unroll
    for (int k = 0; k < 2; ++k) {
        const int i = i0 + ty + 32 * k, j = j0 + t8;
        float w[8];
        f16x8 hi, lo;
#pragma unroll
        for (int q = 0; q < 8; ++q) {
            w[q] = (float)(v[k][q] * by);
            hi[q] = (half_t)(w[q] * kUp);
            lo[q] = (half_t)(w[q] * kUp - (float)hi[q]);
        }
        const size_t at = at_column<PL>(L.mp, i, j);
        *reinterpret_cast<f16x8 *>(x + at) = hi;
        if constexpr (PL == 2) *reinterpret_cast<f16x8 *>(x + at + 32) = lo;
        float *x32 = L.x32 + b * mn + at_x32(L.mp, i, j);
        *reinterpret_cast<f32x4 *>(x32) = f32x4{w[0], w[1], w[2], w[3]};
        *reinterpret_cast<f32x4 *>(x32 + 4) = f32x4{w[4], w[5], w[6], w[7]};
    }
}

// -------------------------------------------------------------------------------------------------- products
enum { kGram, kPoly, kApply, kLast };


// What the last product writes: X itself, or the step that it makes.
struct Target {
    void *out;             // [batch][rows][cols], or null:
    float *theta;          // theta <- keep theta - rate X
    float keep, rate;
};

typedef __attribute__((address_space(3))) char lds_char;

// Workgroups go round the eight XCDs; each takes a run of the work, so that neighbours share their operands in its L2.
__device__ __forceinline__ int spread(int id, int count)
{
    const int per = count >> 3, more = count & 7, xcd = id & 7, at = id >> 3;
    return xcd * per + (xcd < more ? xcd : more) + at;
}

// Eight consecutive elements of what the last product writes, the first n of them.
template <typename T> __device__ __forceinline__ void write_some(const Target &out, size_t at, int n, const f32x4 (&w)[2])
{
    if (out.theta) {
        float *to = out.theta + at;
        float t[8];
        load_some<float, 8>(to, n, t);
#pragma unroll
        for (int q = 0; q < 8; ++q) t[q] = __builtin_fmaf(-out.rate, w[q / 4][q % 4], out.keep * t[q]);
        store_some<float, 8>(to, n, t);
    } else {
        float t[8];
#pragma unroll
        for (int q = 0; q < 8; ++q) t[q] = w[q / 4][q % 4];
        store_some<T, 8>(static_cast<T *>(out.out) + at, n, t);
    }
}

// A workgroup of eight waves (2 x 4): TILE x TILE of C = A B^T (kGram, kPoly) or A B (kApply, kLast).  A stage is 128 bytes of
// every row of A (64 contraction indices, or 32 in two planes), and as many rows or bytes of B; STAGES of them in LDS, all but one
// on their way (128 KB, one workgroup to a compute unit).  A 16-byte segment s of a row r of A lies at s ^ (r / 2 % 8), so that
// sixteen rows of one segment are in different banks; the two 64-byte blocks of a row r of
// B that is read transposed change places where r / 2 is odd, for the four rows that sixteen lanes read.  256 x 256 tiles take 2/3 of the
// LDS traffic of 128 x 128 ones, and four times the work.  Large products are bound by the matrix unit and its power (4096 x 25088, two
// planes: G in 1.02 ms, 1.33 PFLOP/s of f16 products, pipes busy 0.73; P X in 2.1 ms, 1.2 PFLOP/s), smaller ones by what P X moves
// between the eight L2s and memory (two planes: 7 x 512 x 4608: 72 to 87 us for 270 MB; 1000 x 4096: 32 us for 98 MB) and by their
// beginnings and ends, not by LDS or barriers: four waves to a tile are 2 to 5 % slower, stages twice as long or what the end
// reads asked for at the start make no difference, two workgroups to a compute unit 4 % for many rounds and -3 % for one.
template <typename T, int PL, int MODE, int TILE>
__global__ __launch_bounds__(512) void muon_product_kernel(Layout L, int from, Target out)
{
    extern __shared__ __align__(16) char lds[];   // [STAGES][A, B: TILE x 128 bytes each]
    constexpr bool TR = MODE == kApply || MODE == kLast;
    constexpr int STAGES = TILE == 256 ? 2 : 4, HALF = TILE * 128, BX = TILE / 64, BY = TILE / 128, COPIES = TILE / 64, KS = 64 / PL;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, b = blockIdx.y;
    const int mt = L.mp / TILE, nt = L.np / TILE;
    int ti, tj, split = 0;
    const int unit = spread(blockIdx.x, gridDim.x);
    if constexpr (TR) {                           // eight tiles down, then one to the right
        const int wide = 8 * nt, group = unit / wide, in = unit - group * wide, rows = mt - group * 8 < 8 ? mt - group * 8 : 8;
        ti = group * 8 + in % rows;
        tj = in / rows;
    } else {                                      // tiles on and below the diagonal, row by row
        const int tiles = mt * (mt + 1) / 2;
        split = unit / tiles;
        const int t = unit - split * tiles;
        ti = (int)((sqrtf(8.f * t + 1.f) - 1.f) * 0.5f);
        while ((ti + 1) * (ti + 2) / 2 <= t) ++ti;
        while (ti * (ti + 1) / 2 > t) --ti;
        tj = t - ti * (ti + 1) / 2;
    }
    const size_t mm = (size_t)L.mp * L.mp, mn = (size_t)L.mp * L.np;
    const int K = MODE == kGram ? L.np : L.mp, all = K / KS;
    const int splits = TR ? 1 : L.splits[MODE];
    const int s0 = (int)((long)all * split / splits), stages = (int)((long)all * (split + 1) / splits) - s0;
    const half_t *pa = MODE == kGram ? L.x[from] + b * mn * PL : MODE == kPoly ? L.g + b * mm * PL : L.p + b * mm * PL;
    const size_t column = (size_t)L.mp * 128;     // bytes
    const char *ga = reinterpret_cast<const char *>(pa) + s0 * column + (size_t)ti * TILE * 128;
    const char *gb = TR ? reinterpret_cast<const char *>(L.x[from] + b * mn * PL) + (size_t)(tj * TILE / KS) * column
                        : reinterpret_cast<const char *>(pa) + s0 * column + (size_t)tj * TILE * 128;
    const unsigned lds0 = __builtin_amdgcn_readfirstlane((unsigned)(uintptr_t)(lds_char *)lds + wave * 1024);

    // where this thread's copies come from
    const char *src_a[COPIES], *src_b[COPIES];
#pragma unroll
    for (int q = 0; q < COPIES; ++q) {
        const int at = (q * 512 + (int)threadIdx.x) * 16, r = at >> 7, seg = ((at >> 4) & 7) ^ (r >> 1 & 7);
        src_a[q] = ga + r * 128 + seg * 16;
        if constexpr (TR) {                        // [TILE / KS columns][KS rows][128 bytes]
            const int k = r % KS;
            src_b[q] = gb + r / KS * column + k * 128 + ((at & 127) ^ (k >> 1 & 1) << 6);
        } else
            src_b[q] = gb + r * 128 + seg * 16;
    }
    const size_t step_b = TR ? (size_t)KS * 128 : column;
    int slot = 0;
    auto copy_one = [&](int n) __attribute__((always_inline)) {      // of a stage's 2 COPIES
        const int q = n >> 1;
        if (n & 1) {
            copy16_to_lds(lds0 + slot * (2 * HALF) + HALF + q * 8192, src_b[q]);
            src_b[q] += step_b;
        } else {
            copy16_to_lds(lds0 + slot * (2 * HALF) + q * 8192, src_a[q]);
            src_a[q] += column;
        }
        if (n == 2 * COPIES - 1) slot = slot + 1 == STAGES ? 0 : slot + 1;
    };

    f32x16 acc[BX][BY] = {};
    const int wi = (wave >> 2) * (TILE / 2), wj = (wave & 3) * (TILE / 4);
    // this lane's part of a fragment's address: rows (of A, of B by rows), or the transposed read's
    const int arow = wi + (lane & 31), brow = wj + (lane & 31), rx = lane >> 1 & 7;
    const int s16 = lane & 15, tr_k = 8 * (lane >> 5) + (s16 >> 2), tr_x = s16 >> 3, tr_at = (lane >> 4 & 1) * 32 + (s16 & 3) * 8;
    // A stage is KK steps of 16 contraction indices.  Between a step's products the next step's fragments are read, and in a stage's
    // last step, after the barrier, the next stage's first fragments and the copies of a stage to come: none of it would hide
    // behind products in a block of its own, since the barrier lines the waves up.
    constexpr int KK = 4 / PL, M = (PL == 2 ? 3 : 1) * BX * BY, R = PL * (BX + BY);
    struct Fragments { f16x8 a[PL][BX], b[PL][BY]; };
    auto read_one = [&](int use, int k, int n, Fragments &f) __attribute__((always_inline)) {
        const char *A = lds + use * (2 * HALF), *B = A + HALF;
        const int p = n / (BX + BY), q = n % (BX + BY), r = q - BX, seg = p * 4 + k * 2 + (lane >> 5);
        if (q < BX) f.a[p][q] = *reinterpret_cast<const f16x8 *>(A + (arow + q * 32) * 128 + ((seg ^ rx) << 4));
        else if constexpr (TR) {
            typedef _Float16 f16x4 __attribute__((ext_vector_type(4)));
            typedef __fp16 fp16x4 __attribute__((__vector_size__(8)));
            typedef __attribute__((address_space(3))) fp16x4 lds_f16x4;
            const int c = ((wj >> 5) + r) * PL + p;      // 64-byte block of a row
            const char *at = B + (c >> 1) * (KS * 128) + (k * 16 + tr_k) * 128 + (((c & 1) ^ tr_x) << 6) + tr_at;
            const auto lo = __builtin_amdgcn_ds_read_tr16_b64_v4f16((lds_f16x4 *)at);
            const auto hi = __builtin_amdgcn_ds_read_tr16_b64_v4f16((lds_f16x4 *)(at + 4 * 128));
            f.b[p][r] = __builtin_shufflevector(__builtin_bit_cast(f16x4, lo), __builtin_bit_cast(f16x4, hi), 0, 1, 2, 3, 4, 5, 6, 7);
        } else
            f.b[p][r] = *reinterpret_cast<const f16x8 *>(B + (brow + r * 32) * 128 + ((seg ^ rx) << 4));
    };
    Fragments f[2];
    int use = 0;
    // One stage; READ: there is a next one, COPY: there is one to be copied.
    auto stage = [&](auto READ, auto COPY) __attribute__((always_inline)) {
        constexpr bool reads = decltype(READ)::value, copies = decltype(COPY)::value;
#pragma unroll
        for (int k = 0; k < KK; ++k) {
            const bool last = k + 1 == KK;
            const int lead = last ? M / 3 : 0, tasks = last ? (reads ? R : 0) + (copies ? 2 * COPIES : 0) : R;
            const Fragments &g = f[k & 1];
            Fragments &next = f[(k + 1) & 1];
#pragma unroll
            for (int i = 0; i < M; ++i) {
                // (the blocks' sums take one product each in turn: a sum's next product waits for its last)
                const int p = PL == 2 ? i / (BX * BY) : 2, x = i % (BX * BY) / BY, y = i % BY;
                if (last && reads && i == lead) {
                    // The next stage's copies have landed (those of later ones may be on their way), and all waves have read what they
                    // need of this one, whose place the next copies take.
                    asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" : : "n"(copies ? (STAGES - 2) * 2 * COPIES : 0) : "memory");
                    use = use + 1 == STAGES ? 0 : use + 1;
                }
                // (TR: the block's transpose, for four consecutive columns of X in a lane)
                if constexpr (TR) acc[x][y] = __builtin_amdgcn_mfma_f32_32x32x16_f16(g.b[p == 1][y], g.a[p == 0][x], acc[x][y], 0, 0, 0);
                else acc[x][y] = __builtin_amdgcn_mfma_f32_32x32x16_f16(g.a[p == 0][x], g.b[p == 1][y], acc[x][y], 0, 0, 0);
                if (i >= lead)
#pragma unroll
                    for (int n = (i - lead) * tasks / (M - lead); n < (i - lead + 1) * tasks / (M - lead); ++n) {
                        if (!last) read_one(use, k + 1, n, next);
                        else if (n < R) read_one(use, 0, n, next);
                        else copy_one(n - R);
                    }
                __builtin_amdgcn_sched_barrier(0);
            }
        }
    };
#pragma unroll
    for (int k = 0; k < STAGES; ++k)
        if (k < stages)
#pragma unroll
            for (int n = 0; n < 2 * COPIES; ++n) copy_one(n);
    if (stages >= STAGES) asm volatile("s_waitcnt vmcnt(%0)\n\ts_barrier" : : "n"((STAGES - 1) * 2 * COPIES) : "memory");
    else asm volatile("s_waitcnt vmcnt(0)\n\ts_barrier" : : : "memory");
#pragma unroll
    for (int n = 0; n < R; ++n) read_one(0, 0, n, f[0]);
    int st = 0;
    for (; st + STAGES < stages; ++st) stage(std::true_type{}, std::true_type{});
    for (; st + 1 < stages; ++st) stage(std::true_type{}, std::false_type{});
    stage(std::false_type{}, std::false_type{});

    // Value v of a block: row 8 (v / 4) + 4 (lane / 32) + v % 4, column lane % 32.
    if constexpr (!TR) {
        const int row0 = wi + 4 * (lane >> 5), col0 = wj + (lane & 31);
        float *c = L.sums + (((size_t)b * (mt * (mt + 1) / 2) + ti * (ti + 1) / 2 + tj) * splits + split) * (TILE * TILE);
#pragma unroll
        for (int x = 0; x < BX; ++x)
#pragma unroll
            for (int y = 0; y < BY; ++y)
#pragma unroll
                for (int v = 0; v < 16; ++v) c[(row0 + x * 32 + 8 * (v >> 2) + (v & 3)) * TILE + col0 + y * 32] = acc[x][y][v];
    } else {
        // A wave's 32 rows and all its columns go through LDS, in which it has a place of its own once no wave reads operands any more:
        // then a lane has eight consecutive columns of X, 16 bytes of f16, and what it reads and writes are runs of 64 or 128 bytes.
        constexpr int COLS = BY * 32, STRIDE = COLS * 4 + 16, LANES = COLS / 8, CHUNKS = COLS / 16;   // lanes of a row; a lane's chunks
        char *turned = lds + wave * (32 * STRIDE);
        asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" : : : "memory");
        auto wave_sync = [&]() __attribute__((always_inline)) {
            __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
            __builtin_amdgcn_wave_barrier();
            __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
        };
        const int row = lane / LANES, c8 = lane % LANES * 8, j = tj * TILE + wj + c8;
#pragma unroll
        for (int x = 0; x < BX; ++x) {
            const int i = ti * TILE + wi + x * 32 + row;                 // and every (64 / LANES)-th further one
            float old[CHUNKS][8], pd[CHUNKS];
#pragma unroll
            for (int k = 0; k < CHUNKS; ++k) {
                pd[k] = kA + L.pd[(size_t)b * L.mp + i + k * (64 / LANES)];
                const float *from32 = L.x32 + b * mn + at_x32(L.mp, i + k * (64 / LANES), j);
                const f32x4 lo = *reinterpret_cast<const f32x4 *>(from32), hi = *reinterpret_cast<const f32x4 *>(from32 + 4);
#pragma unroll
                for (int q = 0; q < 4; ++q) { old[k][q] = lo[q]; old[k][4 + q] = hi[q]; }
            }
#pragma unroll
            for (int y = 0; y < BY; ++y)
#pragma unroll
                for (int q = 0; q < 4; ++q)
                    *reinterpret_cast<f32x4 *>(turned + (lane & 31) * STRIDE + (y * 32 + 8 * q + 4 * (lane >> 5)) * 4) =
                        f32x4{acc[x][y][4 * q], acc[x][y][4 * q + 1], acc[x][y][4 * q + 2], acc[x][y][4 * q + 3]};
            wave_sync();
#pragma unroll
            for (int k = 0; k < CHUNKS; ++k) {
                f32x4 *here = reinterpret_cast<f32x4 *>(turned + (row + k * (64 / LANES)) * STRIDE + c8 * 4);
                f32x4 w[2] = {here[0], here[1]};
#pragma unroll
                for (int q = 0; q < 8; ++q) w[q / 4][q % 4] = __builtin_fmaf(pd[k], old[k][q], w[q / 4][q % 4] * (kDown * kDown));
                if constexpr (MODE == kApply) {
                    half_t *to = L.x[1 - from] + b * mn * PL + at_column<PL>(L.mp, i + k * (64 / LANES), j);
                    f16x8 h, r;
#pragma unroll
                    for (int q = 0; q < 8; ++q) {
                        const float c = w[q / 4][q % 4] * kUp;
                        h[q] = (half_t)c;
                        r[q] = (half_t)(c - (float)h[q]);
                    }
                    *reinterpret_cast<f16x8 *>(to) = h;
                    if constexpr (PL == 2) *reinterpret_cast<f16x8 *>(to + 32) = r;
                    f32x4 *to32 = reinterpret_cast<f32x4 *>(L.x32 + b * mn + at_x32(L.mp, i + k * (64 / LANES), j));
                    to32[0] = w[0];
                    to32[1] = w[1];
                } else if (L.tall) {
                    here[0] = w[0];
                    here[1] = w[1];
                } else if (i + k * (64 / LANES) < L.m) {
                    write_some<T>(out, (size_t)b * L.rows * L.cols + (size_t)(i + k * (64 / LANES)) * L.cols + j, L.n - j, w);
                }
            }
            wave_sync();
            if constexpr (MODE == kLast)
                if (L.tall) {                                            // along the rows of what is written: columns of X
                    const int ic = ti * TILE + wi + x * 32 + (lane & 31), jc = tj * TILE + wj + (lane >> 5);
#pragma unroll
                    for (int h = 0; h < COLS / 2; h += 8) {
                        float w[8];
                        size_t o[8];
                        bool there[8];
#pragma unroll
                        for (int k = 0; k < 8; ++k) {
                            w[k] = *reinterpret_cast<const float *>(turned + (lane & 31) * STRIDE + ((lane >> 5) + 2 * (h + k)) * 4);
                            there[k] = ic < L.m && jc + 2 * (h + k) < L.n;
                            o[k] = there[k] ? (size_t)b * L.rows * L.cols + (size_t)(jc + 2 * (h + k)) * L.cols + ic : 0;
                        }
                        if (out.theta) {
                            float t[8];
#pragma unroll
                            for (int k = 0; k < 8; ++k) t[k] = there[k] ? out.theta[o[k]] : 0.f;
#pragma unroll
                            for (int k = 0; k < 8; ++k)
                                if (there[k]) out.theta[o[k]] = __builtin_fmaf(-out.rate, w[k], out.keep * t[k]);
                        } else
#pragma unroll
                            for (int k = 0; k < 8; ++k)
                                if (there[k]) Elem<T>::store(static_cast<T *>(out.out) + o[k], w[k]);
                    }
                    wave_sync();
                }
        }
    }
}

// The ranges' sums to G, or to P = b G + c G G: 32 x 32 of a tile to a workgroup, and its mirror image.  5 us for m up to 1000, most of it
// the launch; 32 to 43 us at m = 4096.
template <int PL, int MODE, int TILE>
__global__ __launch_bounds__(256) void muon_symmetric_kernel(Layout L)
{
    __shared__ float turned[32][33];
    constexpr int Q = TILE / 32;
    const int b = blockIdx.y, t = blockIdx.x / (Q * Q), in = blockIdx.x - t * (Q * Q);
    int ti = (int)((sqrtf(8.f * t + 1.f) - 1.f) * 0.5f);
    while ((ti + 1) * (ti + 2) / 2 <= t) ++ti;
    while (ti * (ti + 1) / 2 > t) --ti;
    const int tj = t - ti * (ti + 1) / 2, mt = L.mp / TILE, splits = L.splits[MODE];
    const int i0 = ti * TILE + in / Q * 32, j0 = tj * TILE + in % Q * 32;
    const size_t mm = (size_t)L.mp * L.mp;
    const int tx = threadIdx.x & 7, ty = threadIdx.x >> 3, i = i0 + ty, j = j0 + tx * 4;
    const float *c = L.sums + ((size_t)b * (mt * (mt + 1) / 2) + t) * splits * (TILE * TILE) + (size_t)(in / Q * 32 + ty) * TILE + in % Q * 32 + tx * 4;
    half_t *to = (MODE == kGram ? L.g : L.p) + b * mm * PL;
    const half_t *g = L.g + b * mm * PL + at_column<PL>(L.mp, i, j);
    float *gd = L.gd + (size_t)b * L.mp, *pd = L.pd + (size_t)b * L.mp;
    typedef half_t f16x4 __attribute__((ext_vector_type(4)));
    auto store = [&](int i, int j, const f32x4 &v) __attribute__((always_inline)) {
        half_t *row = to + at_column<PL>(L.mp, i, j);
        f16x4 h, l;
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            const float w = i == j + k ? 0.f : v[k];
            h[k] = (half_t)w;
            l[k] = (half_t)(w - (float)h[k]);
        }
        *reinterpret_cast<f16x4 *>(row) = h;
        if constexpr (PL == 2) *reinterpret_cast<f16x4 *>(row + 32) = l;
    };
    f32x4 v = {0.f, 0.f, 0.f, 0.f};
    constexpr int U = 8;                           // sums on their way
    for (int s = 0; s < splits; s += U) {
        f32x4 u[U];
#pragma unroll
        for (int k = 0; k < U; ++k) u[k] = s + k < splits ? *reinterpret_cast<const f32x4 *>(c + (size_t)(s + k) * (TILE * TILE)) : f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int k = 0; k < U; ++k) v += u[k];
    }
    v *= kDown;
    if constexpr (MODE == kGram) {
#pragma unroll
        for (int k = 0; k < 4; ++k)
            if (i == j + k) gd[i] = v[k] * kDown;
    } else {
        const float di = gd[i];
        f32x4 e = __builtin_convertvector(*reinterpret_cast<const f16x4 *>(g), f32x4);
        if constexpr (PL == 2) e += __builtin_convertvector(*reinterpret_cast<const f16x4 *>(g + 32), f32x4);
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            if (i == j + k) pd[i] = __builtin_fmaf(kC, __builtin_fmaf(di, di, v[k] * kDown), kB * di);
            v[k] = __builtin_fmaf(kC, v[k], __builtin_fmaf(kC, di + gd[j + k], kB) * e[k]);
        }
    }
    store(i, j, v);
    if (ti == tj) return;                          // (all of a diagonal tile is formed)
#pragma unroll
    for (int k = 0; k < 4; ++k) turned[tx * 4 + k][ty] = v[k];
    __syncthreads();
#pragma unroll
    for (int k = 0; k < 4; ++k) v[k] = turned[ty][tx * 4 + k];
    store(j0 + ty, i0 + tx * 4, v);
}

// ------------------------------------------------------------------------------------------- matrices of few rows
// Up to 64 rows (of X), and the columns that a workgroup of eight waves has: X in registers, in the layout of the products' results
// (32 columns w + 8 c to wave w), X^T's planes, G's and P's in LDS.  By columns, a lane's four consecutive rows of a result are one
// LDS store; P X then reads columns of X as they lie, and G reads its rows transposed.  G and G G are 16 blocks of 16 x 16, two to
// a wave; the sum (i, j) is stored as (j, i), the same by symmetry and four in a row again.
template <typename T, int PL, int CB>
struct FewRows {
    typedef half_t f16x4 __attribute__((ext_vector_type(4)));
    static constexpr int S = row_stride(PL), W = 8, Q = 16 / W;   // waves; blocks of G of a wave
    int m, n, blocks, first, lane, wave, half, col, i_step, j_step;   // blocks of 32 columns: this workgroup's, from `first` on
    char *X, *G, *P;
    float *gd, *pd;
    double *red;
    float x[CB][2][16];    // (r, v) of column block c: row 32 r + 8 (v / 4) + 4 half + v % 4, column 32 (wave + W c) + col
    f32x4 acc[Q];          // G or G G: value v is (16 bi + 4 quarter + v, 16 (bj + q) + r16)

    __device__ __forceinline__ FewRows(char *lds, int rows, int cols, int first_block, int most_blocks)
    {
        const bool tall = rows > cols;
        m = tall ? cols : rows;
        n = tall ? rows : cols;
        first = first_block;
        blocks = (n + 31) / 32 - first;
        if (blocks > most_blocks) blocks = most_blocks;
        lane = threadIdx.x & 63;
        wave = threadIdx.x >> 6;
        half = lane >> 5;
        col = lane & 31;
        i_step = tall ? 1 : cols;
        j_step = tall ? cols : 1;
        X = lds;
        G = X + blocks * 32 * S;
        P = G + kFewRows * S;
        gd = reinterpret_cast<float *>(P + kFewRows * S);
        pd = gd + 64;
        red = reinterpret_cast<double *>(pd + 64);
    }
    // The place of element (c, r, v) in a matrix as the caller keeps it; that of an element that is there, where this one is not.
    __device__ __forceinline__ unsigned place(int c, int r, int v, bool &there) const
    {
        const int i = r * 32 + 8 * (v >> 2) + 4 * half + (v & 3), j = (first + wave + W * c) * 32 + col;
        there = i < m && j < n && wave + W * c < blocks;
        return there ? (unsigned)i * i_step + (unsigned)j * j_step : 0u;   // (at most 2^28)
    }
    // Places are found again where they are used next: they would fill the registers in between.
    __device__ __forceinline__ void forget_places() { asm volatile("" : "+v"(col), "+v"(half)); }
    // (32-bit offsets from addresses that the workgroup shares)
    template <typename U> static __device__ __forceinline__ U &element(U *p, unsigned at)
    {
        return *reinterpret_cast<U *>(reinterpret_cast<uintptr_t>(p) + at * (unsigned)sizeof(U));
    }
    // Four consecutive elements k.. of a row, scaled, into its planes; and back.
    static __device__ __forceinline__ void put4(char *row, int k, const f32x4 &v)
    {
        f16x4 h, l;
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            h[q] = (half_t)v[q];
            l[q] = (half_t)(v[q] - (float)h[q]);
        }
        char *to = row + at_plane<PL>(k, 0) * 2;
        *reinterpret_cast<f16x4 *>(to) = h;
        if constexpr (PL == 2) *reinterpret_cast<f16x4 *>(to + 64) = l;
    }
    static __device__ __forceinline__ f32x4 get4(const char *row, int k)
    {
        const char *from = row + at_plane<PL>(k, 0) * 2;
        f32x4 v = __builtin_convertvector(*reinterpret_cast<const f16x4 *>(from), f32x4);
        if constexpr (PL == 2) v += __builtin_convertvector(*reinterpret_cast<const f16x4 *>(from + 64), f32x4);
        return v;
    }
    __device__ __forceinline__ void put_x() const
    {
#pragma unroll
        for (int c = 0; c < CB; ++c)
            if (wave + W * c < blocks)
#pragma unroll
                for (int r = 0; r < 2; ++r)
#pragma unroll
                    for (int q = 0; q < 4; ++q) {
                        const f32x4 v = {x[c][r][4 * q], x[c][r][4 * q + 1], x[c][r][4 * q + 2], x[c][r][4 * q + 3]};
                        put4(X + ((wave + W * c) * 32 + col) * S, r * 32 + 8 * q + 4 * half, v * kUp);
                    }
    }
    static __device__ __forceinline__ f32x4 mfma16(const f16x8 (&fa)[PL], const f16x8 (&fb)[PL], f32x4 acc)
    {
        if constexpr (PL == 2) {
            acc = __builtin_amdgcn_mfma_f32_16x16x32_f16(fa[1], fb[0], acc, 0, 0, 0);
            acc = __builtin_amdgcn_mfma_f32_16x16x32_f16(fa[0], fb[1], acc, 0, 0, 0);
        }
        return __builtin_amdgcn_mfma_f32_16x16x32_f16(fa[0], fb[0], acc, 0, 0, 0);
    }
    struct Rows { f16x8 a[PL], b[Q][PL]; };
    __device__ __forceinline__ void clear()
    {
#pragma unroll
        for (int q = 0; q < Q; ++q) acc[q] = f32x4{0.f, 0.f, 0.f, 0.f};
    }
    // acc <- X X^T of the workgroup's columns, this wave's blocks
    __device__ __forceinline__ void gram()
    {
        const int bi = wave / (W / 4), bj = wave % (W / 4) * Q, r16 = lane & 15, quarter = lane >> 4;
        auto columns = [&](int jb, Rows &f) __attribute__((always_inline)) {        // 32 columns of X's rows
            auto rows_of = [&](int b, f16x8 (&f)[PL]) __attribute__((always_inline)) {
#pragma unroll
                for (int p = 0; p < PL; ++p) {
                    typedef __fp16 fp16x4 __attribute__((__vector_size__(8)));
                    typedef __attribute__((address_space(3))) fp16x4 lds_f16x4;
                    const char *at = X + (jb * 32 + 8 * quarter + (r16 >> 2)) * S + at_plane<PL>(b * 16, p) * 2 + (r16 & 3) * 8;
                    const auto lo = __builtin_amdgcn_ds_read_tr16_b64_v4f16((lds_f16x4 *)at);
                    const auto hi = __builtin_amdgcn_ds_read_tr16_b64_v4f16((lds_f16x4 *)(at + 4 * S));
                    f[p] = __builtin_shufflevector(__builtin_bit_cast(f16x4, lo), __builtin_bit_cast(f16x4, hi), 0, 1, 2, 3, 4, 5, 6, 7);
                }
            };
            rows_of(bi, f.a);
#pragma unroll
            for (int q = 0; q < Q; ++q) rows_of(bj + q, f.b[q]);
        };
        clear();
        Rows f0, f1;                               // one being multiplied, one on its way
        columns(0, f0);
        for (int jb = 0; jb < blocks; jb += 2) {
            if (jb + 1 < blocks) columns(jb + 1, f1);
#pragma unroll
            for (int q = 0; q < Q; ++q) acc[q] = mfma16(f0.a, f0.b[q], acc[q]);
            if (jb + 1 == blocks) break;
            if (jb + 2 < blocks) columns(jb + 2, f0);
#pragma unroll
            for (int q = 0; q < Q; ++q) acc[q] = mfma16(f1.a, f1.b[q], acc[q]);
        }
    }
    // G = acc, then P = b G + c G G, both to LDS (barriers between and after)
    __device__ __forceinline__ void polynomial()
    {
        const int bi = wave / (W / 4), bj = wave % (W / 4) * Q, r16 = lane & 15, quarter = lane >> 4, i = bi * 16 + 4 * quarter;
#pragma unroll
        for (int q = 0; q < Q; ++q) {
            const int j = (bj + q) * 16 + r16;
            f32x4 v = acc[q] * kDown;
#pragma unroll
            for (int k = 0; k < 4; ++k)
                if (i + k == j) {
                    gd[j] = v[k] * kDown;
                    v[k] = 0.f;
                }
            put4(G + j * S, i, v);
        }
        __syncthreads();
        clear();
#pragma unroll
        for (int jb = 0; jb < 2; ++jb) {
            auto rows_of = [&](int b, f16x8 (&f)[PL]) __attribute__((always_inline)) {
#pragma unroll
                for (int p = 0; p < PL; ++p) f[p] = *reinterpret_cast<const f16x8 *>(G + (b * 16 + r16) * S + jb * 64 * PL + p * 64 + quarter * 16);
            };
            Rows f;
            rows_of(bi, f.a);
#pragma unroll
            for (int q = 0; q < Q; ++q) rows_of(bj + q, f.b[q]);
#pragma unroll
            for (int q = 0; q < Q; ++q) acc[q] = mfma16(f.a, f.b[q], acc[q]);
        }
        const f32x4 di = *reinterpret_cast<const f32x4 *>(gd + i);
#pragma unroll
        for (int q = 0; q < Q; ++q) {
            const int j = (bj + q) * 16 + r16;
            const float dj = gd[j];
            const f32x4 e = get4(G + j * S, i);
            f32x4 v;
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                v[k] = __builtin_fmaf(kC, acc[q][k] * kDown, __builtin_fmaf(kC, di[k] + dj, kB) * e[k]);
                if (i + k == j) {
                    pd[j] = __builtin_fmaf(kC, __builtin_fmaf(dj, dj, acc[q][k] * (kDown * kDown)), kB * dj);
                    v[k] = 0.f;
                }
            }
            put4(P + j * S, i, v);
        }
        __syncthreads();
    }
    // X <- a X + P X
    __device__ __forceinline__ void apply()
    {
#pragma unroll
        for (int c = 0; c < CB; ++c) {
            const int jb = wave + W * c;
            if (jb >= blocks) continue;
#pragma unroll
            for (int r = 0; r < 2; ++r) {
                f32x16 sum = {};
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    const int at = (k >> 1) * 64 * PL + (k & 1) * 32 + half * 16;
                    f16x8 fb[PL], fa[PL];
#pragma unroll
                    for (int p = 0; p < PL; ++p) {
                        fb[p] = *reinterpret_cast<const f16x8 *>(X + (jb * 32 + col) * S + at + p * 64);
                        fa[p] = *reinterpret_cast<const f16x8 *>(P + (r * 32 + col) * S + at + p * 64);
                    }
                    if constexpr (PL == 2) {
                        sum = __builtin_amdgcn_mfma_f32_32x32x16_f16(fa[1], fb[0], sum, 0, 0, 0);
                        sum = __builtin_amdgcn_mfma_f32_32x32x16_f16(fa[0], fb[1], sum, 0, 0, 0);
                    }
                    sum = __builtin_amdgcn_mfma_f32_32x32x16_f16(fa[0], fb[0], sum, 0, 0, 0);
                }
#pragma unroll
                for (int q = 0; q < 4; ++q) {
                    const f32x4 pdv = *reinterpret_cast<const f32x4 *>(pd + r * 32 + 8 * q + 4 * half);
#pragma unroll
                    for (int v = 0; v < 4; ++v) x[c][r][4 * q + v] = __builtin_fmaf(kA + pdv[v], x[c][r][4 * q + v], sum[4 * q + v] * (kDown * kDown));
                }
            }
        }
    }
    __device__ __forceinline__ void scale(double by)
    {
#pragma unroll
        for (int c = 0; c < CB; ++c)
#pragma unroll
            for (int r = 0; r < 2; ++r)
#pragma unroll
                for (int v = 0; v < 16; ++v) {
                    x[c][r][v] = (float)(x[c][r][v] * by);
                }
    }
    __device__ __forceinline__ void write(const Target &out, size_t base)
    {
        float *theta = out.theta + base;
        T *y = static_cast<T *>(out.out) + base;
#pragma unroll
        for (int c = 0; c < CB; ++c)
#pragma unroll
            for (int r = 0; r < 2; ++r) {
                bool there[16];
                unsigned at[16];
#pragma unroll
                for (int v = 0; v < 16; ++v) at[v] = place(c, r, v, there[v]);
                if (out.theta) {
                    float t[16];
#pragma unroll
                    for (int v = 0; v < 16; ++v) t[v] = element(theta, at[v]);
#pragma unroll
                    for (int v = 0; v < 16; ++v)
                        if (there[v]) element(theta, at[v]) = __builtin_fmaf(-out.rate, x[c][r][v], out.keep * t[v]);
                } else
#pragma unroll
                    for (int v = 0; v < 16; ++v)
                        if (there[v]) Elem<T>::store(&element(y, at[v]), x[c][r][v]);
            }
    }
};

// All columns in one workgroup: everything of a matrix in one launch, and nothing but its input and output passes memory.  Three
// barriers a step, which with the chains of LDS reads and products between them are all of its time (two planes, fp32: 64 x 27: 20 us; 64 x 448:
// 46 us; 64 matrices of 64 x 27 at once: 21 us).  Sixteen waves, one plane: 4 % faster for 64 x 512, 8 % slower for 64 x 256, and registers
// for one block a wave only.
template <typename T, int PL, int CB>
__global__ __launch_bounds__(512) void muon_small_kernel(Source src, Target out, int rows, int cols, int steps)
{
    extern __shared__ __align__(16) char lds[];
    FewRows<T, PL, CB> w(lds, rows, cols, 0, CB * 8);
    const size_t base = (size_t)blockIdx.x * rows * cols;
    const T *in = static_cast<const T *>(src.x) + base;
    float *momentum = src.momentum + base;
    double sum = 0;
#pragma unroll
    for (int c = 0; c < CB; ++c)
#pragma unroll
        for (int r = 0; r < 2; ++r) {
            bool there[16];
            unsigned at[16];
#pragma unroll
            for (int v = 0; v < 16; ++v) {
                at[v] = w.place(c, r, v, there[v]);
                w.x[c][r][v] = Elem<T>::load(&w.element(in, at[v]));
            }
            if (src.momentum) {
                float mom[16];
#pragma unroll
                for (int v = 0; v < 16; ++v) mom[v] = w.element(momentum, at[v]);
#pragma unroll
                for (int v = 0; v < 16; ++v) {
                    mom[v] = __builtin_fmaf(src.mu, mom[v], w.x[c][r][v]);
                    if (there[v]) w.element(momentum, at[v]) = mom[v];
                    w.x[c][r][v] = src.nesterov ? __builtin_fmaf(src.mu, mom[v], w.x[c][r][v]) : mom[v];
                }
            }
#pragma unroll
            for (int v = 0; v < 16; ++v) {
                w.x[c][r][v] = there[v] ? w.x[c][r][v] : 0.f;
                sum = __builtin_fma((double)w.x[c][r][v], (double)w.x[c][r][v], sum);
            }
        }
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) sum += __shfl_xor(sum, o, kWave);
    if (w.lane == 0) w.red[w.wave] = sum;
    __syncthreads();
    sum = 0;
#pragma unroll
    for (int k = 0; k < 8; ++k) sum += w.red[k];
    w.scale(scale_of(sum));
    w.forget_places();
    for (int step = 0; step < steps; ++step) {
        w.put_x();                                 // (a wave's own columns, which no other reads before the barrier)
        __syncthreads();
        w.gram();
        w.polynomial();
        w.apply();
    }
    w.forget_places();
    w.write(out, base);
}

// More columns: `each` blocks of 32 to a workgroup (up to 8 CB), and a launch a step.  Every workgroup adds up all workgroups' shares
// of G itself, in order, and forms P; what it writes for the next launch is its columns of X, as its registers hold them, and its share of their G.
// Bound by six launches of some 8 us each until the columns are many (two planes, fp32: 64 x 768: 51 us; 2 x 28 x 7933: 93 us; 64 x 25088:
// 120 us; with an update's step 148 us, 178 us by tiles of products).  step 0: X_0 from the input; step `steps`: the output.
template <typename T, int PL, int CB>
__global__ __launch_bounds__(512) void muon_wide_kernel(Source src, Target out, int rows, int cols, int each, int step, int steps, const double *part,
                                                        int parts, float *x32, const f32x4 *shares, f32x4 *share)
{
    extern __shared__ __align__(16) char lds[];
    const int wgs = gridDim.x, b = blockIdx.y;
    FewRows<T, PL, CB> w(lds, rows, cols, blockIdx.x * each, each);
    const size_t base = (size_t)b * rows * cols;
    float *mine = x32 + ((size_t)b * wgs + blockIdx.x) * (CB * 8 * 2048) + w.wave * 2048 + w.lane;   // [c][wave][r][v][lane]
    const size_t at = ((size_t)b * wgs * 8 + w.wave) * 128 + w.lane;                                 // [workgroup][wave][q][lane]
    if (step == 0) {
#pragma unroll
        for (int c = 0; c < CB; ++c)
#pragma unroll
            for (int r = 0; r < 2; ++r)
#pragma unroll
                for (int v = 0; v < 16; ++v) {
                    bool there;
                    const size_t k = base + w.place(c, r, v, there);
                    const float u = source_at<T>(src, k);
                    w.x[c][r][v] = there ? u : 0.f;
                }
        double norm2 = 0;
        for (int k = threadIdx.x; k < parts; k += 512) norm2 += part[b * kParts + k];
#pragma unroll
        for (int o = 32; o > 0; o >>= 1) norm2 += __shfl_xor(norm2, o, kWave);
        if (w.lane == 0) w.red[w.wave] = norm2;
        __syncthreads();
        norm2 = 0;
#pragma unroll
        for (int k = 0; k < 8; ++k) norm2 += w.red[k];
        w.scale(scale_of(norm2));
    } else {
#pragma unroll
        for (int c = 0; c < CB; ++c)
#pragma unroll
            for (int r = 0; r < 2; ++r)
#pragma unroll
                for (int v = 0; v < 16; ++v) w.x[c][r][v] = mine[c * (8 * 2048) + (r * 16 + v) * 64];
        w.put_x();
        w.clear();
        constexpr int U = 8;                       // shares on their way
        for (int g = 0; g < wgs; g += U) {
            f32x4 u[U][2];
#pragma unroll
            for (int k = 0; k < U; ++k)
#pragma unroll
                for (int q = 0; q < 2; ++q) u[k][q] = g + k < wgs ? shares[at + (size_t)(g + k) * 1024 + q * 64] : f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int k = 0; k < U; ++k)
#pragma unroll
                for (int q = 0; q < 2; ++q) w.acc[q] += u[k][q];
        }
        w.polynomial();
        w.apply();
    }
    if (step == steps) {
        w.write(out, base);
        return;
    }
    w.put_x();
#pragma unroll
    for (int c = 0; c < CB; ++c)
#pragma unroll
        for (int r = 0; r < 2; ++r)
#pragma unroll
            for (int v = 0; v < 16; ++v) mine[c * (8 * 2048) + (r * 16 + v) * 64] = w.x[c][r][v];
    __syncthreads();
    w.gram();
#pragma unroll
    for (int q = 0; q < 2; ++q) share[at + (size_t)blockIdx.x * 1024 + q * 64] = w.acc[q];
}

struct Wide : FewPlan { int parts; size_t part, x32, share, total; };
Wide wide_plan(int planes, int batch, int rows, int cols)
{
    Wide w = {few_plan(planes, rows, cols)};
    w.parts = norm_parts((size_t)rows * cols, kNormLot<float>);
    w.part = round_up((size_t)batch * kParts * 8, 256);
    w.x32 = round_up((size_t)batch * w.wgs * w.cb * 8 * 2048 * 4, 256);
    w.share = round_up((size_t)batch * w.wgs * 16384, 256);
    w.total = w.part + w.x32 + 2 * w.share;
    return w;
}

// How many ranges a contraction of `all` stages is cut into for `tiles` workgroups each: rounds of the chip's 256 compute units
// times what one takes, in cycles (a stage at the matrix unit's rate, some thousand to begin and end), and the sums' way through
// memory.
int split_count(int planes, int tile, long tiles, int all)
{
    const double stage = (tile == 256 ? 4 : 1) * (planes == 2 ? 768.0 : 512.0) * 1.3;
    int best = 1;
    double least = 0;
    for (int s = 1; s <= 64 && s <= all; ++s) {
        const double t = (double)((tiles * s + 255) / 256) * ((all + s - 1) / s * stage + 4000) + (double)tiles * s * tile * tile * 8 / 1600 + s * 150;
        if (s == 1 || t < least) { least = t; best = s; }
    }
    return best;
}

Layout layout_of(int planes, int batch, int rows, int cols, char *ws, size_t &total)
{
    Layout L;
    L.rows = rows; L.cols = cols; L.tall = rows > cols; L.batch = batch;
    L.m = L.tall ? cols : rows; L.n = L.tall ? rows : cols;
    L.tile = muon_tile(batch, L.m, L.n);
    L.mp = round_to(L.m, L.tile); L.np = round_to(L.n, L.tile);
    const int mt = L.mp / L.tile;
    const long tiles = (long)batch * (mt * (mt + 1) / 2);
    L.splits[kGram] = split_count(planes, L.tile, tiles, L.np * planes / 64);
    L.splits[kPoly] = split_count(planes, L.tile, tiles, L.mp * planes / 64);
    L.parts = norm_parts((size_t)rows * cols, kNormLot<float>);
    size_t off = 0;
    auto take = [&](size_t bytes) { char *p = ws + off; off += round_up(bytes, 256); return p; };
    const size_t mn = (size_t)batch * L.mp * L.np, mm = (size_t)batch * L.mp * L.mp;
    L.part = reinterpret_cast<double *>(take((size_t)batch * kParts * 8));
    L.x32 = reinterpret_cast<float *>(take(mn * 4));
    for (int k = 0; k < 2; ++k) L.x[k] = reinterpret_cast<half_t *>(take(mn * 2 * planes));
    L.g = reinterpret_cast<half_t *>(take(mm * 2 * planes));
    L.p = reinterpret_cast<half_t *>(take(mm * 2 * planes));
    L.gd = reinterpret_cast<float *>(take((size_t)batch * L.mp * 4));
    L.pd = reinterpret_cast<float *>(take((size_t)batch * L.mp * 4));
    const int most = L.splits[kGram] > L.splits[kPoly] ? L.splits[kGram] : L.splits[kPoly];
    L.sums = reinterpret_cast<float *>(take((size_t)tiles * most * L.tile * L.tile * 4));
    total = off;
    return L;
}

template <typename T, int PL, int MODE, int TILE>
int product(const Layout &L, int from, const Target &out, hipStream_t s)
{
    auto kern = muon_product_kernel<T, PL, MODE, TILE>;
    if (!raise_lds_limit(reinterpret_cast<const void *>(kern))) return VGG_ERR_LAUNCH;
    const int mt = L.mp / TILE, nt = L.np / TILE;
    if constexpr (MODE == kApply || MODE == kLast) {
        hipLaunchKernelGGL(kern, dim3(mt * nt, L.batch), dim3(512), 131072, s, L, from, out);
    } else {
        const int tiles = mt * (mt + 1) / 2;
        hipLaunchKernelGGL(kern, dim3(tiles * L.splits[MODE], L.batch), dim3(512), 131072, s, L, from, out);
        hipLaunchKernelGGL((muon_symmetric_kernel<PL, MODE, TILE>), dim3(tiles * (TILE / 32) * (TILE / 32), L.batch), dim3(256), 0, s, L);
    }
    return VGG_OK;
}

template <typename T, int PL, int TILE>
int steps_of(const Layout &L, int steps, const Target &out, hipStream_t s)
{
    for (int k = 0; k < steps; ++k) {
        if (const int rc = product<float, PL, kGram, TILE>(L, k & 1, out, s)) return rc;
        if (const int rc = product<float, PL, kPoly, TILE>(L, k & 1, out, s)) return rc;
        if (const int rc = k + 1 < steps ? product<float, PL, kApply, TILE>(L, k & 1, out, s) : product<T, PL, kLast, TILE>(L, k & 1, out, s)) return rc;
    }
    return VGG_OK;
}

template <typename T, int PL>
int run(int batch, int rows, int cols, int steps, const Source &src, const Target &out, void *ws, hipStream_t s)
{
    if (const int cb = small_blocks(PL, rows, cols)) {
        auto kern = cb == 1 ? muon_small_kernel<T, PL, 1> : muon_small_kernel<T, PL, 2>;
        if constexpr (PL == 1)                         // (two planes of so many columns have no room)
            if (cb == 3) kern = muon_small_kernel<T, PL, 3>;
        if (!raise_lds_limit(reinterpret_cast<const void *>(kern))) return VGG_ERR_LAUNCH;
        hipLaunchKernelGGL(kern, dim3(batch), dim3(512), few_lds(PL, ((rows < cols ? cols : rows) + 31) / 32), s, src, out, rows, cols, steps);
        return launch_status();
    }
    if (is_wide(PL, rows, cols)) {
        const Wide p = wide_plan(PL, batch, rows, cols);
        auto kern = p.cb == 1 ? muon_wide_kernel<T, PL, 1> : muon_wide_kernel<T, PL, 2>;
        if (!raise_lds_limit(reinterpret_cast<const void *>(kern))) return VGG_ERR_LAUNCH;
        double *part = static_cast<double *>(ws);
        float *x32 = reinterpret_cast<float *>(static_cast<char *>(ws) + p.part);
        f32x4 *share[2];
        for (int k = 0; k < 2; ++k) share[k] = reinterpret_cast<f32x4 *>(static_cast<char *>(ws) + p.part + p.x32 + k * p.share);
        hipLaunchKernelGGL((muon_norm_kernel<T>), dim3(p.parts, batch), dim3(256), 0, s, src, part, (size_t)rows * cols);
        for (int k = 0; k <= steps; ++k)
            hipLaunchKernelGGL(kern, dim3(p.wgs, batch), dim3(512), few_lds(PL, p.each), s, src, out, rows, cols, p.each, k, steps, part, p.parts, x32, share[1 - (k & 1)], share[k & 1]);
        return launch_status();
    }
    size_t total;
    const Layout L = layout_of(PL, batch, rows, cols, static_cast<char *>(ws), total);
    hipLaunchKernelGGL((muon_norm_kernel<T>), dim3(L.parts, batch), dim3(256), 0, s, src, L.part, (size_t)rows * cols);
    hipLaunchKernelGGL((muon_start_kernel<T, PL>), dim3(L.np / 64, L.mp / 64, batch), dim3(256), 0, s, src, L);
    if (const int rc = L.tile == 256 ? steps_of<T, PL, 256>(L, steps, out, s) : steps_of<T, PL, 128>(L, steps, out, s)) return rc;
    return launch_status();
}

}  // namespace

// What either number of planes takes: both of a type's calls ask for the same.
size_t muon_workspace(int batch, int rows, int cols)
{
    size_t most = 0;
    for (int planes = 1; planes <= 2; ++planes) {
        size_t total;
        if (is_wide(planes, rows, cols)) total = wide_plan(planes, batch, rows, cols).total;   // (one workgroup alone needs none)
        else layout_of(planes, batch, rows, cols, nullptr, total);
        if (total > most) most = total;
    }
    return most;
}

int orthogonalize(int dtype, int batch, int rows, int cols, int steps, const void *x, void *y, void *ws, hipStream_t s)
{
    const Source src = {x, nullptr, 0.f, 0};
    const Target out = {y, nullptr, 0.f, 0.f};
    return dtype == VGG_BF16 ? run<bf16_t, 2>(batch, rows, cols, steps, src, out, ws, s) : run<float, 2>(batch, rows, cols, steps, src, out, ws, s);
}

int muon_update(int dtype, int batch, int rows, int cols, int steps, float *theta, const float *grad, float *momentum, float lr, float mu,
                int nesterov, float weight_decay, void *ws, hipStream_t s)
{
    const float wide = rows > cols ? (float)sqrt((double)rows / cols) : 1.f;
    const Source src = {grad, momentum, mu, nesterov};
    const Target out = {nullptr, theta, 1.f - lr * weight_decay, lr * wide};
    return dtype == VGG_BF16 ? run<float, 1>(batch, rows, cols, steps, src, out, ws, s) : run<float, 2>(batch, rows, cols, steps, src, out, ws, s);
}

}  // namespace vgg
