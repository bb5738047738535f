// Orthogonalised updates: Newton-Schulz products, and the optimiser step around them.
//
// X_0 = U / (|U| + eps), |U| the Frobenius norm; then, X of m x n with m <= n (a tall U is taken transposed),
//     G = X X^T,   X <- a X + (b G + c G G) X.
// The polynomial a s + b s^3 + c s^5 takes the singular values, all in [0, 1], towards 1, within [0, 1.21] throughout.
//
// Products are on the f16 matrix unit with fp32 sums.  X, G and P = b G + c G G are bounded (|X|, |G|, |P| <= 1.21, 1.47, 2.9), so
// that they are held times 2^14, below f16's largest, and need no other scale; f16 then keeps 11 bits of everything down to
// 2^-28.  PLANES = 2 (VGG_F32): a value is two f16 numbers, the nearest and what that leaves, 22 bits; hi hi + hi lo + lo hi
// leaves out 2^-22 of a product at most.  PLANES = 1 (VGG_BF16): operands are rounded to 11 bits.  In both the term a X adds an
// fp32 copy of X, since a rounding of X there would grow 3.4-fold in every later step where X has no (or small) singular values;
// and the diagonals of G and P, which hold most of them, are kept apart in fp32 (zeros in the planes): with G = D + E,
//     (G G)_ij = (E E)_ij + (d_i + d_j) e_ij,   (G G)_ii = (E E)_ii + d_i^2,   (P X)_i = p_i X_i + (the rest of P) X.
// One plane is then 3e-4 to 1e-3 off in all, against 1.3e-3 to 2.4e-3 with the diagonals rounded (bf16's own rounding: 1.7e-3).
//
// All products are "row times row": C[i][j] = sum_k A[i][k] B[j][k].  G: rows of X; G G: rows of the symmetric G; P X: rows of P
// and of X^T, for which X is also kept transposed.  An operand's row holds, for every 32 contraction indices, 64 bytes of the
// first plane and then of the second.
#include "common.h"

namespace vgg {

namespace {

typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 half_t;

constexpr float kA = 3.4445f, kB = -4.7750f, kC = 2.0315f, kEps = 1e-7f;
constexpr float kUp = 16384.f, kDown = 1.f / 16384.f;   // 2^14
constexpr int kTile = 128;                              // every padded size is a multiple of it
constexpr int kParts = 256;                             // partial sums of squares of a matrix

__host__ __device__ inline int padded(int v) { return (v + kTile - 1) / kTile * kTile; }

// Element k of a row of K-blocks of 32 with PL planes.
template <int PL> __device__ __forceinline__ size_t at_plane(int k, int plane) { return (size_t)(k >> 5) * (32 * PL) + plane * 32 + (k & 31); }
template <int PL> __device__ __forceinline__ void put(half_t *row, int k, float scaled)
{
    const half_t hi = (half_t)scaled;
    row[at_plane<PL>(k, 0)] = hi;
    if constexpr (PL == 2) row[at_plane<PL>(k, 1)] = (half_t)(scaled - (float)hi);
}
template <int PL> __device__ __forceinline__ float get(const half_t *row, int k)
{
    float v = (float)row[at_plane<PL>(k, 0)];
    if constexpr (PL == 2) v += (float)row[at_plane<PL>(k, 1)];
    return v;
}

// ----------------------------------------------------------------------------------- momentum and the norm
// Squares are summed in 64 bits: they neither overflow nor vanish.
__device__ __forceinline__ double block_sum(double v)
{
    __shared__ double red[4];
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) v += __shfl_xor(v, o, kWave);
    if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = v;
    __syncthreads();
    return red[0] + red[1] + red[2] + red[3];
}

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

template <typename T>
__global__ __launch_bounds__(256) void muon_norm_kernel(Source s, double *__restrict__ part, size_t count)
{
    const size_t base = (size_t)blockIdx.y * count;
    double sum = 0;
    for (size_t i = (size_t)blockIdx.x * 256 + threadIdx.x; i < count; i += (size_t)kParts * 256) {
        if (s.momentum) s.momentum[base + i] = __builtin_fmaf(s.mu, s.momentum[base + i], Elem<T>::load(static_cast<const T *>(s.x) + base + i));
        const float u = source_at<T>(s, base + i);
        sum += (double)u * u;
    }
    sum = block_sum(sum);
    if (threadIdx.x == 0) part[blockIdx.y * kParts + blockIdx.x] = sum;
}

// X_0 in all its layouts, zeros where they are padded.  A workgroup: 64 x 64 of the padded X.
struct Layout {
    int rows, cols, m, n, mp, np, tall;
    float *x32;            // [batch][mp][np]
    half_t *x, *xt[2];     // [batch][mp][np], [batch][np][mp], PLANES each
    half_t *g, *p;         // [batch][mp][mp], PLANES each, zero diagonals
    float *gd, *pd;        // [batch][mp], the diagonals
    double *part;          // [batch][kParts]
};
template <typename T, int PL>
__global__ __launch_bounds__(256) void muon_start_kernel(Source s, Layout L)
{
    __shared__ float tile[64][65];
    const int b = blockIdx.z, i0 = blockIdx.y * 64, j0 = blockIdx.x * 64, tx = threadIdx.x & 63, ty = threadIdx.x >> 6;
    const double norm2 = block_sum(L.part[b * kParts + threadIdx.x]);
    const float by = norm2 < (double)INFINITY ? 1.f / ((float)sqrt(norm2) + kEps) : NAN;
    const size_t base = (size_t)b * L.rows * L.cols;
    // the source is read along its own rows
    for (int y = ty; y < 64; y += 4) {
        const int i = L.tall ? i0 + tx : i0 + y, j = L.tall ? j0 + y : j0 + tx;      // of X
        const float v = i < L.m && j < L.n ? source_at<T>(s, base + (L.tall ? (size_t)j * L.cols + i : (size_t)i * L.cols + j)) * by : 0.f;
        if (L.tall) tile[tx][y] = v;
        else tile[y][tx] = v;
    }
    __syncthreads();
    float *x32 = L.x32 + (size_t)b * L.mp * L.np;
    half_t *x = L.x + (size_t)b * L.mp * L.np * PL, *xt = L.xt[0] + (size_t)b * L.mp * L.np * PL;
    for (int y = ty; y < 64; y += 4) {
        x32[(size_t)(i0 + y) * L.np + j0 + tx] = tile[y][tx];
        put<PL>(x + (size_t)(i0 + y) * L.np * PL, j0 + tx, tile[y][tx] * kUp);
        put<PL>(xt + (size_t)(j0 + y) * L.mp * PL, i0 + tx, tile[tx][y] * kUp);
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

__device__ __forceinline__ void copy16(unsigned lds, const void *src)   // 16 bytes a lane to lds + 16 lane
{
    const unsigned at = __builtin_amdgcn_readfirstlane(lds);
    asm volatile("s_mov_b32 m0, %0\n\tglobal_load_lds_dwordx4 %1, off" : : "s"(at), "v"(src) : "m0", "memory");
}

// A workgroup of four waves: 128 x 128 of C, 64 x 64 to a wave.  128 bytes of each operand row a stage (64 contraction indices,
// or 32 in two planes), two stages in LDS; 16-byte segment s of row r lies at s ^ (r & 7), so that eight rows of one segment are
// in different banks.
template <typename T, int PL, int MODE>
__global__ __launch_bounds__(256, 2) void muon_product_kernel(Layout L, int from, Target out)
{
    extern __shared__ __align__(16) char lds[];   // [2][A 16 KB, B 16 KB]
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, b = blockIdx.z;
    int ti = blockIdx.y, tj = blockIdx.x;
    if constexpr (MODE == kGram || MODE == kPoly) {   // tiles on and below the diagonal, counted row by row
        const int t = blockIdx.x;
        ti = (int)((sqrtf(8.f * t + 1.f) - 1.f) * 0.5f);
        while ((ti + 1) * (ti + 2) / 2 <= t) ++ti;
        while (ti * (ti + 1) / 2 > t) --ti;
        tj = t - ti * (ti + 1) / 2;
    }
    const size_t mm = (size_t)L.mp * L.mp, mn = (size_t)L.mp * L.np;
    const int K = MODE == kGram ? L.np : L.mp;
    const size_t row_bytes = (size_t)K * PL * 2;
    const half_t *pa = MODE == kGram ? L.x + b * mn * PL : MODE == kPoly ? L.g + b * mm * PL : L.p + b * mm * PL;
    const half_t *pb = MODE == kGram ? pa : MODE == kPoly ? pa : L.xt[from] + b * mn * PL;
    const char *ga = reinterpret_cast<const char *>(pa) + (size_t)ti * 128 * row_bytes;
    const char *gb = reinterpret_cast<const char *>(pb) + (size_t)tj * 128 * row_bytes;
    const unsigned lds0 = (unsigned)(uintptr_t)(__attribute__((address_space(3))) char *)lds;
    const int stages = (int)(row_bytes / 128);

    auto stage_copy = [&](int st) __attribute__((always_inline)) {
        const unsigned dst = lds0 + (st & 1) * 32768;
#pragma unroll
        for (int q = 0; q < 8; ++q) {            // 8 rows of one operand each: waves 0, 1 copy A, waves 2, 3 B
            const int r = (wave & 1) * 64 + q * 8 + (lane >> 3), seg = (lane & 7) ^ (r & 7);
            copy16(dst + (wave >> 1) * 16384 + ((wave & 1) * 64 + q * 8) * 128, (wave >> 1 ? gb : ga) + r * row_bytes + (size_t)st * 128 + seg * 16);
        }
    };

    f32x16 acc[2][2] = {};
    const int wi = (wave >> 1) * 64, wj = (wave & 1) * 64;
    stage_copy(0);
    for (int st = 0; st < stages; ++st) {
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
        __syncthreads();
        if (st + 1 < stages) stage_copy(st + 1);
        const char *A = lds + (st & 1) * 32768, *B = A + 16384;
        auto frag = [&](const char *p, int row, int seg) __attribute__((always_inline)) {
            return *reinterpret_cast<const f16x8 *>(p + row * 128 + ((seg ^ (row & 7)) << 4));
        };
#pragma unroll
        for (int k = 0; k < 4 / PL; ++k) {
            f16x8 fa[PL][2], fb[PL][2];
#pragma unroll
            for (int p = 0; p < PL; ++p)
#pragma unroll
                for (int q = 0; q < 2; ++q) {
                    const int seg = p * 4 + k * 2 + (lane >> 5);
                    fa[p][q] = frag(A, wi + q * 32 + (lane & 31), seg);
                    fb[p][q] = frag(B, wj + q * 32 + (lane & 31), seg);
                }
#pragma unroll
            for (int x = 0; x < 2; ++x)
#pragma unroll
                for (int y = 0; y < 2; ++y) {
                    if constexpr (PL == 2) {
                        acc[x][y] = __builtin_amdgcn_mfma_f32_32x32x16_f16(fa[1][x], fb[0][y], acc[x][y], 0, 0, 0);
                        acc[x][y] = __builtin_amdgcn_mfma_f32_32x32x16_f16(fa[0][x], fb[1][y], acc[x][y], 0, 0, 0);
                    }
                    acc[x][y] = __builtin_amdgcn_mfma_f32_32x32x16_f16(fa[0][x], fb[0][y], acc[x][y], 0, 0, 0);
                }
        }
    }

    // Value v of a block: row 8 (v / 4) + 4 (lane / 32) + v % 4, column lane % 32.
#pragma unroll
    for (int x = 0; x < 2; ++x)
#pragma unroll
        for (int y = 0; y < 2; ++y)
#pragma unroll
            for (int v = 0; v < 16; ++v) {
                const int i = ti * 128 + wi + x * 32 + 8 * (v >> 2) + 4 * (lane >> 5) + (v & 3), j = tj * 128 + wj + y * 32 + (lane & 31);
                const float c = acc[x][y][v];
                if constexpr (MODE == kGram) {
                    half_t *gm = L.g + b * mm * PL;
                    if (i == j) L.gd[(size_t)b * L.mp + i] = c * (kDown * kDown);
                    put<PL>(gm + (size_t)i * L.mp * PL, j, i == j ? 0.f : c * kDown);
                    if (ti != tj) put<PL>(gm + (size_t)j * L.mp * PL, i, c * kDown);
                } else if constexpr (MODE == kPoly) {
                    const float *gd = L.gd + (size_t)b * L.mp;
                    const float di = gd[i], dj = gd[j];
                    const float w = __builtin_fmaf(kC, c * kDown, __builtin_fmaf(kC, di + dj, kB) * get<PL>(L.g + b * mm * PL + (size_t)i * L.mp * PL, j));
                    half_t *pm = L.p + b * mm * PL;
                    if (i == j) L.pd[(size_t)b * L.mp + i] = __builtin_fmaf(kC, __builtin_fmaf(di, di, c * (kDown * kDown)), kB * di);
                    put<PL>(pm + (size_t)i * L.mp * PL, j, i == j ? 0.f : w);
                    if (ti != tj) put<PL>(pm + (size_t)j * L.mp * PL, i, w);
                } else {
                    float *x32 = L.x32 + b * mn + (size_t)i * L.np + j;
                    const float w = __builtin_fmaf(kA + L.pd[(size_t)b * L.mp + i], *x32, c * (kDown * kDown));
                    if constexpr (MODE == kApply) {
                        *x32 = w;
                        put<PL>(L.x + b * mn * PL + (size_t)i * L.np * PL, j, w * kUp);
                        put<PL>(L.xt[1 - from] + b * mn * PL + (size_t)j * L.mp * PL, i, w * kUp);
                    } else if (i < L.m && j < L.n) {
                        const size_t o = (size_t)b * L.rows * L.cols + (L.tall ? (size_t)j * L.cols + i : (size_t)i * L.cols + j);
                        if (out.theta) out.theta[o] = __builtin_fmaf(-out.rate, w, out.keep * out.theta[o]);
                        else Elem<T>::store(static_cast<T *>(out.out) + o, w);
                    }
                }
            }
}

Layout layout_of(int planes, int batch, int rows, int cols, char *ws, size_t &total)
{
    Layout L;
    L.rows = rows; L.cols = cols; L.tall = rows > cols;
    L.m = L.tall ? cols : rows; L.n = L.tall ? rows : cols;
    L.mp = padded(L.m); L.np = padded(L.n);
    size_t off = 0;
    auto take = [&](size_t bytes) { char *p = ws + off; off += round_up(bytes, 256); return p; };
    const size_t mn = (size_t)batch * L.mp * L.np, mm = (size_t)batch * L.mp * L.mp;
    L.part = reinterpret_cast<double *>(take((size_t)batch * kParts * 8));
    L.x32 = reinterpret_cast<float *>(take(mn * 4));
    L.x = reinterpret_cast<half_t *>(take(mn * 2 * planes));
    for (int k = 0; k < 2; ++k) L.xt[k] = reinterpret_cast<half_t *>(take(mn * 2 * planes));
    L.g = reinterpret_cast<half_t *>(take(mm * 2 * planes));
    L.p = reinterpret_cast<half_t *>(take(mm * 2 * planes));
    L.gd = reinterpret_cast<float *>(take((size_t)batch * L.mp * 4));
    L.pd = reinterpret_cast<float *>(take((size_t)batch * L.mp * 4));
    total = off;
    return L;
}

template <typename T, int PL>
int run(int batch, int rows, int cols, int steps, const Source &src, const Target &out, void *ws, hipStream_t s)
{
    size_t total;
    const Layout L = layout_of(PL, batch, rows, cols, static_cast<char *>(ws), total);
    const unsigned mt = L.mp / kTile, nt = L.np / kTile, b = batch;
    hipLaunchKernelGGL((muon_norm_kernel<T>), dim3(kParts, b), dim3(256), 0, s, src, L.part, (size_t)rows * cols);
    hipLaunchKernelGGL((muon_start_kernel<T, PL>), dim3(L.np / 64, L.mp / 64, b), dim3(256), 0, s, src, L);
    for (int k = 0; k < steps; ++k) {
        hipLaunchKernelGGL((muon_product_kernel<T, PL, kGram>), dim3(mt * (mt + 1) / 2, 1, b), dim3(256), 65536, s, L, 0, out);
        hipLaunchKernelGGL((muon_product_kernel<T, PL, kPoly>), dim3(mt * (mt + 1) / 2, 1, b), dim3(256), 65536, s, L, 0, out);
        if (k + 1 < steps) hipLaunchKernelGGL((muon_product_kernel<T, PL, kApply>), dim3(nt, mt, b), dim3(256), 65536, s, L, k & 1, out);
        else hipLaunchKernelGGL((muon_product_kernel<T, PL, kLast>), dim3(nt, mt, b), dim3(256), 65536, s, L, k & 1, out);
    }
    return launch_status();
}

}  // namespace

size_t muon_workspace(int dtype, int batch, int rows, int cols)
{
    size_t total;
    layout_of(dtype == VGG_BF16 ? 1 : 2, batch, rows, cols, nullptr, total);
    return total;
}

int orthogonalize(int dtype, int batch, int rows, int cols, int steps, const void *x, void *y, void *ws, hipStream_t s)
{
    const Source src = {x, nullptr, 0.f, 0};
    const Target out = {y, nullptr, 0.f, 0.f};
    return dtype == VGG_BF16 ? run<bf16_t, 1>(batch, rows, cols, steps, src, out, ws, s) : run<float, 2>(batch, rows, cols, steps, src, out, ws, s);
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
