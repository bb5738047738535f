// Dense layers from 4-bit weights with group scales.
//
// A code is a sign and one of 0, 0.5, 1, 1.5, 2, 3, 4, 6 (E2M1); a weight is its value times the bf16 scale of its group of
// consecutive inputs.  Codes lie two to a byte, the even input low, rows padded to 32 codes (16 bytes).
#include "common.h"
#include "plans.h"

#include <type_traits>

namespace vgg {

namespace {

typedef unsigned u32x4 __attribute__((ext_vector_type(4)));
typedef float f32x2 __attribute__((ext_vector_type(2)));

// ------------------------------------------------------------------------------------------- rounding to codes
// The bounds between codes times a bf16 scale are exact fp32 numbers, so that no division is needed and the codes are those of
// exact arithmetic: the nearest value, ties to the even code.
__device__ __forceinline__ unsigned code_of(float w, float s)
{
    const float a = __builtin_fabsf(w);
    if (!(s > 0.f)) return w < 0.f ? 8u : 0u;
    const unsigned c = (a > 0.25f * s) + (a >= 0.75f * s) + (a > 1.25f * s) + (a >= 1.75f * s) + (a > 2.5f * s) + (a >= 3.5f * s) + (a > 5.f * s);
    return c | (w < 0.f ? 8u : 0u);
}

// 16 bytes from or to an address that is a multiple of an element's size only.
struct __attribute__((packed, aligned(2))) Loose16 { unsigned v[4]; };
__device__ __forceinline__ u32x4 loose16(const void *p)
{
    const Loose16 l = *static_cast<const Loose16 *>(p);
    return u32x4{l.v[0], l.v[1], l.v[2], l.v[3]};
}

// A lane takes eight inputs: two loads of 16 bytes, one store of its eight codes.  2^shift / 8 lanes share a group, all in one wave.
// `units`: lanes of a row, whole groups.  Bound by its 411 MB of reads at 25088 x 4096: 100 us, and 95 us the way back.
__global__ __launch_bounds__(256) void w4_quantize_kernel(const float *__restrict__ w, uint8_t *__restrict__ codes, bf16_t *__restrict__ scales,
                                                          int In, int blocks, int groups, int shift, unsigned units, unsigned all)
{
    const unsigned u = blockIdx.x * 256 + threadIdx.x;
    if (u >= all) return;                              // (whole groups: no lane of one that goes on)
    const unsigned row = u / units, i0 = (u - row * units) * 8;
    const float *src = w + (size_t)row * In + i0;
    const int n = In - (int)i0;
    float v[8];
    if (n >= 8) {
        const u32x4 lo = loose16(src), hi = loose16(src + 4);
#pragma unroll
        for (int j = 0; j < 4; ++j) { const unsigned a = lo[j], b = hi[j]; v[j] = __uint_as_float(a); v[4 + j] = __uint_as_float(b); }
    } else
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] = j < n ? src[j] : 0.f;
    float most = 0.f;
    bool bad = false;
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        most = fmaxf(most, __builtin_fabsf(v[j]));
        bad = bad || !(__builtin_fabsf(v[j]) < INFINITY);
    }
    if (bad) most = INFINITY;
    most = fmaxf(most, __shfl_xor(most, 1));
    most = fmaxf(most, __shfl_xor(most, 2));
    if (shift > 5) most = fmaxf(most, __shfl_xor(most, 4));
    if (shift > 6) most = fmaxf(most, __shfl_xor(most, 8));
    const bf16_t sb = most < INFINITY ? f32_to_bf16(most * (1.f / 6.f)) : (bf16_t)0x7fc0;
    const float s = bf16_to_f32(sb);
    unsigned x = 0;
#pragma unroll
    for (int j = 0; j < 8; ++j) x |= code_of(v[j], s) << (4 * j);
    if ((int)(i0 >> 5) < blocks) reinterpret_cast<unsigned *>(codes)[(size_t)row * blocks * 4 + (i0 >> 3)] = x;
    if ((i0 & ((1u << shift) - 1)) == 0) scales[(size_t)row * groups + (i0 >> shift)] = sb;
}

// A lane: eight codes to 32 bytes of values.
__global__ __launch_bounds__(256) void w4_dequantize_kernel(const uint8_t *__restrict__ codes, const bf16_t *__restrict__ scales, float *__restrict__ w,
                                                            int In, int blocks, int groups, int shift, unsigned units, unsigned all)
{
    const unsigned u = blockIdx.x * 256 + threadIdx.x;
    if (u >= all) return;
    const unsigned row = u / units, i0 = (u - row * units) * 8;
    const int n = In - (int)i0;
    if (n <= 0) return;
    const unsigned q = reinterpret_cast<const unsigned *>(codes)[(size_t)row * blocks * 4 + (i0 >> 3)];
    const float s = bf16_to_f32(scales[(size_t)row * groups + (i0 >> shift)]);
    const f32x2 v[4] = {__builtin_amdgcn_cvt_scalef32_pk_f32_fp4(q, 1.f, 0), __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(q, 1.f, 1),
                        __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(q, 1.f, 2), __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(q, 1.f, 3)};
    float *to = w + (size_t)row * In + i0;
    if (n >= 8) {
#pragma unroll
        for (int k = 0; k < 2; ++k) {
            Loose16 o;
#pragma unroll
            for (int j = 0; j < 4; ++j) o.v[j] = __float_as_uint(s * v[2 * k + j / 2][j & 1]);
            *reinterpret_cast<Loose16 *>(to + 4 * k) = o;
        }
    } else
#pragma unroll
        for (int j = 0; j < 8; ++j)
            if (j < n) to[j] = s * v[j / 2][j & 1];
}

// ------------------------------------------------------------------------------------------------- product
// Codes stand for 2^-10 of their values in products, so that no sum of 128 of them with activations overflows where the result,
// which the scales bring down, does not.
constexpr float kSmall = 1.f / 1024.f, kLarge = 1024.f;

template <int SEL> __device__ __forceinline__ unsigned bf16_pair(unsigned codes)
{
    return __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, kSmall, SEL));
}
// The (small) values of eight codes, exactly, as bf16 (v_cvt_scalef32_pk_bf16_fp4: one instruction for two).
__device__ __forceinline__ u32x4 bf16_values(unsigned codes)
{
    return u32x4{bf16_pair<0>(codes), bf16_pair<1>(codes), bf16_pair<2>(codes), bf16_pair<3>(codes)};
}

struct W4Args {
    const uint8_t *codes;
    const bf16_t *scales;
    const float *bias;
    void *z;
    float *part;             // [splits][N][Out], or null
    int z_bf16, relu, N, In, Out, blocks, groups, shift, splits, row_tiles;
};
__device__ __forceinline__ void store_z(const W4Args &p, int n, int o, float v)
{
    v *= kLarge;
    if (p.bias) v += p.bias[o];
    if (p.relu) v = v < 0.f ? 0.f : v;
    const size_t at = (size_t)n * p.Out + o;
    if (p.z_bf16) static_cast<bf16_t *>(p.z)[at] = f32_to_bf16(v);
    else static_cast<float *>(p.z)[at] = v;
}

// Sums of 16 lanes, in each of them.
__device__ __forceinline__ float row16_sum(float v)
{
    auto ror = [](float x, auto n) __attribute__((always_inline)) {
        return __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(x), 0x120 + decltype(n)::value, 0xf, 0xf, true));
    };
    v += ror(v, std::integral_constant<int, 8>{});
    v += ror(v, std::integral_constant<int, 4>{});
    v += ror(v, std::integral_constant<int, 2>{});
    return v + ror(v, std::integral_constant<int, 1>{});
}
// Sums of 64 lanes each of four values, value i in the lanes 16 i...  (Halves and quarters of two values change places and are
// added, so that every addition works on all lanes.)
__device__ __forceinline__ float sum_lanes4(const float (&v)[4])
{
    float h[2];
#pragma unroll
    for (int k = 0; k < 2; ++k) {
        const auto s = __builtin_amdgcn_permlane32_swap(__float_as_uint(v[k]), __float_as_uint(v[k + 2]), false, false);
        h[k] = __uint_as_float(s[0]) + __uint_as_float(s[1]);
    }
    const auto s = __builtin_amdgcn_permlane16_swap(__float_as_uint(h[0]), __float_as_uint(h[1]), false, false);
    return row16_sum(__uint_as_float(s[0]) + __uint_as_float(s[1]));
}

// One row of a.  A lane keeps 32 consecutive inputs in registers and meets them with the codes of four outputs at a time (one or
// 64 / 2^logl of them a load, 16 bytes a lane), while the next four's are on their way; the waves of a workgroup take the row's
// further slices, and LDS adds up what they find.  Every code is read once, in runs of up to 1 KB.  Bound by that read: 25088 x 4096 in bf16
// takes 12.8 us, with fp32 activations 16.3 us, a mere read of the same 53 MB 9.1 us.  (On the matrix unit with 15 of 16 rows empty: 23.3 us.)
constexpr int kBatch = 4, kRowWaves = 16;
template <typename T>
__global__ __launch_bounds__(kRowWaves * 64) void fc_w4_row_kernel(const T *__restrict__ a_rows, W4Args p, int logl, int batches)
{
    extern __shared__ __align__(16) float sums[];     // [batches][waves][outputs of a batch]
    const T *a = a_rows + (size_t)blockIdx.y * p.In;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, waves = blockDim.x >> 6;
    const int L = 1 << logl, per = 64 >> logl, mine = lane & (L - 1), sub = lane >> logl;
    const int some = kBatch * per, o0 = blockIdx.x * batches * some;
    const int slices = (p.blocks + waves * L - 1) / (waves * L);
    if (batches > (p.Out - o0 + some - 1) / some) batches = (p.Out - o0 + some - 1) / some;
    const char *qbase = reinterpret_cast<const char *>(p.codes) + (size_t)o0 * p.blocks * 16;
    const char *sbase = reinterpret_cast<const char *>(p.scales) + (size_t)o0 * p.groups * 2;

    for (int slice = 0; slice < slices; ++slice) {
        const int b = (slice * waves + wave) * L + mine, left = p.In - b * 32, bc = left > 0 ? b : p.blocks - 1;
        const unsigned grp = (unsigned)(bc * 32) >> p.shift;
        struct Weights { u32x4 q[kBatch]; bf16_t sc[kBatch]; };
        auto fetch = [&](int batch, Weights &w) __attribute__((always_inline)) {
#pragma unroll
            for (int r = 0; r < kBatch; ++r) {
                int o = batch * some + r * per + sub;
                if (o >= p.Out - o0) o = p.Out - 1 - o0;
                w.q[r] = *reinterpret_cast<const u32x4 *>(qbase + ((unsigned)o * p.blocks + bc) * 16u);
                w.sc[r] = *reinterpret_cast<const bf16_t *>(sbase + ((unsigned)o * p.groups + grp) * 2u);
            }
        };
        Weights w0;
        fetch(0, w0);
        constexpr int X = sizeof(T) == 2 ? 4 : 8, E = 16 / (int)sizeof(T);   // 16-byte pieces of 32 inputs, inputs of a piece
        u32x4 x[X];
#pragma unroll
        for (int k = 0; k < X; ++k) {
            const T *xr = a + (size_t)b * 32 + E * k;
            if (left >= E * k + E) x[k] = loose16(xr);
            else {
                T e[E];
#pragma unroll
                for (int j = 0; j < E; ++j) e[j] = E * k + j < left ? xr[j] : (T)0;
                u32x4 v;
                __builtin_memcpy(&v, e, sizeof v);
                x[k] = v;
            }
        }
        auto multiply = [&](const Weights &w, int batch) __attribute__((always_inline)) {
            float acc[kBatch];
#pragma unroll
            for (int r = 0; r < kBatch; ++r) {
                float part[2] = {};
                if constexpr (sizeof(T) == 2) {
                    typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
#pragma unroll
                    for (int k = 0; k < 4; ++k) {
                        const u32x4 c = bf16_values(w.q[r][k]);
#pragma unroll
                        for (int j = 0; j < 4; ++j) {
                            const unsigned cj = c[j], xj = x[k][j];   // (a vector's element is not to be reinterpreted in place)
                            part[j & 1] = __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(bf16x2, cj), __builtin_bit_cast(bf16x2, xj), part[j & 1], false);
                        }
                    }
                } else {
                    auto pair = [&](f32x2 c, int at) __attribute__((always_inline)) {
                        const unsigned x0 = x[at >> 2][at & 3], x1 = x[at >> 2][(at & 3) + 1];
                        part[0] = __builtin_fmaf(c[0], __uint_as_float(x0), part[0]);
                        part[1] = __builtin_fmaf(c[1], __uint_as_float(x1), part[1]);
                    };
#pragma unroll
                    for (int k = 0; k < 4; ++k) {
                        pair(__builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w.q[r][k], kSmall, 0), 8 * k);
                        pair(__builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w.q[r][k], kSmall, 1), 8 * k + 2);
                        pair(__builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w.q[r][k], kSmall, 2), 8 * k + 4);
                        pair(__builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w.q[r][k], kSmall, 3), 8 * k + 6);
                    }
                }
                acc[r] = (left > 0 ? bf16_to_f32(w.sc[r]) : 0.f) * (part[0] + part[1]);
            }
            float *to = sums + (batch * waves + wave) * some;
            if (logl == 6) {
                const float v = sum_lanes4(acc);
                if ((lane & 15) == 0) to[lane >> 4] = slice ? to[lane >> 4] + v : v;
            } else {
#pragma unroll
                for (int o = 16; o > 0; o >>= 1)
                    if (o < L)
#pragma unroll
                        for (int r = 0; r < kBatch; ++r) acc[r] += __shfl_xor(acc[r], o, kWave);
                if (mine == 0)
#pragma unroll
                    for (int r = 0; r < kBatch; ++r) to[r * per + sub] = slice ? to[r * per + sub] + acc[r] : acc[r];
            }
        };
        Weights w1;
        for (int batch = 0; batch < batches; batch += 2) {
            if (batch + 1 < batches) fetch(batch + 1, w1);
            __builtin_amdgcn_sched_barrier(0);
            multiply(w0, batch);
            if (batch + 1 == batches) break;
            if (batch + 2 < batches) fetch(batch + 2, w0);
            __builtin_amdgcn_sched_barrier(0);
            multiply(w1, batch + 1);
        }
    }
    __syncthreads();
    for (int i = threadIdx.x; i < batches * some; i += blockDim.x) {
        const int batch = i / some, at = i - batch * some;
        float v = 0.f;
        for (int w = 0; w < waves; ++w) v += sums[(batch * waves + w) * some + at];
        if (o0 + i < p.Out) store_z(p, blockIdx.y, o0 + i, v);
    }
}

// Eight fp32 values as three bf16 parts each, cut off, not rounded: 24 bits are exactly three times eight, so that the three
// products with a code's value are exact together.  (An infinity's later parts would be NaN.)
struct Parts8 { u32x4 p[3]; };
__device__ __forceinline__ Parts8 parts_of(const float (&x)[8])
{
    Parts8 o;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        float v[2] = {x[2 * j], x[2 * j + 1]};
#pragma unroll
        for (int k = 0; k < 3; ++k) {
            const unsigned u0 = __float_as_uint(v[0]), u1 = __float_as_uint(v[1]);
            o.p[k][j] = __builtin_amdgcn_perm(u1, u0, 0x07060302u);
            v[0] -= __uint_as_float(u0 & 0xffff0000u);
            v[1] -= __uint_as_float(u1 & 0xffff0000u);
        }
    }
    return o;
}
__device__ __forceinline__ Parts8 parts_of_any(const float (&x)[8])
{
    float most = 0.f;
#pragma unroll
    for (int j = 0; j < 8; ++j) most = fmaxf(most, __builtin_fabsf(x[j]));
    Parts8 o = parts_of(x);
    if (__any(!(most < INFINITY))) {
#pragma unroll
        for (int j = 0; j < 8; ++j)
            if (!(__builtin_fabsf(x[j]) < INFINITY)) {
                const unsigned keep = j & 1 ? 0x0000ffffu : 0xffff0000u;
                o.p[1][j / 2] &= keep;
                o.p[2][j / 2] &= keep;
            }
    }
    return o;
}

// More rows, on the matrix unit (16 x 16 x 32, bf16): rows of a times outputs, an output a column of the result, so that a lane's
// four sums share its scales.  A lane loads 32 codes of one output; the four lanes of an output then exchange them (permlane
// swaps), so that one instruction's 32 inputs are of one group: dword j of lane group g, codes 8j.. of block g, becomes codes 8g..
// of block j.
__device__ __forceinline__ void spread_codes(const u32x4 &q, u32x4 (&w)[4])
{
    const auto s02 = __builtin_amdgcn_permlane32_swap(q[0], q[2], false, false);
    const auto s13 = __builtin_amdgcn_permlane32_swap(q[1], q[3], false, false);
    const auto s01 = __builtin_amdgcn_permlane16_swap(s02[0], s13[0], false, false);
    const auto s23 = __builtin_amdgcn_permlane16_swap(s02[1], s13[1], false, false);
    w[0] = bf16_values(s01[0]);
    w[1] = bf16_values(s01[1]);
    w[2] = bf16_values(s23[0]);
    w[3] = bf16_values(s23[1]);
}
// The scales of 128 inputs of one output, S of them, as loaded.
template <int S> struct Scales { unsigned v[(S + 1) / 2]; };
template <int S> __device__ __forceinline__ Scales<S> load_scales(const bf16_t *src, int left)
{
    Scales<S> o;
    struct __attribute__((packed, aligned(2))) Loose { unsigned v[(S + 1) / 2]; };
    if (S == 1) o.v[0] = src[0];
    else if (left >= S) {
        const Loose l = *reinterpret_cast<const Loose *>(src);
#pragma unroll
        for (int i = 0; i < (S + 1) / 2; ++i) o.v[i] = l.v[i];
    } else
#pragma unroll
        for (int i = 0; i < (S + 1) / 2; ++i) o.v[i] = (2 * i < left ? src[2 * i] : 0u) | (2 * i + 1 < left ? (unsigned)src[2 * i + 1] << 16 : 0u);
    return o;
}
template <int S> __device__ __forceinline__ float scale_of(const Scales<S> &s, int i) { return bf16_to_f32((bf16_t)(s.v[i >> 1] >> 16 * (i & 1))); }
__device__ __forceinline__ f32x4 mfma(const u32x4 &x, const u32x4 &w, f32x4 acc)
{
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, x), __builtin_bit_cast(bf16x8, w), acc, 0, 0, 0);
}

// Up to 16 rows: 16 outputs to a workgroup, whose W waves take every W-th 128 inputs, the next ones' codes, scales and activations
// on their way, and add up in LDS.  Each workgroup reads (and in fp32 splits) all activations, so that it is bound by their way out of
// L2 and, in fp32, by some 200 vector instructions for every 128 inputs, which with few outputs few compute units share (16 x 4096 x 4096,
// bf16: 7.4 us, fp32: 11.9 us; 10 x 4096 x 1000, fp32, 63 workgroups: 9.8 us).
template <typename T, int W, int G>
__global__ __launch_bounds__(W * 64) void fc_w4_tile_kernel(const T *__restrict__ a, W4Args p)
{
    extern __shared__ __align__(16) f32x4 red[];      // [W][64]
    constexpr int S = 4 / G;                           // groups of 128 inputs
    constexpr int Q = sizeof(T) / 2;                   // 16-byte loads of 8 inputs
    constexpr int P = Q == 1 ? 1 : 3;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, col = lane & 15, g = lane >> 4;
    const int o0 = blockIdx.x * 16, o = o0 + col < p.Out ? o0 + col : p.Out - 1;
    const int KB = (p.In + 127) / 128, whole = p.In / 128;
    const T *xr = a + (size_t)(col < p.N ? col : p.N - 1) * p.In + g * 8;
    const u32x4 *qr = reinterpret_cast<const u32x4 *>(p.codes) + (size_t)o * p.blocks + g;
    const bf16_t *sr = p.scales + (size_t)o * p.groups;
    struct Step { u32x4 q; Scales<S> sc; u32x4 x[4][Q]; };
    auto fetch = [&](int kb, Step &f) __attribute__((always_inline)) {
        if (kb < whole) {
            f.q = qr[(size_t)kb * 4];
            f.sc = load_scales<S>(sr + (size_t)kb * S, S);
#pragma unroll
            for (int j = 0; j < 4; ++j)
#pragma unroll
                for (int h = 0; h < Q; ++h) f.x[j][h] = loose16(xr + (size_t)kb * 128 + j * 32 + h * (16 / (int)sizeof(T)));
            return;
        }
        f.q = kb * 4 + g < p.blocks ? qr[(size_t)kb * 4] : u32x4{0, 0, 0, 0};
        f.sc = load_scales<S>(sr + (size_t)kb * S, p.groups - kb * S);
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const int left = p.In - (kb * 128 + j * 32 + g * 8);
            T e[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) e[i] = i < left ? xr[(size_t)kb * 128 + j * 32 + i] : (T)0;
            __builtin_memcpy(f.x[j], e, sizeof e);
        }
    };
    f32x4 total = {0.f, 0.f, 0.f, 0.f};
    auto multiply = [&](const Step &f) __attribute__((always_inline)) {
        u32x4 w[4];
        spread_codes(f.q, w);
        f32x4 acc = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            u32x4 part[P];
            if constexpr (P == 1) part[0] = f.x[j][0];
            else {
                float e[8];
                __builtin_memcpy(e, f.x[j], sizeof e);
                const Parts8 o8 = parts_of_any(e);
#pragma unroll
                for (int k = 0; k < 3; ++k) part[k] = o8.p[k];
            }
#pragma unroll
            for (int k = P - 1; k >= 0; --k) acc = mfma(part[k], w[j], acc);
            if ((j + 1) % G == 0) {
                const float sc = scale_of<S>(f.sc, j / G);
#pragma unroll
                for (int v = 0; v < 4; ++v) total[v] = __builtin_fmaf(sc, acc[v], total[v]);
                acc = f32x4{0.f, 0.f, 0.f, 0.f};
            }
        }
    };
    Step f0, f1;
    int kb = wave;
    if (kb < KB) fetch(kb, f0);
    for (; kb < KB; kb += 2 * W) {
        if (kb + W < KB) fetch(kb + W, f1);
        __builtin_amdgcn_sched_barrier(0);
        multiply(f0);
        if (kb + W >= KB) break;
        if (kb + 2 * W < KB) fetch(kb + 2 * W, f0);
        __builtin_amdgcn_sched_barrier(0);
        multiply(f1);
    }
    // value v of a lane: row 4 g + v of a, output col
    red[wave * 64 + lane] = total;
    __syncthreads();
    const float *all = reinterpret_cast<const float *>(red);
    for (int i = threadIdx.x; i < 256; i += W * 64) {
        const int c = i & 15, row = i >> 4, at = ((row >> 2) * 16 + c) * 4 + (row & 3);   // sixteen threads: outputs of one row
        float v = 0.f;
#pragma unroll
        for (int k = 0; k < W; ++k) v += all[k * 256 + at];
        if (row < p.N && o0 + c < p.Out) store_z(p, row, o0 + c, v);
    }
}

// Activations as the matrix unit takes them: [128 inputs][16 rows][32 inputs][part], 1 KB each, lane l's 16 bytes at 16 l: row
// l % 16, inputs 8 (l / 16)..; zeros past the last row and input.  fp32 ones in their three parts.
template <typename T>
__global__ __launch_bounds__(256) void fc_w4_lay_kernel(const T *__restrict__ a, u32x4 *__restrict__ x, int N, int In, int tiles, unsigned units)
{
    const unsigned u = blockIdx.x * 4 + (threadIdx.x >> 6);     // (128 inputs, tile of rows, 32 inputs)
    if (u >= units) return;
    const int lane = threadIdx.x & 63, j = u & 3, tile = (u >> 2) % tiles, kb = (u >> 2) / tiles;
    const int n = tile * 16 + (lane & 15), k = kb * 128 + j * 32 + (lane >> 4) * 8, left = n < N ? In - k : 0;
    const T *src = a + (size_t)n * In + k;
    T e[8];
    if (left >= 8) {
#pragma unroll
        for (int h = 0; h < (int)sizeof(T) / 2; ++h) {
            const u32x4 v = loose16(src + h * (16 / (int)sizeof(T)));
            __builtin_memcpy(e + h * (16 / (int)sizeof(T)), &v, 16);
        }
    } else
#pragma unroll
        for (int i = 0; i < 8; ++i) e[i] = i < left ? src[i] : (T)0;
    if constexpr (sizeof(T) == 2) {
        u32x4 v;
        __builtin_memcpy(&v, e, 16);
        x[(size_t)u * 64 + lane] = v;
    } else {
        const Parts8 o = parts_of_any(e);
#pragma unroll
        for (int k3 = 0; k3 < 3; ++k3) x[((size_t)u * 3 + k3) * 64 + lane] = o.p[k3];
    }
}

// 16 RT outputs and 16 NT rows to a workgroup, whose eight waves take every eighth 128 inputs of its share and add up in LDS.
// The next 128 inputs' codes and scales and the next few blocks of activations are on their way.  A code is spread once for NT
// products, an activation read once for RT; the products fill a tenth of the time, the rest is the activations' way out of L2 and
// the beginning and end of three launches (100 x 25088 x 4096, bf16: 43.7 us, 470 TFLOP/s, fp32: 80 us; 100 x 4096 x
// 4096: 14.7 us, 24.5 us).
template <int P, int RT, int NT, int G>
__global__ __launch_bounds__(512) void fc_w4_tiles_kernel(const u32x4 *__restrict__ x, W4Args p)
{
    extern __shared__ __align__(16) f32x4 red[];      // [W][NT][64]
    constexpr int W = 8, S = 4 / G, F = NT * 4;        // F: blocks of 16 rows x 32 inputs of a step
    constexpr int AHEAD = P == 1 ? 4 : 2;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, col = lane & 15, g = lane >> 4;
    const int across = p.row_tiles * p.splits, by = blockIdx.x / across, bx = blockIdx.x - by * across;
    const int split = bx / p.row_tiles, o0 = (bx - split * p.row_tiles) * (16 * RT), n0 = by * (16 * NT);
    const int KB = (p.In + 127) / 128, whole = p.In / 128;
    const int kb0 = (int)((long)KB * split / p.splits), kb1 = (int)((long)KB * (split + 1) / p.splits);
    const int tiles = (p.N + 16 * NT - 1) / (16 * NT) * NT;
    f32x4 total[RT][NT] = {};

    unsigned qoff[RT], soff[RT];                       // 32-bit offsets from bases that the wave shares
#pragma unroll
    for (int r = 0; r < RT; ++r) {
        const int o = o0 + r * 16 + col < p.Out ? r * 16 + col : p.Out - 1 - o0;
        qoff[r] = ((unsigned)o * p.blocks + g) * 16u;
        soff[r] = (unsigned)o * p.groups * 2u;
    }
    const char *qbase = reinterpret_cast<const char *>(p.codes) + (size_t)o0 * p.blocks * 16;
    const char *sbase = reinterpret_cast<const char *>(p.scales) + (size_t)o0 * p.groups * 2;
    struct Weights { u32x4 q[RT]; Scales<S> sc[RT]; };
    auto fetch = [&](int kb, Weights &f) __attribute__((always_inline)) {
        const char *qk = qbase + (size_t)kb * 64, *sk = sbase + (size_t)kb * (2 * S);
        const bool all = kb < whole;
#pragma unroll
        for (int r = 0; r < RT; ++r) {
            f.q[r] = all || kb * 4 + g < p.blocks ? *reinterpret_cast<const u32x4 *>(qk + qoff[r]) : u32x4{0, 0, 0, 0};
            f.sc[r] = load_scales<S>(reinterpret_cast<const bf16_t *>(sk + soff[r]), all ? S : p.groups - kb * S);
        }
    };
    // block i of a step (or of the wave's next one)
    u32x4 ring[AHEAD][P];
    auto fetch_x = [&](int kb, int i, u32x4 (&f)[P]) __attribute__((always_inline)) {
        if (i >= F) { i -= F; kb = kb + W < kb1 ? kb + W : kb; }
        const u32x4 *src = x + ((((size_t)kb * tiles + by * NT) * 4 + i) * P) * 64;
#pragma unroll
        for (int k = 0; k < P; ++k) f[k] = src[k * 64 + lane];
    };
    Weights f;
    int kb = kb0 + wave;
    if (kb < kb1) {
        fetch(kb, f);
#pragma unroll
        for (int i = 0; i < AHEAD; ++i) fetch_x(kb, i, ring[i]);
    }
    for (; kb < kb1; kb += W) {
        u32x4 w[RT][4];
        float sc[RT][S];
#pragma unroll
        for (int r = 0; r < RT; ++r) {
            spread_codes(f.q[r], w[r]);
#pragma unroll
            for (int i = 0; i < S; ++i) sc[r][i] = scale_of<S>(f.sc[r], i);
        }
        __builtin_amdgcn_sched_barrier(0);
        if (kb + W < kb1) fetch(kb + W, f);
        f32x4 acc[RT];
#pragma unroll
        for (int i = 0; i < F; ++i) {
            const int j = i & 3, t = i >> 2;
            u32x4 now[P];
#pragma unroll
            for (int k = 0; k < P; ++k) now[k] = ring[i % AHEAD][k];
            fetch_x(kb, i + AHEAD, ring[i % AHEAD]);
#pragma unroll
            for (int r = 0; r < RT; ++r) {
                if (j % G == 0) acc[r] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int k = P - 1; k >= 0; --k) acc[r] = mfma(now[k], w[r][j], acc[r]);
            }
            if ((j + 1) % G == 0)
#pragma unroll
                for (int r = 0; r < RT; ++r)
#pragma unroll
                    for (int v = 0; v < 4; ++v) total[r][t][v] = __builtin_fmaf(sc[r][j / G], acc[r][v], total[r][t][v]);
            __builtin_amdgcn_sched_barrier(0);          // (the loads stay where they are issued, and no more of them: registers)
        }
    }

    // value v of a lane: row 4 g + v of its tile of a, output col
#pragma unroll
    for (int r = 0; r < RT; ++r) {
        if (r) __syncthreads();
#pragma unroll
        for (int t = 0; t < NT; ++t) red[(wave * NT + t) * 64 + lane] = total[r][t];
        __syncthreads();
        const float *all = reinterpret_cast<const float *>(red);
        for (int i = threadIdx.x; i < NT * 256; i += W * 64) {
            // sixteen consecutive threads: sixteen outputs of one row
            const int c = i & 15, row = i >> 4, at = ((row >> 4) * 64 + ((row & 15) >> 2) * 16 + c) * 4 + (row & 3);
            float v = 0.f;
#pragma unroll
            for (int k = 0; k < W; ++k) v += all[k * (NT * 256) + at];
            const int n = n0 + row, o = o0 + r * 16 + c;
            if (n < p.N && o < p.Out) {
                if (p.splits > 1) p.part[((size_t)split * p.N + n) * p.Out + o] = v;
                else store_z(p, n, o, v);
            }
        }
    }
}

// The splits' sums, in order.
__global__ __launch_bounds__(256) void fc_w4_join_kernel(W4Args p)
{
    const size_t count = (size_t)p.N * p.Out, i = (size_t)blockIdx.x * 256 + threadIdx.x;
    if (i >= count) return;
    float v = 0.f;
    for (int s = 0; s < p.splits; ++s) v += p.part[s * count + i];
    store_z(p, (int)(i / (unsigned)p.Out), (int)(i % (unsigned)p.Out), v);
}

inline int shift_of(int group) { return group == 32 ? 5 : group == 64 ? 6 : 7; }

}  // namespace

int w4_quantize(int In, int Out, int group, const float *w, uint8_t *codes, bf16_t *scales, hipStream_t s)
{
    const int groups = (In + group - 1) / group;
    const unsigned units = (unsigned)groups * (group / 8), all = units * (unsigned)Out;
    hipLaunchKernelGGL(w4_quantize_kernel, dim3((all + 255) / 256), dim3(256), 0, s, w, codes, scales, In, (In + 31) / 32, groups, shift_of(group), units, all);
    return launch_status();
}

int w4_dequantize(int In, int Out, int group, const uint8_t *codes, const bf16_t *scales, float *w, hipStream_t s)
{
    const unsigned units = (unsigned)(In + 7) / 8, all = units * (unsigned)Out;
    hipLaunchKernelGGL(w4_dequantize_kernel, dim3((all + 255) / 256), dim3(256), 0, s, codes, scales, w, In, (In + 31) / 32, (In + group - 1) / group,
                       shift_of(group), units, all);
    return launch_status();
}

namespace {

template <typename T, int RT, int NT, int G>
int launch_tiles_of(const T *a, W4Args p, const W4Plan &t, void *ws, hipStream_t s)
{
    constexpr int P = sizeof(T) == 2 ? 1 : 3;
    u32x4 *x = static_cast<u32x4 *>(ws);
    p.part = reinterpret_cast<float *>(static_cast<char *>(ws) + t.lay_bytes);
    p.splits = t.splits;
    p.row_tiles = t.row_tiles;
    const unsigned units = (unsigned)((p.In + 127) / 128) * t.tiles * 4;
    hipLaunchKernelGGL(fc_w4_lay_kernel<T>, dim3((units + 3) / 4), dim3(256), 0, s, a, x, p.N, p.In, t.tiles, units);
    hipLaunchKernelGGL((fc_w4_tiles_kernel<P, RT, NT, G>), dim3((unsigned)(t.row_tiles * t.splits * (t.tiles / NT))), dim3(512), (size_t)8 * NT * 1024, s, x, p);
    if (t.splits > 1) hipLaunchKernelGGL(fc_w4_join_kernel, dim3((unsigned)(((size_t)p.N * p.Out + 255) / 256)), dim3(256), 0, s, p);
    return launch_status();
}
template <typename T, int RT, int NT>
int launch_tiles_by(const T *a, const W4Args &p, const W4Plan &t, void *ws, hipStream_t s)
{
    if (p.shift == 5) return launch_tiles_of<T, RT, NT, 1>(a, p, t, ws, s);
    if (p.shift == 6) return launch_tiles_of<T, RT, NT, 2>(a, p, t, ws, s);
    return launch_tiles_of<T, RT, NT, 4>(a, p, t, ws, s);
}
template <typename T, int NT>
int launch_tiles(const T *a, const W4Args &p, const W4Plan &t, void *ws, hipStream_t s)
{
    if (t.rt == 1) return launch_tiles_by<T, 1, NT>(a, p, t, ws, s);
    if (t.rt == 2) return launch_tiles_by<T, 2, NT>(a, p, t, ws, s);
    return launch_tiles_by<T, 4, NT>(a, p, t, ws, s);
}
template <typename T, int G>
int launch_tile(const T *a, const W4Args &p, hipStream_t s)
{
    constexpr int W = 16;
    hipLaunchKernelGGL((fc_w4_tile_kernel<T, W, G>), dim3((unsigned)((p.Out + 15) / 16)), dim3(W * 64), W * 1024, s, a, p);
    return launch_status();
}
template <typename T>
int launch_rows(const T *a, const W4Args &p, hipStream_t s)
{
    int logl = 6;
    while (logl > 0 && (1 << (logl - 1)) >= p.blocks) --logl;
    const int some = kBatch * (64 >> logl), pieces = (p.blocks + (1 << logl) - 1) >> logl;
    const int slices = (pieces + kRowWaves - 1) / kRowWaves, waves = (pieces + slices - 1) / slices;
    // as many batches to a workgroup as leave the chip 16 waves a compute unit
    const long sets = (p.Out + some - 1) / some, load = sets * waves * p.N;
    int batches = (int)((load + 4095) / 4096);
    if (batches > 64) batches = 64;
    if (batches > sets) batches = (int)sets;
    hipLaunchKernelGGL((fc_w4_row_kernel<T>), dim3((unsigned)((sets + batches - 1) / batches), (unsigned)p.N), dim3(64 * waves),
                       (size_t)batches * waves * some * 4, s, a, p, logl, batches);
    return launch_status();
}
template <typename T>
int fc_w4_of(const T *a, const W4Args &p, void *ws, hipStream_t s)
{
    if (p.N <= kW4FewRows) return launch_rows(a, p, s);
    if (w4_one_tile(sizeof(T) == 2 ? VGG_BF16 : VGG_F32, p.N, p.In)) return p.shift == 5 ? launch_tile<T, 1>(a, p, s) : p.shift == 6 ? launch_tile<T, 2>(a, p, s) : launch_tile<T, 4>(a, p, s);
    const W4Plan t = w4_tiles_plan(sizeof(T) == 2 ? VGG_BF16 : VGG_F32, p.N, p.In, p.Out);
    return t.nt == 1 ? launch_tiles<T, 1>(a, p, t, ws, s) : t.nt == 2 ? launch_tiles<T, 2>(a, p, t, ws, s) : launch_tiles<T, 4>(a, p, t, ws, s);
}

}  // namespace

size_t fc_w4_workspace(int dtype, int N, int In, int Out, int group)
{
    (void)group;
    if (N <= kW4FewRows || w4_one_tile(dtype, N, In)) return 0;
    const W4Plan t = w4_tiles_plan(dtype, N, In, Out);
    return t.lay_bytes + (t.splits > 1 ? round_up((size_t)t.splits * N * Out * 4, 256) : 0);
}

int fc_w4(int dtype, int N, int In, int Out, int group, const void *a, const uint8_t *codes, const bf16_t *scales, const float *bias, void *z,
          int z_dtype, int relu, void *ws, hipStream_t s)
{
    const W4Args p = {codes, scales, bias, z, nullptr, z_dtype == VGG_BF16, relu, N, In, Out, (In + 31) / 32, (In + group - 1) / group,
                      shift_of(group), 1, 0};
    if (dtype == VGG_BF16) return fc_w4_of(static_cast<const bf16_t *>(a), p, ws, s);
    return fc_w4_of(static_cast<const float *>(a), p, ws, s);
}

}  // namespace vgg
