// Dense layers from 4-bit weights with group scales.
//
// A code is a sign and one of 0, 0.5, 1, 1.5, 2, 3, 4, 6 (E2M1); a weight is its value times the bf16 scale of its group of
// consecutive inputs.  Codes lie two to a byte, the even input low, rows padded to 32 codes (16 bytes).
#include "common.h"

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

// A lane takes 32 inputs of a group (or what the row has of them): G lanes to a group.
template <int G>
__global__ __launch_bounds__(256) void w4_quantize_kernel(const float *__restrict__ w, uint8_t *__restrict__ codes, bf16_t *__restrict__ scales,
                                                          int In, int Out, int blocks, int groups, size_t units)
{
    const size_t u = (size_t)blockIdx.x * 256 + threadIdx.x;
    const size_t row = u / (unsigned)(groups * G);
    const int b = (int)(u - row * (unsigned)(groups * G)), i0 = b * 32;
    const bool there = u < units && i0 < In;
    const int n = !there ? 0 : In - i0 < 32 ? In - i0 : 32;
    const float *src = w + row * In + i0;
    float v[32];
    float most = 0.f;
    bool bad = false;
#pragma unroll
    for (int j = 0; j < 32; ++j) {
        v[j] = j < n ? src[j] : 0.f;
        most = fmaxf(most, __builtin_fabsf(v[j]));
        bad = bad || !(__builtin_fabsf(v[j]) < INFINITY);
    }
    if (bad) most = INFINITY;
#pragma unroll
    for (int o = 1; o < G; o <<= 1) most = fmaxf(most, __shfl_xor(most, o));
    const bf16_t sb = most < INFINITY ? f32_to_bf16(most * (1.f / 6.f)) : (bf16_t)0x7fc0;
    const float s = bf16_to_f32(sb);
    if (!there) return;
    u32x4 q;
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        unsigned x = 0;
#pragma unroll
        for (int j = 0; j < 8; ++j) x |= code_of(v[8 * k + j], s) << (4 * j);
        q[k] = x;
    }
    reinterpret_cast<u32x4 *>(codes)[row * blocks + b] = q;
    if (b % G == 0) scales[row * groups + b / G] = sb;
}

__device__ __forceinline__ float value_of(unsigned code)
{
    const float mag = code & 4u ? (float)(2u + (code & 1u)) * (code & 2u ? 2.f : 1.f) : 0.5f * (float)(code & 3u);
    return code & 8u ? -mag : mag;
}
__global__ __launch_bounds__(256) void w4_dequantize_kernel(const uint8_t *__restrict__ codes, const bf16_t *__restrict__ scales, float *__restrict__ w,
                                                            int In, int ld, int shift, int groups, int chunks)
{
    const size_t row = blockIdx.x / (unsigned)chunks;
    const int i = (int)(blockIdx.x - row * (unsigned)chunks) * 256 + threadIdx.x;
    if (i >= In) return;
    const unsigned byte = codes[row * ld + i / 2];
    w[row * In + i] = value_of(i & 1 ? byte >> 4 : byte & 15u) * bf16_to_f32(scales[row * groups + (i >> shift)]);
}

// ------------------------------------------------------------------------------------------------- product
// 16 bytes from an address that is a multiple of an element's size only.
struct __attribute__((packed, aligned(2))) Loose16 { unsigned v[4]; };
__device__ __forceinline__ u32x4 loose16(const void *p)
{
    const Loose16 l = *static_cast<const Loose16 *>(p);
    return u32x4{l.v[0], l.v[1], l.v[2], l.v[3]};
}

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

// A few rows of a.  A lane keeps 32 consecutive inputs of each row of a in registers and meets them with R outputs' codes, 16
// bytes a load, 2^logl lanes side by side along an output's row; the waves of a workgroup take the row's further slices, and LDS
// adds up what they find.  Every code is read once and nothing else is read more than once a workgroup.
template <int NV> constexpr int kRowWaves = NV == 1 ? 16 : 8;   // of a workgroup at most: registers
template <typename T, int NV, int R>
__global__ __launch_bounds__(kRowWaves<NV> * 64) void fc_w4_rows_kernel(const T *__restrict__ a, W4Args p, int logl)
{
    extern __shared__ __align__(16) float sums[];     // [waves][outputs][NV]
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, waves = blockDim.x >> 6;
    const int L = 1 << logl, per = 64 >> logl, mine = lane & (L - 1), sub = lane >> logl;
    const int n0 = blockIdx.y * NV, o0 = blockIdx.x * (R * per);
    float acc[R][NV] = {};
    for (int b = wave * L + mine; b - mine < p.blocks; b += waves * L) {
        const bool there = b < p.blocks;
        u32x4 q[R];
        bf16_t sc[R];
#pragma unroll
        for (int r = 0; r < R; ++r) {
            const int o = o0 + r * per + sub;
            const bool ok = there && o < p.Out;
            q[r] = ok ? reinterpret_cast<const u32x4 *>(p.codes)[(size_t)o * p.blocks + b] : u32x4{0, 0, 0, 0};
            sc[r] = ok ? p.scales[(size_t)o * p.groups + (b * 32 >> p.shift)] : (bf16_t)0;
        }
        const int left = there ? p.In - b * 32 : 0;
        if constexpr (sizeof(T) == 2) {
            u32x4 x[NV][4];
#pragma unroll
            for (int n = 0; n < NV; ++n) {
                const T *xr = a + (size_t)(n0 + n < p.N ? n0 + n : p.N - 1) * p.In + (size_t)b * 32;
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    if (left >= 8 * k + 8) x[n][k] = loose16(xr + 8 * k);
                    else {
                        unsigned short e[8];
#pragma unroll
                        for (int j = 0; j < 8; ++j) e[j] = 8 * k + j < left ? xr[8 * k + j] : (unsigned short)0;
#pragma unroll
                        for (int j = 0; j < 4; ++j) x[n][k][j] = e[2 * j] | (unsigned)e[2 * j + 1] << 16;
                    }
                }
            }
#pragma unroll
            for (int r = 0; r < R; ++r) {
                float part[NV] = {};
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    const u32x4 w = bf16_values(q[r][k]);
#pragma unroll
                    for (int n = 0; n < NV; ++n)
#pragma unroll
                        for (int j = 0; j < 4; ++j) {
                            typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
                            const unsigned wj = w[j], xj = x[n][k][j];   // (a vector's element is not to be reinterpreted in place)
                            part[n] = __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(bf16x2, wj), __builtin_bit_cast(bf16x2, xj), part[n], false);
                        }
                }
#pragma unroll
                for (int n = 0; n < NV; ++n) acc[r][n] = __builtin_fmaf(bf16_to_f32(sc[r]), part[n], acc[r][n]);
            }
        } else {
            float x[NV][32];
#pragma unroll
            for (int n = 0; n < NV; ++n) {
                const T *xr = a + (size_t)(n0 + n < p.N ? n0 + n : p.N - 1) * p.In + (size_t)b * 32;
#pragma unroll
                for (int k = 0; k < 8; ++k) {
                    if (left >= 4 * k + 4) {
                        const u32x4 v = loose16(xr + 4 * k);
#pragma unroll
                        for (int j = 0; j < 4; ++j) x[n][4 * k + j] = __uint_as_float(v[j]);
                    } else
#pragma unroll
                        for (int j = 0; j < 4; ++j) x[n][4 * k + j] = 4 * k + j < left ? (float)xr[4 * k + j] : 0.f;
                }
            }
#pragma unroll
            for (int r = 0; r < R; ++r) {
                float part[NV] = {};
                auto pair = [&](f32x2 w, int at) __attribute__((always_inline)) {
#pragma unroll
                    for (int n = 0; n < NV; ++n) part[n] = __builtin_fmaf(w[1], x[n][at + 1], __builtin_fmaf(w[0], x[n][at], part[n]));
                };
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    pair(__builtin_amdgcn_cvt_scalef32_pk_f32_fp4(q[r][k], kSmall, 0), 8 * k);
                    pair(__builtin_amdgcn_cvt_scalef32_pk_f32_fp4(q[r][k], kSmall, 1), 8 * k + 2);
                    pair(__builtin_amdgcn_cvt_scalef32_pk_f32_fp4(q[r][k], kSmall, 2), 8 * k + 4);
                    pair(__builtin_amdgcn_cvt_scalef32_pk_f32_fp4(q[r][k], kSmall, 3), 8 * k + 6);
                }
#pragma unroll
                for (int n = 0; n < NV; ++n) acc[r][n] = __builtin_fmaf(bf16_to_f32(sc[r]), part[n], acc[r][n]);
            }
        }
    }
#pragma unroll
    for (int r = 0; r < R; ++r)
#pragma unroll
        for (int n = 0; n < NV; ++n) {
            float v = acc[r][n];
            for (int o = L >> 1; o > 0; o >>= 1) v += __shfl_xor(v, o, kWave);
            if (mine == 0) sums[(wave * (R * per) + r * per + sub) * NV + n] = v;
        }
    __syncthreads();
    for (int i = threadIdx.x; i < R * per * NV; i += blockDim.x) {
        float v = 0.f;
        for (int w = 0; w < waves; ++w) v += sums[w * (R * per * NV) + i];
        const int o = o0 + i / NV, n = n0 + i % NV;
        if (o < p.Out && n < p.N) store_z(p, n, o, v);
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

// Many rows of a, on the matrix unit (16 x 16 x 32, bf16): rows of a times 16 RT outputs a wave, NT tiles of 16 rows; the waves of
// a workgroup take every W-th 128 inputs and LDS adds them up.  A lane loads 32 codes of one output; the four lanes of an output
// then exchange them (permlane swaps), so that one instruction's 32 inputs are of one group and its sum can take the group's
// scale: an output is a column of the result, so that a lane's four sums share it.
template <typename T, int RT, int NT, int W, int G>
__global__ __launch_bounds__(W * 64) void fc_w4_tiles_kernel(const T *__restrict__ a, W4Args p)
{
    extern __shared__ __align__(16) f32x4 red[];      // [W][NT][64]
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, col = lane & 15, g = lane >> 4;
    const int split = blockIdx.x / p.row_tiles, o0 = (blockIdx.x - split * p.row_tiles) * (16 * RT), n0 = blockIdx.y * (16 * NT);
    const int KB = (p.In + 127) / 128;
    const int kb0 = (int)((long)KB * split / p.splits), kb1 = (int)((long)KB * (split + 1) / p.splits);
    f32x4 total[RT][NT] = {};

    // (32-bit offsets from a base that the wave shares)
    unsigned xoff[NT], qoff[RT], soff[RT];
#pragma unroll
    for (int t = 0; t < NT; ++t) {
        const int n = n0 + t * 16 + col < p.N ? t * 16 + col : p.N - 1 - n0;
        xoff[t] = ((unsigned)n * (unsigned)p.In + g * 8) * (unsigned)sizeof(T);
    }
#pragma unroll
    for (int r = 0; r < RT; ++r) {
        const int o = o0 + r * 16 + col < p.Out ? r * 16 + col : p.Out - 1 - o0;
        qoff[r] = ((unsigned)o * p.blocks + g) * 16u;
        soff[r] = (unsigned)o * p.groups * 2u;
    }
    const char *xbase = reinterpret_cast<const char *>(a + (size_t)n0 * p.In);
    const char *qbase = reinterpret_cast<const char *>(p.codes) + (size_t)o0 * p.blocks * 16;
    const char *sbase = reinterpret_cast<const char *>(p.scales) + (size_t)o0 * p.groups * 2;
    constexpr int S = 4 / G;                           // groups of 128 inputs
    constexpr int Q = sizeof(T) / 2;                   // 16-byte loads of 8 inputs
    constexpr int P = Q == 1 ? 1 : 3;

    // 128 inputs; FULL: all of them are there
    auto step = [&](int kb, auto FULL) __attribute__((always_inline)) {
        constexpr bool full = decltype(FULL)::value;
        const char *xk = xbase + (size_t)kb * (128 * sizeof(T)), *qk = qbase + (size_t)kb * 64, *sk = sbase + (size_t)kb * (2 * S);
        u32x4 q[RT];
        float sc[RT][S];
#pragma unroll
        for (int r = 0; r < RT; ++r) {
            q[r] = full || kb * 4 + g < p.blocks ? *reinterpret_cast<const u32x4 *>(qk + qoff[r]) : u32x4{0, 0, 0, 0};
            if constexpr (full && S == 4) {
                struct __attribute__((packed, aligned(2))) L8 { unsigned v[2]; };
                const L8 v = *reinterpret_cast<const L8 *>(sk + soff[r]);
#pragma unroll
                for (int i = 0; i < S; ++i) sc[r][i] = bf16_to_f32((bf16_t)(v.v[i >> 1] >> 16 * (i & 1)));
            } else if constexpr (full && S == 2) {
                struct __attribute__((packed, aligned(2))) L4 { unsigned v; };
                const L4 v = *reinterpret_cast<const L4 *>(sk + soff[r]);
#pragma unroll
                for (int i = 0; i < S; ++i) sc[r][i] = bf16_to_f32((bf16_t)(v.v >> 16 * (i & 1)));
            } else
#pragma unroll
                for (int i = 0; i < S; ++i) sc[r][i] = kb * S + i < p.groups ? bf16_to_f32(reinterpret_cast<const bf16_t *>(sk + soff[r])[i]) : 0.f;
        }
        // what a tile of 16 rows needs, as loaded: 8 inputs of each of the four blocks
        auto load_x = [&](int t, u32x4 (&x)[4][Q]) __attribute__((always_inline)) {
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const T *xr = reinterpret_cast<const T *>(xk + xoff[t]) + j * 32;
                if constexpr (full) {
#pragma unroll
                    for (int h = 0; h < Q; ++h) x[j][h] = loose16(xr + h * (16 / (int)sizeof(T)));
                } else {
                    const int left = p.In - (kb * 128 + j * 32 + g * 8);
                    T e[8];
#pragma unroll
                    for (int i = 0; i < 8; ++i) e[i] = i < left ? xr[i] : (T)0;
                    __builtin_memcpy(x[j], e, sizeof e);
                }
            }
        };
        u32x4 x[4][Q], next[4][Q];
        load_x(0, x);
        u32x4 w[RT][4];
#pragma unroll
        for (int r = 0; r < RT; ++r) {
            // dword j of lane group g: codes 8j.. of block g  ->  codes 8g.. of block j
            const auto s02 = __builtin_amdgcn_permlane32_swap(q[r][0], q[r][2], false, false);
            const auto s13 = __builtin_amdgcn_permlane32_swap(q[r][1], q[r][3], false, false);
            const auto s01 = __builtin_amdgcn_permlane16_swap(s02[0], s13[0], false, false);
            const auto s23 = __builtin_amdgcn_permlane16_swap(s02[1], s13[1], false, false);
            w[r][0] = bf16_values(s01[0]);
            w[r][1] = bf16_values(s01[1]);
            w[r][2] = bf16_values(s23[0]);
            w[r][3] = bf16_values(s23[1]);
        }
#pragma unroll
        for (int t = 0; t < NT; ++t) {
            if (t + 1 < NT) load_x(t + 1, next);
            if (NT > 1) __builtin_amdgcn_sched_barrier(0);         // (one tile ahead, not all: registers)
            u32x4 part[4][P];
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                if constexpr (P == 1) part[j][0] = x[j][0];
                else {
                    float e[8];
                    __builtin_memcpy(e, x[j], sizeof e);
                    const Parts8 o = parts_of_any(e);
#pragma unroll
                    for (int k = 0; k < 3; ++k) part[j][k] = o.p[k];
                }
            }
#pragma unroll
            for (int r = 0; r < RT; ++r) {
                f32x4 acc = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int j = 0; j < 4; ++j) {
#pragma unroll
                    for (int k = P - 1; k >= 0; --k)
                        acc = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, part[j][k]), __builtin_bit_cast(bf16x8, w[r][j]), acc, 0, 0, 0);
                    if ((j + 1) % G == 0) {
#pragma unroll
                        for (int v = 0; v < 4; ++v) total[r][t][v] = __builtin_fmaf(sc[r][j / G], acc[v], total[r][t][v]);
                        acc = f32x4{0.f, 0.f, 0.f, 0.f};
                    }
                }
                if (RT > 1 && G < 4) __builtin_amdgcn_sched_barrier(0);   // (every group's sum apart would take its registers)
            }
            if (NT > 1) __builtin_amdgcn_sched_barrier(0);
#pragma unroll
            for (int j = 0; j < 4; ++j)
#pragma unroll
                for (int h = 0; h < Q; ++h) x[j][h] = next[j][h];
        }
    };
    const int whole = p.In / 128;
    int kb = kb0 + wave;
    for (; kb < kb1 && kb < whole; kb += W) step(kb, std::true_type{});
    if (kb < kb1) step(kb, std::false_type{});

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
    const int groups = (In + group - 1) / group, blocks = (In + 31) / 32, G = group / 32;
    const size_t units = (size_t)Out * groups * G;
    const dim3 grid((unsigned)((units + 255) / 256)), block(256);
    if (G == 1) hipLaunchKernelGGL(w4_quantize_kernel<1>, grid, block, 0, s, w, codes, scales, In, Out, blocks, groups, units);
    else if (G == 2) hipLaunchKernelGGL(w4_quantize_kernel<2>, grid, block, 0, s, w, codes, scales, In, Out, blocks, groups, units);
    else hipLaunchKernelGGL(w4_quantize_kernel<4>, grid, block, 0, s, w, codes, scales, In, Out, blocks, groups, units);
    return launch_status();
}

int w4_dequantize(int In, int Out, int group, const uint8_t *codes, const bf16_t *scales, float *w, hipStream_t s)
{
    const int chunks = (In + 255) / 256;
    hipLaunchKernelGGL(w4_dequantize_kernel, dim3((unsigned)chunks * (unsigned)Out), dim3(256), 0, s, codes, scales, w, In, (In + 31) / 32 * 16,
                       shift_of(group), (In + group - 1) / group, chunks);
    return launch_status();
}

namespace {

constexpr int kFewRows = 4;    // rows of a up to which the first kernel runs

struct W4Plan { int rt, nt, splits, row_tiles; };
W4Plan tiles_plan(int dtype, int N, int In, int Out)
{
    W4Plan t;
    t.nt = N <= 16 ? 1 : N <= 32 ? 2 : 4;
    t.rt = t.nt <= 2 ? 1 : dtype == VGG_BF16 ? 4 : 2;
    t.row_tiles = (Out + 16 * t.rt - 1) / (16 * t.rt);
    t.splits = 1;
    if (t.rt > 1) {
        const int kb = (In + 127) / 128, most = (kb + 7) / 8;
        const long units = (long)t.row_tiles * ((N + 16 * t.nt - 1) / (16 * t.nt));
        t.splits = (int)(units >= 256 ? 1 : (256 + units - 1) / units);
        if (t.splits > most) t.splits = most;
    }
    return t;
}

template <typename T, int RT, int NT, int W, int G>
int launch_tiles_of(const T *a, const W4Args &p, hipStream_t s)
{
    auto kern = fc_w4_tiles_kernel<T, RT, NT, W, G>;
    const size_t lds = (size_t)W * NT * 1024;
    hipLaunchKernelGGL(kern, dim3((unsigned)(p.row_tiles * p.splits), (unsigned)((p.N + 16 * NT - 1) / (16 * NT))), dim3(W * 64), lds, s, a, p);
    if (p.splits > 1) hipLaunchKernelGGL(fc_w4_join_kernel, dim3((unsigned)(((size_t)p.N * p.Out + 255) / 256)), dim3(256), 0, s, p);
    return launch_status();
}
template <typename T, int RT, int NT, int W>
int launch_tiles(const T *a, const W4Args &p, hipStream_t s)
{
    if (p.shift == 5) return launch_tiles_of<T, RT, NT, W, 1>(a, p, s);
    if (p.shift == 6) return launch_tiles_of<T, RT, NT, W, 2>(a, p, s);
    return launch_tiles_of<T, RT, NT, W, 4>(a, p, s);
}
template <typename T, int NV, int R>
int launch_rows(const T *a, const W4Args &p, hipStream_t s)
{
    int logl = 6;
    while (logl > 0 && (1 << (logl - 1)) >= p.blocks) --logl;
    const int per = R * (64 >> logl);
    int waves = (p.blocks + (1 << logl) - 1) >> logl;
    if (waves > kRowWaves<NV>) waves = kRowWaves<NV>;
    hipLaunchKernelGGL((fc_w4_rows_kernel<T, NV, R>), dim3((unsigned)((p.Out + per - 1) / per), (unsigned)((p.N + NV - 1) / NV)), dim3(64 * waves),
                       (size_t)waves * per * NV * 4, s, a, p, logl);
    return launch_status();
}
template <typename T>
int fc_w4_of(const T *a, W4Args p, hipStream_t s)
{
    if (p.N == 1) return launch_rows<T, 1, 8>(a, p, s);
    if (p.N == 2) return launch_rows<T, 2, 8>(a, p, s);
    if (p.N <= kFewRows) return launch_rows<T, 4, 8>(a, p, s);
    const W4Plan t = tiles_plan(sizeof(T) == 2 ? VGG_BF16 : VGG_F32, p.N, p.In, p.Out);
    p.splits = t.splits;
    p.row_tiles = t.row_tiles;
    if (t.nt == 1) return launch_tiles<T, 1, 1, 16>(a, p, s);
    if (t.nt == 2) return launch_tiles<T, 1, 2, sizeof(T) == 2 ? 16 : 8>(a, p, s);
    constexpr int RT = sizeof(T) == 2 ? 4 : 2;
    return launch_tiles<T, RT, 4, 8>(a, p, s);
}

}  // namespace

size_t fc_w4_workspace(int dtype, int N, int In, int Out, int group)
{
    (void)group;
    if (N <= kFewRows) return 0;
    const W4Plan t = tiles_plan(dtype, N, In, Out);
    return t.splits > 1 ? round_up((size_t)t.splits * N * Out * 4, 256) : 0;
}

int fc_w4(int dtype, int N, int In, int Out, int group, const void *a, const uint8_t *codes, const bf16_t *scales, const float *bias, void *z,
          int z_dtype, int relu, void *ws, hipStream_t s)
{
    const W4Args p = {codes, scales, bias, z, static_cast<float *>(ws), z_dtype == VGG_BF16, relu, N, In, Out, (In + 31) / 32, (In + group - 1) / group,
                      shift_of(group), 1, 0};
    if (dtype == VGG_BF16) return fc_w4_of(static_cast<const bf16_t *>(a), p, s);
    return fc_w4_of(static_cast<const float *>(a), p, s);
}

}  // namespace vgg
