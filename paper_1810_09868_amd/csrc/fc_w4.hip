// Dense layers from 4-bit weights with group scales.
//
// A code is a sign and one of 0, 0.5, 1, 1.5, 2, 3, 4, 6 (E2M1); a weight is its value times the bf16 scale of its group of
// consecutive inputs.  Codes lie two to a byte, the even input low, rows padded to 32 codes (16 bytes).
#include "common.h"

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
constexpr int kRows = 4;   // rows of a that a wave holds sums for
template <typename T>
__global__ __launch_bounds__(256) void fc_w4_kernel(const T *__restrict__ a, const uint8_t *__restrict__ codes, const bf16_t *__restrict__ scales,
                                                    const float *__restrict__ bias, void *__restrict__ z, int z_bf16, int relu, int N, int In, int Out,
                                                    int blocks, int shift, int groups)
{
    const int lane = threadIdx.x & 63, o = blockIdx.x * 4 + (threadIdx.x >> 6), n0 = blockIdx.y * kRows;
    if (o >= Out) return;
    float sum[kRows] = {};
    for (int b = lane; b < blocks; b += 64) {
        const u32x4 q = reinterpret_cast<const u32x4 *>(codes)[(size_t)o * blocks + b];
        const float s = bf16_to_f32(scales[(size_t)o * groups + (b * 32 >> shift)]);
        const int n_in = In - b * 32 < 32 ? In - b * 32 : 32;
#pragma unroll
        for (int n = 0; n < kRows; ++n) {
            if (n0 + n >= N) break;
            const T *x = a + (size_t)(n0 + n) * In + b * 32;
            float part = 0.f;
            for (int j = 0; j < n_in; ++j) part = __builtin_fmaf(value_of(q[j >> 3] >> (4 * (j & 7)) & 15u), Elem<T>::load(x + j), part);
            sum[n] = __builtin_fmaf(s, part, sum[n]);
        }
    }
#pragma unroll
    for (int n = 0; n < kRows; ++n) {
        float v = wave_sum(sum[n]);
        if (lane == 0 && n0 + n < N) {
            if (bias) v += bias[o];
            if (relu) v = v < 0.f ? 0.f : v;
            const size_t at = (size_t)(n0 + n) * Out + o;
            if (z_bf16) static_cast<bf16_t *>(z)[at] = f32_to_bf16(v);
            else static_cast<float *>(z)[at] = v;
        }
    }
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

size_t fc_w4_workspace(int dtype, int N, int In, int Out, int group)
{
    (void)dtype; (void)N; (void)In; (void)Out; (void)group;
    return 0;
}

int fc_w4(int dtype, int N, int In, int Out, int group, const void *a, const uint8_t *codes, const bf16_t *scales, const float *bias, void *z,
          int z_dtype, int relu, void *ws, hipStream_t s)
{
    (void)ws;
    const dim3 grid((unsigned)((Out + 3) / 4), (unsigned)((N + kRows - 1) / kRows)), block(256);
    const int blocks = (In + 31) / 32, groups = (In + group - 1) / group, shift = shift_of(group), zb = z_dtype == VGG_BF16;
    if (dtype == VGG_BF16) hipLaunchKernelGGL(fc_w4_kernel<bf16_t>, grid, block, 0, s, static_cast<const bf16_t *>(a), codes, scales, bias, z, zb, relu, N, In, Out, blocks, shift, groups);
    else hipLaunchKernelGGL(fc_w4_kernel<float>, grid, block, 0, s, static_cast<const float *>(a), codes, scales, bias, z, zb, relu, N, In, Out, blocks, shift, groups);
    return launch_status();
}

}  // namespace vgg
