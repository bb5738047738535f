// Dropout's random numbers, and rows eight columns at a time: what the kernels that drop values have in common.
#pragma once
#include "common.h"

namespace vgg {

// Eight neighbouring values as they lie in memory; past the n-th: zeros, and never read or written.
template <typename T> struct Eight;
template <> struct Eight<float> {
    f32x4 lo, hi;
    // What is computed from these values is computed anew after this, not kept in registers.
    __device__ __forceinline__ void forget() { asm volatile("" : "+v"(lo), "+v"(hi)); }
    __device__ __forceinline__ void load(const float *p, int n)
    {
        if (n >= 8) {                      // (rows begin anywhere: 16-byte accesses of 4-byte alignment)
            __builtin_memcpy(&lo, p, 16);
            __builtin_memcpy(&hi, p + 4, 16);
        } else
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                lo[k] = k < n ? p[k] : 0.f;
                hi[k] = k + 4 < n ? p[k + 4] : 0.f;
            }
    }
    __device__ __forceinline__ void store(float *p, int n) const
    {
        if (n >= 8) {
            __builtin_memcpy(p, &lo, 16);
            __builtin_memcpy(p + 4, &hi, 16);
        } else
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                if (k < n) p[k] = lo[k];
                if (k + 4 < n) p[k + 4] = hi[k];
            }
    }
    __device__ __forceinline__ float get(int k) const { return k < 4 ? lo[k & 3] : hi[k & 3]; }
    __device__ __forceinline__ void set(const float (&v)[8])
    {
        lo = f32x4{v[0], v[1], v[2], v[3]};
        hi = f32x4{v[4], v[5], v[6], v[7]};
    }
};
// (two to a register: numbers of 16 bits by themselves would take one each)
template <> struct Eight<bf16_t> {
    typedef unsigned u32x4 __attribute__((ext_vector_type(4)));
    u32x4 w;
    __device__ __forceinline__ void forget() { asm volatile("" : "+v"(w)); }
    __device__ __forceinline__ void load(const bf16_t *p, int n)
    {
        if (n >= 8) __builtin_memcpy(&w, p, 16);
        else
#pragma unroll
            for (int k = 0; k < 4; ++k) w[k] = (2 * k < n ? (unsigned)p[2 * k] : 0u) | (2 * k + 1 < n ? (unsigned)p[2 * k + 1] << 16 : 0u);
    }
    __device__ __forceinline__ void store(bf16_t *p, int n) const
    {
        if (n >= 8) __builtin_memcpy(p, &w, 16);
        else
#pragma unroll
            for (int k = 0; k < 8; ++k)
                if (k < n) p[k] = (bf16_t)(k & 1 ? w[k / 2] >> 16 : w[k / 2] & 0xffffu);
    }
    __device__ __forceinline__ float get(int k) const { return __uint_as_float(k & 1 ? w[k / 2] & 0xffff0000u : w[k / 2] << 16); }
    __device__ __forceinline__ void set(const float (&v)[8])
    {
        typedef float f32x2_t __attribute__((ext_vector_type(2)));
        typedef __bf16 bf16x2_t __attribute__((ext_vector_type(2)));
#pragma unroll
        for (int k = 0; k < 4; ++k) w[k] = __builtin_bit_cast(unsigned, __builtin_convertvector(f32x2_t{v[2 * k], v[2 * k + 1]}, bf16x2_t));
    }
};

// What a call drops: numbers below `bar` of 65536.  state: seed and step, in device memory, so that a recorded graph's replays drop anew.
struct Drop {
    const uint64_t *state;   // null: nothing is dropped
    uint32_t layer, bar;     // bar: 65536ths in the upper half (65536 of them: `all`)
    float scale;             // 65536 / (65536 - those)
    int all;
};
inline Drop make_drop(float p, const void *state, unsigned layer)
{
    Drop d;
    const uint32_t of_65536 = (uint32_t)(p * 65536.0 + 0.5);
    d.state = of_65536 ? static_cast<const uint64_t *>(state) : nullptr;
    d.layer = layer;
    d.all = of_65536 == 65536;
    d.bar = d.all ? 0 : of_65536 << 16;
    d.scale = d.all ? 0.f : (float)(65536.0 / (65536 - (int)of_65536));
    return d;
}

// Philox 4x32 with ten rounds (Salmon, Moraes, Dror, Shaw: Parallel random numbers: as easy as 1, 2, 3; SC 2011), one block for eight
// neighbouring columns of a row.  The key and its schedule are the same for all lanes.
struct Philox {
    uint32_t k0, k1, c2, c3;
    __device__ __forceinline__ explicit Philox(const Drop &d)
    {
        const uint64_t seed = d.state[0], step = d.state[1];
        k0 = (uint32_t)seed;
        k1 = (uint32_t)(seed >> 32);
        c2 = (uint32_t)step;
        c3 = ((uint32_t)(step >> 32) & 0xffffu) | d.layer << 16;
    }
    // Bit k: column 8 group + k of the row is kept.  A number in a word's upper half is at least the bar where the word is at least the bar's
    // 65536-fold.
    __device__ __forceinline__ unsigned kept(uint32_t group, uint32_t row, const Drop &d) const
    {
        uint32_t x0 = group, x1 = row, x2 = c2, x3 = c3, a = k0, b = k1;
#pragma unroll
        for (int r = 0; r < 10; ++r) {
            const uint64_t p = (uint64_t)x0 * 0xD2511F53u, q = (uint64_t)x2 * 0xCD9E8D57u;
            x0 = (uint32_t)(q >> 32) ^ x1 ^ a;
            x1 = (uint32_t)q;
            x2 = (uint32_t)(p >> 32) ^ x3 ^ b;
            x3 = (uint32_t)p;
            a += 0x9E3779B9u;
            b += 0xBB67AE85u;
        }
        const uint32_t x[4] = {x0, x1, x2, x3};
        unsigned keep = 0;
#pragma unroll
        for (int k = 0; k < 8; ++k) keep |= (k & 1 ? x[k / 2] : x[k / 2] << 16) >= d.bar ? 1u << k : 0u;
        return d.all ? 0u : keep;
    }
};

}  // namespace vgg
