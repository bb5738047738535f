// Dropout's random numbers, and rows eight columns at a time: what the kernels that drop values have in common.
#pragma once
#include "common.h"

namespace vgg {

// 16 bytes of any alignment.
template <typename T> struct __attribute__((packed, aligned(sizeof(T)))) Loose16 { T v[16 / sizeof(T)]; };

// Eight neighbouring values as they lie in memory; past the n-th: zeros, and never read or written.
template <typename T> struct Eight {
    static constexpr int L = 16 / (int)sizeof(T), P = 8 / L;
    Loose16<T> part[P];
    __device__ __forceinline__ void load(const T *p, int n)
    {
        if (n >= 8) {
#pragma unroll
            for (int h = 0; h < P; ++h) part[h] = *reinterpret_cast<const Loose16<T> *>(p + h * L);
        } else
#pragma unroll
            for (int k = 0; k < 8; ++k) part[k / L].v[k % L] = k < n ? p[k] : T(0);
    }
    __device__ __forceinline__ void store(T *p, int n) const
    {
        if (n >= 8) {
#pragma unroll
            for (int h = 0; h < P; ++h) *reinterpret_cast<Loose16<T> *>(p + h * L) = part[h];
        } else
#pragma unroll
            for (int k = 0; k < 8; ++k)
                if (k < n) p[k] = part[k / L].v[k % L];
    }
    __device__ __forceinline__ float get(int k) const { return Elem<T>::load(&part[k / L].v[k % L]); }
    __device__ __forceinline__ void set(int k, float v) { Elem<T>::store(&part[k / L].v[k % L], v); }
};

// What a call drops: numbers below `bar` of 65536.  state: seed and step, in device memory, so that a recorded graph's replays drop anew.
struct Drop {
    const uint64_t *state;   // null: nothing is dropped
    uint32_t layer, bar;
    float scale;             // 65536 / (65536 - bar)
};
inline Drop make_drop(float p, const void *state, unsigned layer)
{
    Drop d;
    d.bar = (uint32_t)(p * 65536.0 + 0.5);
    d.state = d.bar ? static_cast<const uint64_t *>(state) : nullptr;
    d.layer = layer;
    d.scale = d.bar < 65536 ? (float)(65536.0 / (65536 - (int)d.bar)) : 0.f;
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
    // Bit k: column 8 group + k of the row is kept.
    __device__ __forceinline__ unsigned kept(uint32_t group, uint32_t row, uint32_t bar) const
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
        for (int k = 0; k < 8; ++k) keep |= (unsigned)((k & 1 ? x[k / 2] >> 16 : x[k / 2] & 0xffffu) >= bar) << k;
        return keep;
    }
};

}  // namespace vgg
