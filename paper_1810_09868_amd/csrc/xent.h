// What the kernels of losses over many classes have in common.
#pragma once
#include "common.h"

namespace vgg {

// Scores in `parts` sums [parts][N][ld] of contraction ranges, without their biases.
struct Scores {
    const float *part;
    int parts, N, classes;
    size_t ld;
    const float *bias;
    // of four neighbouring classes, -inf past the last
    __device__ __forceinline__ f32x4 at(int row, int k) const
    {
        f32x4 z = {};
#pragma unroll 8
        for (int q = 0; q < parts; ++q) z += *reinterpret_cast<const f32x4 *>(part + ((size_t)q * N + row) * ld + k);
#pragma unroll
        for (int j = 0; j < 4; ++j) z[j] = k + j < classes ? z[j] + (bias ? bias[k + j] : 0.f) : -INFINITY;
        return z;
    }
};

// Loss and stats of every row.
int xent_rows(const Scores &z, const int32_t *labels, float *loss, float *stats, hipStream_t s);

// Short fp32 products (xent_is_small): fc_xent_small.hip
size_t fc_xent_small_workspace(int N, int K);
int fc_xent_small(int N, int In, int K, const float *a, const float *w, const float *bias, const int32_t *labels, float *loss, float *stats, void *ws, hipStream_t s);
int fc_xent_small_bwd(int N, int In, int K, const float *a, const float *w, const float *bias, const int32_t *labels, const float *stats, const float *g, float *da, float *dw,
                      float *db, int relu_mask, void *ws, hipStream_t s);

}  // namespace vgg
