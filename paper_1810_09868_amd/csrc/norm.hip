// Layer norm of rows, forward and backward, and dropout, by itself and of what a layer norm writes.
//
// Forward: mean and variance of a row (two passes over the values in registers), y = drop(gamma (x - mean) rstd + beta).
// Backward, with g = drop(dy) and xh = (x - mean) rstd:
//     dbeta = sum_n g,  dgamma = sum_n g xh,
//     dx = rstd (g gamma - mean_c(g gamma) - xh mean_c(g gamma xh)),  0 where a ReLU left no x > 0.
// All sums and statistics are fp32; what a bf16 tensor takes is rounded once.
#include "common.h"
#include "dropout.h"
#include "wave.h"

#include <type_traits>

namespace vgg {

namespace {

struct Rows {
    int N, C;
    size_t ldx, ldy, lddx;    // ldy: of y, or of dy
    const float *gamma, *beta;
    float *stats;             // [N][2]: mean, rstd
    float eps;
    Drop drop;
};

// A team of LANES threads has a row, U groups of eight neighbouring values each: group u LANES + thread.  Teams of less than a workgroup
// take a row each of its 256 threads'; teams of several waves exchange their sums through LDS, one barrier a row.
constexpr int kPlace = 64;    // floats of LDS for the sums of up to 16 waves, twice
template <int LANES> constexpr int kBlock = LANES < 256 ? 256 : LANES;

// Sums of two values over the team; `turn` alternates from row to row, so that one barrier is enough.
// The place in LDS is the caller's: [2][LANES / 64].
template <int LANES> __device__ __forceinline__ void team_sums(float &a, float &b, int turn, float2 *place)
{
    constexpr int W = LANES / 64;
    a = team_sum<(LANES < 64 ? LANES : 64)>(a);
    b = team_sum<(LANES < 64 ? LANES : 64)>(b);
    if constexpr (W > 1) {
        float2 *part = place + turn * W;
        if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = make_float2(a, b);
        __syncthreads();
        a = b = 0.f;
#pragma unroll
        for (int w = 0; w < W; ++w) { a += part[w].x; b += part[w].y; }
    }
}

// The row's mean and the sum of the squares around it: those of a wave's values, then of the waves.  A wave has `count` of the row's C
// values, v[u][k] the n[u] first ones of this lane's groups.
template <int LANES, int U> __device__ __forceinline__ void team_moments(const float (&v)[U][8], const int (&n)[U], int C, int turn, float &mean, float &m2)
{
    constexpr int W = LANES / 64, L = LANES < 64 ? LANES : 64;
    int count = C;
    if constexpr (W > 1) {
        count = 0;
        const int first = (threadIdx.x >> 6) * 512;
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int left = C - u * LANES * 8 - first;
            count += left < 0 ? 0 : left < 512 ? left : 512;
        }
    }
    float s = 0.f;
#pragma unroll
    for (int u = 0; u < U; ++u)
#pragma unroll
        for (int k = 0; k < 8; ++k) s += v[u][k];          // (values past the row are zeros)
    mean = count ? team_sum<L>(s) / (float)count : 0.f;
    m2 = 0.f;
#pragma unroll
    for (int u = 0; u < U; ++u)
#pragma unroll
        for (int k = 0; k < 8; ++k) {
            const float d = v[u][k] - mean;
            m2 = k < n[u] ? __builtin_fmaf(d, d, m2) : m2;
        }
    m2 = team_sum<L>(m2);
    if constexpr (W > 1) {
        __shared__ float part[2][W][3];
        if ((threadIdx.x & 63) == 0) {
            float *to = part[turn][threadIdx.x >> 6];
            to[0] = (float)count; to[1] = mean; to[2] = m2;
        }
        __syncthreads();
        float all = 0.f;
#pragma unroll
        for (int w = 0; w < W; ++w) all = __builtin_fmaf(part[turn][w][0], part[turn][w][1], all);
        mean = all / (float)C;
        m2 = 0.f;
#pragma unroll
        for (int w = 0; w < W; ++w) {
            const float d = part[turn][w][1] - mean;
            m2 += __builtin_fmaf(part[turn][w][0] * d, d, part[turn][w][2]);
        }
    }
}

template <int LANES, int U> __device__ __forceinline__ void groups_of_row(int lane, int C, int (&n)[U])
{
#pragma unroll
    for (int u = 0; u < U; ++u) {
        const int left = C - (u * LANES + lane) * 8;
        n[u] = left < 0 ? 0 : left < 8 ? left : 8;
    }
}

// What eight columns are multiplied by, or what is added to them; `other` where there is no such vector.
__device__ __forceinline__ void load_columns(const float *p, int c, int n, float other, float (&v)[8])
{
    Eight<float> e;
    if (p && n > 0) e.load(p + c, n);
#pragma unroll
    for (int k = 0; k < 8; ++k) v[k] = p && k < n ? e.get(k) : other;
}

template <typename T, int LANES, int U>
__global__ __launch_bounds__(kBlock<LANES>) void layer_norm_kernel(Rows r, const T *__restrict__ x, T *y)
{
    constexpr int TEAMS = kBlock<LANES> / LANES;
    constexpr bool KEEP = !(LANES == 1024 && U == 4 && sizeof(T) == 4);     // gamma and beta in registers (128 of them at 1024 threads)
    const int lane = threadIdx.x % LANES, team = threadIdx.x / LANES;
    int n[U];
    groups_of_row<LANES, U>(lane, r.C, n);
    float gamma[U][8], beta[U][8];
    if constexpr (KEEP)
#pragma unroll
        for (int u = 0; u < U; ++u) {
            load_columns(r.gamma, (u * LANES + lane) * 8, n[u], 1.f, gamma[u]);
            load_columns(r.beta, (u * LANES + lane) * 8, n[u], 0.f, beta[u]);
        }
    int turn = 0;
    // (all lanes stay: sums go over neighbouring ones)
    for (int base = blockIdx.x * TEAMS; base < r.N; base += gridDim.x * TEAMS, turn ^= 1) {
        const int row = base + team;
        const bool there = row < r.N;
        Eight<T> in[U];
#pragma unroll
        for (int u = 0; u < U; ++u) in[u].load(x + (there ? (size_t)row * r.ldx + (u * LANES + lane) * 8 : 0), there ? n[u] : 0);
        float v[U][8], mean, m2;
#pragma unroll
        for (int u = 0; u < U; ++u)
#pragma unroll
            for (int k = 0; k < 8; ++k) v[u][k] = in[u].get(k);
        team_moments<LANES, U>(v, n, r.C, turn, mean, m2);
        const float rstd = 1.f / sqrtf(m2 / (float)r.C + r.eps);
        if (!there) continue;
        if (r.stats && lane == 0) { r.stats[2 * (size_t)row] = mean; r.stats[2 * (size_t)row + 1] = rstd; }
#pragma unroll
        for (int u = 0; u < U; ++u) {
            if constexpr (!KEEP) {
                load_columns(r.gamma, (u * LANES + lane) * 8, n[u], 1.f, gamma[u]);
                load_columns(r.beta, (u * LANES + lane) * 8, n[u], 0.f, beta[u]);
            }
            unsigned keep = 0xff;
            float scale = 1.f;
            if (r.drop.state) {
                keep = Philox(r.drop).kept(u * LANES + lane, row, r.drop.bar);
                scale = r.drop.scale;
            }
            Eight<T> out;
#pragma unroll
            for (int k = 0; k < 8; ++k) {
                const float w = __builtin_fmaf((v[u][k] - mean) * rstd, gamma[u][k], beta[u][k]) * scale;
                out.set(k, keep >> k & 1 ? w : 0.f);
            }
            out.store(y + (size_t)row * r.ldy + (u * LANES + lane) * 8, n[u]);
        }
    }
}

// Rows of any length, met three times by a workgroup of 1024.
template <typename T>
__global__ __launch_bounds__(1024) void layer_norm_long_kernel(Rows r, const T *__restrict__ x, T *y)
{
    __shared__ float2 place[32];
    int turn = 0;
    for (int row = blockIdx.x; row < r.N; row += gridDim.x) {
        const T *from = x + (size_t)row * r.ldx;
        float s = 0.f, none = 0.f, m2 = 0.f;
        for (int c = threadIdx.x * 8; c < r.C; c += 8192) {
            Eight<T> in;
            in.load(from + c, r.C - c);
            float t = 0.f;
#pragma unroll
            for (int k = 0; k < 8; ++k) t += in.get(k);
            s += t;
        }
        team_sums<1024>(s, none, turn, place);
        turn ^= 1;
        const float mean = s / (float)r.C;
        for (int c = threadIdx.x * 8; c < r.C; c += 8192) {
            Eight<T> in;
            in.load(from + c, r.C - c);
            float t = 0.f;
#pragma unroll
            for (int k = 0; k < 8; ++k) {
                const float d = in.get(k) - mean;
                t = k < r.C - c ? __builtin_fmaf(d, d, t) : t;
            }
            m2 += t;
        }
        team_sums<1024>(m2, none, turn, place);
        turn ^= 1;
        const float rstd = 1.f / sqrtf(m2 / (float)r.C + r.eps);
        if (r.stats && threadIdx.x == 0) { r.stats[2 * (size_t)row] = mean; r.stats[2 * (size_t)row + 1] = rstd; }
        for (int c = threadIdx.x * 8; c < r.C; c += 8192) {
            const int n = r.C - c < 8 ? r.C - c : 8;
            Eight<T> in, out;
            in.load(from + c, n);
            float gamma[8], beta[8];
            load_columns(r.gamma, c, n, 1.f, gamma);
            load_columns(r.beta, c, n, 0.f, beta);
            const unsigned keep = r.drop.state ? Philox(r.drop).kept(c / 8, row, r.drop.bar) : 0xff;
            const float scale = r.drop.state ? r.drop.scale : 1.f;
#pragma unroll
            for (int k = 0; k < 8; ++k) {
                const float w = __builtin_fmaf((in.get(k) - mean) * rstd, gamma[k], beta[k]) * scale;
                out.set(k, keep >> k & 1 ? w : 0.f);
            }
            out.store(y + (size_t)row * r.ldy + c, n);
        }
    }
}

// One value's share of the gradients: g after dropout, xh, and g gamma.
struct Share { float g, xh, gg; };
__device__ __forceinline__ Share share_of(float x, float dy, float gamma, float mean, float rstd, bool keep, float scale)
{
    Share s;
    s.g = keep ? dy * scale : 0.f;
    s.xh = (x - mean) * rstd;
    s.gg = s.g * gamma;
    return s;
}

// The gradients' sums over a workgroup's rows go to part [workgroup][2][C] (dgamma, dbeta), or, where there is only one, to where they
// belong.
template <typename T, typename G, int LANES, int U>
__global__ __launch_bounds__(kBlock<LANES>) void layer_norm_bwd_kernel(Rows r, const T *__restrict__ x, const G *dy, G *dx, float *dgamma, float *dbeta,
                                                                       float *part, int relu_mask)
{
    // teams of several waves: the waves' sums, then gamma, where U is 4 (128 registers do not hold it at 1024 threads); else what the teams have to add up
    extern __shared__ __align__(16) float lds[];
    float *lds_gamma = lds + kPlace;
    constexpr int TEAMS = kBlock<LANES> / LANES;
    constexpr bool IN_LDS = LANES == 1024 && U == 4;
    const int lane = threadIdx.x % LANES, team = threadIdx.x / LANES;
    int n[U];
    groups_of_row<LANES, U>(lane, r.C, n);
    float gamma[IN_LDS ? 1 : U][8], at_gamma[U][8], at_beta[U][8];
#pragma unroll
    for (int u = 0; u < U; ++u) {
        if constexpr (IN_LDS) {
            float g[8];
            load_columns(r.gamma, (u * LANES + lane) * 8, n[u], 1.f, g);
#pragma unroll
            for (int k = 0; k < 8; ++k) lds_gamma[(u * LANES + lane) * 8 + k] = g[k];       // (read by this thread only)
        } else
            load_columns(r.gamma, (u * LANES + lane) * 8, n[u], 1.f, gamma[u]);
#pragma unroll
        for (int k = 0; k < 8; ++k) at_gamma[u][k] = at_beta[u][k] = 0.f;
    }
    auto gamma_of = [&](int u, int k) __attribute__((always_inline)) { return IN_LDS ? lds_gamma[(u * LANES + lane) * 8 + k] : gamma[IN_LDS ? 0 : u][k]; };
    const float scale = r.drop.state ? r.drop.scale : 1.f, each = 1.f / (float)r.C;
    int turn = 0;
    for (int base = blockIdx.x * TEAMS; base < r.N; base += gridDim.x * TEAMS, turn ^= 1) {
        const int row = base + team;
        const bool there = row < r.N;
        Eight<T> xs[U];
        Eight<G> gs[U];
        unsigned keep[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int c = (u * LANES + lane) * 8, m = there ? n[u] : 0;
            xs[u].load(x + (there ? (size_t)row * r.ldx + c : 0), m);
            gs[u].load(dy + (there ? (size_t)row * r.ldy + c : 0), m);
        }
        const float mean = there ? r.stats[2 * (size_t)row] : 0.f, rstd = there ? r.stats[2 * (size_t)row + 1] : 0.f;
        float s1 = 0.f, s2 = 0.f;
#pragma unroll
        for (int u = 0; u < U; ++u) {
            keep[u] = r.drop.state ? Philox(r.drop).kept(u * LANES + lane, row, r.drop.bar) : 0xff;
            if (!there) keep[u] = 0;
#pragma unroll
            for (int k = 0; k < 8; ++k) {
                const Share s = share_of(xs[u].get(k), gs[u].get(k), gamma_of(u, k), mean, rstd, k < n[u] && keep[u] >> k & 1, scale);
                at_beta[u][k] += s.g;
                at_gamma[u][k] = __builtin_fmaf(s.g, s.xh, at_gamma[u][k]);
                s1 += s.gg;
                s2 = __builtin_fmaf(s.gg, s.xh, s2);
            }
        }
        team_sums<LANES>(s1, s2, turn, reinterpret_cast<float2 *>(lds));
        s1 *= each;
        s2 *= each;
        if (!there) continue;
#pragma unroll
        for (int u = 0; u < U; ++u) {
            Eight<G> out;
#pragma unroll
            for (int k = 0; k < 8; ++k) {
                const float v = xs[u].get(k);
                const Share s = share_of(v, gs[u].get(k), gamma_of(u, k), mean, rstd, keep[u] >> k & 1, scale);
                const float d = rstd * (s.gg - s1 - s.xh * s2);
                out.set(k, !relu_mask || v > 0.f ? d : 0.f);
            }
            out.store(dx + (size_t)row * r.lddx + (u * LANES + lane) * 8, n[u]);
        }
    }
    if (!part && !dgamma && !dbeta) return;
    float *to_gamma = part ? part + (size_t)blockIdx.x * 2 * r.C : dgamma, *to_beta = part ? part + (size_t)blockIdx.x * 2 * r.C + r.C : dbeta;
    if constexpr (TEAMS == 1) {
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int c = (u * LANES + lane) * 8;
            Eight<float> e;
#pragma unroll
            for (int k = 0; k < 8; ++k) e.set(k, at_gamma[u][k]);
            if (to_gamma) e.store(to_gamma + c, n[u]);
#pragma unroll
            for (int k = 0; k < 8; ++k) e.set(k, at_beta[u][k]);
            if (to_beta) e.store(to_beta + c, n[u]);
        }
    } else {
        constexpr int COLS = LANES * U * 8;     // [TEAMS][2][COLS]
        float *mine = lds + team * 2 * COLS;
#pragma unroll
        for (int u = 0; u < U; ++u)
#pragma unroll
            for (int k = 0; k < 8; k += 4) {
                const int c = (u * LANES + lane) * 8 + k;
                *reinterpret_cast<f32x4 *>(mine + c) = f32x4{at_gamma[u][k], at_gamma[u][k + 1], at_gamma[u][k + 2], at_gamma[u][k + 3]};
                *reinterpret_cast<f32x4 *>(mine + COLS + c) = f32x4{at_beta[u][k], at_beta[u][k + 1], at_beta[u][k + 2], at_beta[u][k + 3]};
            }
        __syncthreads();
        for (int c = threadIdx.x; c < 2 * COLS; c += kBlock<LANES>) {
            const int col = c < COLS ? c : c - COLS;
            float s = 0.f;
#pragma unroll
            for (int t = 0; t < TEAMS; ++t) s += lds[t * 2 * COLS + c];
            float *to = c < COLS ? to_gamma : to_beta;
            if (to && col < r.C) to[col] = s;
        }
    }
}

// Rows of any length: a row's two sums first ...
template <typename T, typename G>
__global__ __launch_bounds__(1024) void layer_norm_bwd_sums_kernel(Rows r, const T *__restrict__ x, const G *__restrict__ dy, float *sums)
{
    __shared__ float2 place[32];
    int turn = 0;
    for (int row = blockIdx.x; row < r.N; row += gridDim.x, turn ^= 1) {
        const float mean = r.stats[2 * (size_t)row], rstd = r.stats[2 * (size_t)row + 1], scale = r.drop.state ? r.drop.scale : 1.f;
        float s1 = 0.f, s2 = 0.f;
        for (int c = threadIdx.x * 8; c < r.C; c += 8192) {
            const int n = r.C - c < 8 ? r.C - c : 8;
            Eight<T> xs;
            Eight<G> gs;
            xs.load(x + (size_t)row * r.ldx + c, n);
            gs.load(dy + (size_t)row * r.ldy + c, n);
            float gamma[8], t1 = 0.f, t2 = 0.f;
            load_columns(r.gamma, c, n, 1.f, gamma);
            const unsigned keep = r.drop.state ? Philox(r.drop).kept(c / 8, row, r.drop.bar) : 0xff;
#pragma unroll
            for (int k = 0; k < 8; ++k) {
                const Share s = share_of(xs.get(k), gs.get(k), gamma[k], mean, rstd, k < n && keep >> k & 1, scale);
                t1 += s.gg;
                t2 = __builtin_fmaf(s.gg, s.xh, t2);
            }
            s1 += t1;
            s2 += t2;
        }
        team_sums<1024>(s1, s2, turn, place);
        if (threadIdx.x == 0) { sums[2 * (size_t)row] = s1 / (float)r.C; sums[2 * (size_t)row + 1] = s2 / (float)r.C; }
    }
}
// ... then 2048 columns of a range of rows to a workgroup.
template <typename T, typename G>
__global__ __launch_bounds__(256) void layer_norm_bwd_long_kernel(Rows r, const T *__restrict__ x, const G *dy, G *dx, const float *__restrict__ sums, float *part,
                                                                  int relu_mask, int tiles)
{
    const int tile = blockIdx.x % tiles, range = blockIdx.x / tiles, ranges = gridDim.x / tiles, c = tile * 2048 + threadIdx.x * 8;
    const int n = r.C - c < 0 ? 0 : r.C - c < 8 ? r.C - c : 8;
    const float scale = r.drop.state ? r.drop.scale : 1.f;
    float gamma[8], at_gamma[8] = {}, at_beta[8] = {};
    load_columns(r.gamma, c, n, 1.f, gamma);
    for (int row = range; row < r.N; row += ranges) {
        if (n == 0) break;
        const float mean = r.stats[2 * (size_t)row], rstd = r.stats[2 * (size_t)row + 1], s1 = sums[2 * (size_t)row], s2 = sums[2 * (size_t)row + 1];
        Eight<T> xs;
        Eight<G> gs, out;
        xs.load(x + (size_t)row * r.ldx + c, n);
        gs.load(dy + (size_t)row * r.ldy + c, n);
        const unsigned keep = r.drop.state ? Philox(r.drop).kept(c / 8, row, r.drop.bar) : 0xff;
#pragma unroll
        for (int k = 0; k < 8; ++k) {
            const float v = xs.get(k);
            const Share s = share_of(v, gs.get(k), gamma[k], mean, rstd, keep >> k & 1, scale);
            at_beta[k] += s.g;
            at_gamma[k] = __builtin_fmaf(s.g, s.xh, at_gamma[k]);
            const float d = rstd * (s.gg - s1 - s.xh * s2);
            out.set(k, !relu_mask || v > 0.f ? d : 0.f);
        }
        out.store(dx + (size_t)row * r.lddx + c, n);
    }
    if (!part || n == 0) return;
    Eight<float> e;
#pragma unroll
    for (int k = 0; k < 8; ++k) e.set(k, at_gamma[k]);
    e.store(part + (size_t)range * 2 * r.C + c, n);
#pragma unroll
    for (int k = 0; k < 8; ++k) e.set(k, at_beta[k]);
    e.store(part + (size_t)range * 2 * r.C + r.C + c, n);
}

// part [parts][2][C] added up in order: 64 columns to a workgroup, sixteen ranges of parts, then these.
__global__ __launch_bounds__(1024) void layer_norm_join_kernel(const float *__restrict__ part, int parts, int C, float *dgamma, float *dbeta)
{
    __shared__ float sums[16][64];
    const int at = threadIdx.x & 63, slice = threadIdx.x >> 6;
    const long col = (long)blockIdx.x * 64 + at, all = 2l * C;
    float s = 0.f;
    if (col < all)
        for (int p = slice; p < parts; p += 16) s += part[(size_t)p * all + col];
    sums[slice][at] = s;
    __syncthreads();
    if (slice || col >= all) return;
    s = 0.f;
#pragma unroll
    for (int k = 0; k < 16; ++k) s += sums[k][at];
    float *to = col < C ? dgamma : dbeta;
    if (to) to[col < C ? col : col - C] = s;
}

// A thread has UNITS groups of eight columns, 256 apart.
constexpr int kDropUnits = 4;
template <typename T>
__global__ __launch_bounds__(256) void dropout_kernel(int C, int groups, FastDiv by_groups, int units, int row0, size_t ldx, size_t ldy, const T *x, T *y, Drop drop)
{
    const int first = blockIdx.x * (256 * kDropUnits) + threadIdx.x;
    Eight<T> v[kDropUnits];
    int row[kDropUnits], group[kDropUnits], n[kDropUnits];
#pragma unroll
    for (int u = 0; u < kDropUnits; ++u) {
        const int unit = first + u * 256, at = unit < units ? unit : units - 1;
        row[u] = fast_div(at, by_groups);
        group[u] = at - row[u] * groups;
        row[u] += row0;
        n[u] = unit >= units ? 0 : C - group[u] * 8 < 8 ? C - group[u] * 8 : 8;
        v[u].load(x + (size_t)row[u] * ldx + (size_t)group[u] * 8, n[u]);
    }
#pragma unroll
    for (int u = 0; u < kDropUnits; ++u) {
        const unsigned keep = drop.state ? Philox(drop).kept(group[u], row[u], drop.bar) : 0xff;
#pragma unroll
        for (int k = 0; k < 8; ++k) v[u].set(k, !(keep >> k & 1) ? 0.f : drop.state ? v[u].get(k) * drop.scale : v[u].get(k));
        v[u].store(y + (size_t)row[u] * ldy + (size_t)group[u] * 8, n[u]);
    }
}

// Which team a row of C values takes: the smallest that holds it.
constexpr int kLongest = 32768;

template <typename F> int by_team(int C, F f)
{
    if (C <= 64) return f(std::integral_constant<int, 8>{}, std::integral_constant<int, 1>{});
    if (C <= 128) return f(std::integral_constant<int, 16>{}, std::integral_constant<int, 1>{});
    if (C <= 256) return f(std::integral_constant<int, 32>{}, std::integral_constant<int, 1>{});
    if (C <= 512) return f(std::integral_constant<int, 64>{}, std::integral_constant<int, 1>{});
    if (C <= 1024) return f(std::integral_constant<int, 64>{}, std::integral_constant<int, 2>{});
    if (C <= 2048) return f(std::integral_constant<int, 256>{}, std::integral_constant<int, 1>{});
    if (C <= 4096) return f(std::integral_constant<int, 256>{}, std::integral_constant<int, 2>{});
    if (C <= 8192) return f(std::integral_constant<int, 256>{}, std::integral_constant<int, 4>{});
    if (C <= 16384) return f(std::integral_constant<int, 1024>{}, std::integral_constant<int, 2>{});
    return f(std::integral_constant<int, 1024>{}, std::integral_constant<int, 4>{});
}
// Workgroups that run at once: four of 256 threads to a compute unit, or one of 1024.
inline int blocks_at_once(int block) { return 256 * (1024 / block); }
inline int lanes_of(int C) { return C <= 64 ? 8 : C <= 128 ? 16 : C <= 256 ? 32 : C <= 1024 ? 64 : C <= 8192 ? 256 : 1024; }
inline int least(long a, long b) { return (int)(a < b ? a : b); }

// Parts that a backward call's gradients of gamma and beta are summed in.
bool bwd_is_long(int dtype, int g_dtype, int C) { return C > kLongest || (C > kLongest / 2 && (dtype == VGG_F32 || g_dtype == VGG_F32)); }
int bwd_parts(int dtype, int g_dtype, int N, int C)
{
    if (bwd_is_long(dtype, g_dtype, C)) {
        const int tiles = (C + 2047) / 2048;
        return least(N, tiles >= 1024 ? 1 : 1024 / tiles);
    }
    const int lanes = lanes_of(C), block = lanes < 256 ? 256 : lanes, teams = block / lanes;
    return least((N + teams - 1) / teams, blocks_at_once(block));
}

template <typename T> int forward_of(const Rows &r, const void *x, void *y, hipStream_t s)
{
    const T *from = static_cast<const T *>(x);
    T *to = static_cast<T *>(y);
    if (r.C > kLongest) layer_norm_long_kernel<T><<<least(r.N, 512), 1024, 0, s>>>(r, from, to);
    else
        by_team(r.C, [&](auto lanes, auto u) {
            constexpr int LANES = decltype(lanes)::value, U = decltype(u)::value, TEAMS = kBlock<LANES> / LANES;
            layer_norm_kernel<T, LANES, U><<<least((r.N + TEAMS - 1) / TEAMS, blocks_at_once(kBlock<LANES>)), kBlock<LANES>, 0, s>>>(r, from, to);
            return 0;
        });
    return launch_status();
}

template <typename T, typename G>
int backward_of(const Rows &r, int dtype, int g_dtype, const void *x, const void *dy, void *dx, float *dgamma, float *dbeta, int relu_mask, void *ws, hipStream_t s)
{
    const T *from = static_cast<const T *>(x);
    const G *dyp = static_cast<const G *>(dy);
    G *dxp = static_cast<G *>(dx);
    const bool sums = dgamma || dbeta, is_long = bwd_is_long(dtype, g_dtype, r.C);
    const int parts = bwd_parts(dtype, g_dtype, r.N, r.C);
    float *row_sums = static_cast<float *>(ws), *part = sums && (parts > 1 || is_long) ? row_sums + (is_long ? 2 * (size_t)((r.N + 1) & ~1) : 0) : nullptr;
    int rc = VGG_OK;
    if (is_long) {
        const int tiles = (r.C + 2047) / 2048;
        layer_norm_bwd_sums_kernel<T, G><<<least(r.N, 512), 1024, 0, s>>>(r, from, dyp, row_sums);
        if ((rc = launch_status()) != VGG_OK) return rc;
        layer_norm_bwd_long_kernel<T, G><<<tiles * parts, 256, 0, s>>>(r, from, dyp, dxp, row_sums, part, relu_mask, tiles);
    } else
        rc = by_team(r.C, [&](auto lanes, auto u) {
            constexpr int LANES = decltype(lanes)::value, U = decltype(u)::value, TEAMS = kBlock<LANES> / LANES;
            if constexpr (LANES == 1024 && U == 4 && (sizeof(T) == 4 || sizeof(G) == 4)) return (int)VGG_ERR_UNSUPPORTED;     // (is_long)
            else {
                auto *kernel = &layer_norm_bwd_kernel<T, G, LANES, U>;
                const size_t lds = (TEAMS > 1 ? (size_t)TEAMS * 2 * LANES * U * 8 : kPlace + (LANES == 1024 && U == 4 ? kLongest : 0)) * 4;
                if (lds > 65536 && !raise_lds_limit(reinterpret_cast<const void *>(kernel))) return (int)VGG_ERR_LAUNCH;
                kernel<<<parts, kBlock<LANES>, lds, s>>>(r, from, dyp, dxp, part ? nullptr : dgamma, part ? nullptr : dbeta, part, relu_mask);
                return (int)VGG_OK;
            }
        });
    if (rc != VGG_OK || (rc = launch_status()) != VGG_OK || !part) return rc;
    layer_norm_join_kernel<<<(int)((2l * r.C + 63) / 64), 1024, 0, s>>>(part, parts, r.C, dgamma, dbeta);
    return launch_status();
}

}  // namespace

int layer_norm(int dtype, int N, int C, size_t ldx, const void *x, const float *gamma, const float *beta, float eps, float p, const void *rng, unsigned layer,
               void *y, size_t ldy, float *stats, hipStream_t s)
{
    const Rows r = {N, C, ldx, ldy, 0, gamma, beta, stats, eps, make_drop(p, rng, layer)};
    return dtype == VGG_BF16 ? forward_of<bf16_t>(r, x, y, s) : forward_of<float>(r, x, y, s);
}

size_t layer_norm_bwd_workspace(int dtype, int g_dtype, int N, int C)
{
    const bool is_long = bwd_is_long(dtype, g_dtype, C);
    const int parts = bwd_parts(dtype, g_dtype, N, C);
    return (is_long ? 8 * (size_t)((N + 1) & ~1) : 0) + (parts > 1 || is_long ? (size_t)parts * 8 * C : 0);
}

int layer_norm_bwd(int dtype, int g_dtype, int N, int C, size_t ldx, const void *x, const float *gamma, const float *stats, float p, const void *rng,
                   unsigned layer, size_t lddy, const void *dy, void *dx, size_t lddx, float *dgamma, float *dbeta, int relu_mask, void *ws, hipStream_t s)
{
    const Rows r = {N, C, ldx, lddy, lddx, gamma, nullptr, const_cast<float *>(stats), 0.f, make_drop(p, rng, layer)};
    if (dtype == VGG_F32) return backward_of<float, float>(r, dtype, g_dtype, x, dy, dx, dgamma, dbeta, relu_mask, ws, s);
    if (g_dtype == VGG_F32) return backward_of<bf16_t, float>(r, dtype, g_dtype, x, dy, dx, dgamma, dbeta, relu_mask, ws, s);
    return backward_of<bf16_t, bf16_t>(r, dtype, g_dtype, x, dy, dx, dgamma, dbeta, relu_mask, ws, s);
}

int dropout(int dtype, int N, int C, size_t ldx, const void *x, float p, const void *rng, unsigned layer, void *y, size_t ldy, hipStream_t s)
{
    const Drop drop = make_drop(p, rng, layer);
    const int groups = (C + 7) / 8;
    // a launch's units stay below 2^30
    const long most = groups >= (1 << 30) ? 1 : (1l << 30) / groups;
    for (long row0 = 0; row0 < N; row0 += most) {
        const int rows = least(N - row0, most), units = rows * groups, grid = (units + 256 * kDropUnits - 1) / (256 * kDropUnits);
        if (dtype == VGG_BF16)
            dropout_kernel<bf16_t><<<grid, 256, 0, s>>>(C, groups, make_fast_div(groups), units, (int)row0, ldx, ldy, static_cast<const bf16_t *>(x),
                                                        static_cast<bf16_t *>(y), drop);
        else
            dropout_kernel<float><<<grid, 256, 0, s>>>(C, groups, make_fast_div(groups), units, (int)row0, ldx, ldy, static_cast<const float *>(x),
                                                       static_cast<float *>(y), drop);
        if (const int rc = launch_status()) return rc;
    }
    return VGG_OK;
}

}  // namespace vgg
