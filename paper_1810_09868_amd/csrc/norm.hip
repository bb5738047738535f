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

// A team of LANES threads has a row, U groups of eight neighbouring values to a thread: group u LANES + thread.  Teams of less than a workgroup
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

// A lane's share of a row: U groups of eight columns, those that are there, and, of the C % 8 columns behind the last whole group, one in
// each of the first lanes.  Groups that are not there are read as the first one and left out of sums: no load hangs on a branch, which
// would cost registers that the rows need.
template <int LANES, int U> struct Columns {
    int C, groups, rest, lane;
    __device__ __forceinline__ Columns(int C_, int lane_) : C(C_), groups(C_ / 8), rest(C_ - C_ / 8 * 8), lane(lane_) {}
    __device__ __forceinline__ int group(int u) const { return u * LANES + lane; }
    __device__ __forceinline__ bool has(int u) const { return group(u) < groups; }
    __device__ __forceinline__ int at(int u) const { return has(u) ? group(u) * 8 : 0; }
    __device__ __forceinline__ bool has_rest() const { return lane < rest; }
    __device__ __forceinline__ int at_rest() const { return has_rest() ? groups * 8 + lane : 0; }
    // how many columns this wave's lanes have
    __device__ __forceinline__ int of_wave() const
    {
        if constexpr (LANES <= 64) return C;
        const int first = lane & ~63;
        int n = first ? 0 : rest;
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int left = groups - u * LANES - first;
            n += 8 * (left < 0 ? 0 : left < 64 ? left : 64);
        }
        return n;
    }
};
// Of the bits that this lane's groups are kept by (a function of u), those of the group that the columns behind the last whole one begin:
// teams within a wave have them from the lane whose place that group would be.
template <int LANES, int U, typename F>
__device__ __forceinline__ unsigned bits_of_rest(const Columns<LANES, U> &cols, const Drop &drop, int row, F bits)
{
    if (!drop.state) return 0xff;
    if constexpr (LANES <= 64 && U > 0) {
        unsigned mine = 0;
#pragma unroll
        for (int u = 0; u < U; ++u) mine = cols.groups / LANES == u ? bits(u) : mine;
        return __shfl(mine, cols.groups % LANES, LANES);
    } else
        return cols.lane < 8 ? Philox(drop).kept(cols.groups, row, drop) : 0;
}
constexpr int at_least_one(int u) { return u ? u : 1; }

// The compiler computes these here, and not where they are used next: it would put a row's groups off until all of their numbers are in
// registers at once.
__device__ __forceinline__ void settle(float (&v)[8])
{
    asm volatile("" : "+v"(v[0]), "+v"(v[1]), "+v"(v[2]), "+v"(v[3]), "+v"(v[4]), "+v"(v[5]), "+v"(v[6]), "+v"(v[7]));
}
__device__ __forceinline__ void settle(float &a, float &b) { asm volatile("" : "+v"(a), "+v"(b)); }

// The row's mean and the sum of the squares around it: those of a wave's values, then of the waves.  in: this lane's groups, one: the column
// behind them.
template <typename T, int LANES, int U>
__device__ __forceinline__ void team_moments(const Columns<LANES, U> &cols, Eight<T> (&in)[at_least_one(U)], float one, int count, float each_of_wave, float each, int turn, float &mean, float &m2)
{
    constexpr int W = LANES / 64, L = LANES < 64 ? LANES : 64;
    float s = cols.has_rest() ? one : 0.f;
#pragma unroll
    for (int u = 0; u < U; ++u) {
        float t = 0.f;
#pragma unroll
        for (int k = 0; k < 8; ++k) t += in[u].get(k);
        s += cols.has(u) ? t : 0.f;
        if constexpr (U > 1) settle(s, t);
    }
    mean = team_sum<L>(s) * each_of_wave;
    m2 = cols.has_rest() ? (one - mean) * (one - mean) : 0.f;
#pragma unroll
    for (int u = 0; u < U; ++u) {
        float t = 0.f;
        in[u].forget();
#pragma unroll
        for (int k = 0; k < 8; ++k) {
            const float d = in[u].get(k) - mean;
            t = __builtin_fmaf(d, d, t);
        }
        m2 += cols.has(u) ? t : 0.f;
        if constexpr (U > 1) settle(m2, t);
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
        mean = all * each;
        m2 = 0.f;
#pragma unroll
        for (int w = 0; w < W; ++w) {
            const float d = part[turn][w][1] - mean;
            m2 += __builtin_fmaf(part[turn][w][0] * d, d, part[turn][w][2]);
        }
    }
}

// 1 / sqrt(v).  The hardware's takes what is below 2^-126 for zeros, so small variances are met 2^64 times as large, and is off by a step of its result, most of which
// one step of Newton's takes away (not of 0 and infinity, whose infinity and 0 stay).  (sqrt and a division, rounded each, take longer: 65536 x 1024 bf16
// 47.7 us for 46.7, 262144 x 64 14.2 for 13.5 without either.)
__device__ __forceinline__ float rstd_of(float v)
{
    const bool small = v < 0x1p-100f;
    const float s = small ? v * 0x1p64f : v, r = __builtin_amdgcn_rsqf(s), left = __builtin_fmaf(-s * r, r, 1.f), near = __builtin_fmaf(0.5f * r, left, r);
    return (left == left ? near : r) * (small ? 0x1p32f : 1.f);
}

// What eight columns are multiplied by, or what is added to them; `other` where there is no such vector.
__device__ __forceinline__ void load_columns(const float *p, int c, int n, float other, float (&v)[8])
{
    Eight<float> e;
    if (p && n > 0) e.load(p + c, n);
#pragma unroll
    for (int k = 0; k < 8; ++k) v[k] = p && k < n ? e.get(k) : other;
}

// y may be x: a row's values are in registers before any of its places is written.
// One read and one write of every value, which bounds it where rows are many (8192 x 25088 bf16: 157 us, 5.2 TB/s; 50001 x 333 fp32 in padded rows with dropout:
// 29 us, 4.6 TB/s).  Few rows are one chain of a load, two sums and a store (1 x 4096 fp32: 3.1 us with the launch, 100 x 4096 bf16 with dropout 4.5).
template <typename T, int LANES, int U>
__global__ __launch_bounds__(kBlock<LANES>) void layer_norm_kernel(Rows r, const T *x, T *y)
{
    constexpr int TEAMS = kBlock<LANES> / LANES, V = at_least_one(U);
    const int lane = threadIdx.x % LANES, team = TEAMS == 1 ? 0 : threadIdx.x / LANES;
    const Columns<LANES, U> cols(r.C, lane);
    const int count = cols.of_wave();
    const float each = 1.f / (float)r.C, each_of_wave = 1.f / (float)(count ? count : 1);
    float gamma[V][8], beta[V][8], gamma1 = 1.f, beta1 = 0.f;
#pragma unroll
    for (int u = 0; u < U; ++u) {
        load_columns(r.gamma, cols.at(u), 8, 1.f, gamma[u]);
        load_columns(r.beta, cols.at(u), 8, 0.f, beta[u]);
    }
    if (r.gamma) gamma1 = r.gamma[cols.at_rest()];
    if (r.beta) beta1 = r.beta[cols.at_rest()];
    int turn = 0;
    Eight<T> in[V];
    T one;
    auto row_at = [&](int row) __attribute__((always_inline)) { return x + (size_t)(row < r.N ? row : r.N - 1) * r.ldx; };
    const T *from = row_at(blockIdx.x * TEAMS + team);
#pragma unroll
    for (int u = 0; u < U; ++u) in[u].load(from + cols.at(u), 8);
    one = from[cols.at_rest()];
    // (all lanes stay: sums go over neighbouring ones)
    for (int base = blockIdx.x * TEAMS; base < r.N; base += gridDim.x * TEAMS, turn ^= 1) {
        const int row = base + team;
        const bool there = row < r.N;
        const float v1 = Elem<T>::load(&one);
        float mean, m2;
        team_moments<T, LANES, U>(cols, in, v1, count, each_of_wave, each, turn, mean, m2);
        const float rstd = rstd_of(__builtin_fmaf(m2, each, r.eps)), scale = r.drop.state ? r.drop.scale : 1.f;
        from = row_at(row + gridDim.x * TEAMS);
        if (r.stats && lane == 0 && there) { r.stats[2 * (size_t)row] = mean; r.stats[2 * (size_t)row + 1] = rstd; }
        T *to = y + (size_t)(there ? row : 0) * r.ldy;
        unsigned kept[V];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const unsigned keep = kept[u] = r.drop.state ? Philox(r.drop).kept(cols.group(u), row, r.drop) : 0xff;
            Eight<T> out;
            float o[8];
            in[u].forget();
            if constexpr (U > 1) __builtin_amdgcn_sched_barrier(0);
#pragma unroll
            for (int k = 0; k < 8; ++k) {
                const float w = __builtin_fmaf((in[u].get(k) - mean) * rstd, gamma[u][k], beta[u][k]) * scale;
                o[k] = keep >> k & 1 ? w : 0.f;
            }
            out.set(o);
            in[u].load(from + cols.at(u), 8);          // the next row's values, while this one's leave
            if (there && cols.has(u)) out.store(to + cols.at(u), 8);
        }
        if (cols.rest) {
            const unsigned keep = bits_of_rest(cols, r.drop, row, [&](int u) { return kept[u]; });
            const float w = __builtin_fmaf((v1 - mean) * rstd, gamma1, beta1) * scale;
            one = from[cols.at_rest()];
            if (there && cols.has_rest()) Elem<T>::store(to + cols.at_rest(), keep >> (lane & 7) & 1 ? w : 0.f);
        }
    }
}

// Rows of any length, met three times by a workgroup of 1024; where y is x, a thread writes what it alone reads.
template <typename T>
__global__ __launch_bounds__(1024) void layer_norm_long_kernel(Rows r, const T *x, T *y)
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
        const float rstd = rstd_of(m2 / (float)r.C + r.eps);
        if (r.stats && threadIdx.x == 0) { r.stats[2 * (size_t)row] = mean; r.stats[2 * (size_t)row + 1] = rstd; }
        for (int c = threadIdx.x * 8; c < r.C; c += 8192) {
            const int n = r.C - c < 8 ? r.C - c : 8;
            Eight<T> in, out;
            in.load(from + c, n);
            float gamma[8], beta[8];
            load_columns(r.gamma, c, n, 1.f, gamma);
            load_columns(r.beta, c, n, 0.f, beta);
            const unsigned keep = r.drop.state ? Philox(r.drop).kept(c / 8, row, r.drop) : 0xff;
            const float scale = r.drop.state ? r.drop.scale : 1.f;
            float o[8];
#pragma unroll
            for (int k = 0; k < 8; ++k) {
                const float w = __builtin_fmaf((in.get(k) - mean) * rstd, gamma[k], beta[k]) * scale;
                o[k] = keep >> k & 1 ? w : 0.f;
            }
            out.set(o);
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

// dgamma and dbeta of 64 columns of all rows by one workgroup: 32 rows at a time, a thread's eight columns.
template <typename T, typename G>
__device__ __forceinline__ void gradients_of_columns(const Rows &r, const T *__restrict__ x, const G *__restrict__ dy, float *dgamma, float *dbeta, int tile, float *lds)
{
    const int at = threadIdx.x & 7, first = threadIdx.x >> 3, c = (tile * 8 + at) * 8, n = r.C - c < 0 ? 0 : r.C - c < 8 ? r.C - c : 8;
    const float scale = r.drop.state ? r.drop.scale : 1.f;
    float sum[2][8] = {};
    for (int row = first; row < r.N; row += 32) {
        Eight<T> xs;
        Eight<G> gs;
        xs.load(x + (size_t)row * r.ldx + c, n);
        gs.load(dy + (size_t)row * r.ldy + c, n);
        const float mean = r.stats[2 * (size_t)row], rstd = r.stats[2 * (size_t)row + 1];
        const unsigned keep = r.drop.state ? Philox(r.drop).kept(c / 8, row, r.drop) : 0xff;
#pragma unroll
        for (int k = 0; k < 8; ++k) {
            const Share s = share_of(xs.get(k), gs.get(k), 1.f, mean, rstd, keep >> k & 1, scale);
            sum[1][k] += s.g;
            sum[0][k] = __builtin_fmaf(s.g, s.xh, sum[0][k]);
        }
    }
    // [32 rows][2][64 columns]
#pragma unroll
    for (int h = 0; h < 2; ++h)
#pragma unroll
        for (int k = 0; k < 8; ++k) lds[first * 129 + h * 64 + at * 8 + k] = sum[h][k];
    __syncthreads();
    if (threadIdx.x >= 128) return;
    float s = 0.f;
#pragma unroll
    for (int k = 0; k < 32; ++k) s += lds[k * 129 + threadIdx.x];
    float *to = threadIdx.x < 64 ? dgamma : dbeta;
    const int col = tile * 64 + (threadIdx.x & 63);
    if (to && col < r.C) to[col] = s;
}
constexpr int kColumnsLds = 32 * 129 * 4;
// Up to this many rows the gradients of gamma and beta are taken by columns, in workgroups of the same launch, which read the rows once more
// (out of L2), instead of from the rows' workgroups by another launch (bf16, 16 to 100 rows of 4096: 6 us
// for 9; 256 rows 6.1 for 12.7; 256 x 333 8.8 for 9.1).
constexpr int kFewRows = 256;

// The gradients' sums over a workgroup's rows go to part [workgroup][2][C] (dgamma, dbeta), or, where there is only one, to where they
// belong.  Two reads and a write of every value bound it (8192 x 25088 bf16: 268 us, 4.6 TB/s, and 20 to join its parts; 50001 x 333 fp32 39 and 7;
// 100 x 4096 bf16, by columns, 5.0).  512 threads with 56 columns each hold the longest rows; 1024 with 28 have too few registers for a row and its next.
template <typename T, typename G, int LANES, int U>
__global__ __launch_bounds__(kBlock<LANES>) void layer_norm_bwd_kernel(Rows r, const T *x, const G *dy, G *dx, float *dgamma, float *dbeta,
                                                                       float *part, int relu_mask, int row_blocks)
{
    // teams of several waves: the waves' sums, then gamma, where U is 7 (the registers do not hold it); else what the teams have to add up
    extern __shared__ __align__(16) float lds[];
    float *lds_gamma = lds + kPlace;
    if constexpr (kBlock<LANES> == 256)
        if ((int)blockIdx.x >= row_blocks) return gradients_of_columns<T, G>(r, x, dy, dgamma, dbeta, blockIdx.x - row_blocks, lds);
    constexpr int TEAMS = kBlock<LANES> / LANES, V = at_least_one(U);
    constexpr bool IN_LDS = U == 7;
    const int lane = threadIdx.x % LANES, team = TEAMS == 1 ? 0 : threadIdx.x / LANES;
    const Columns<LANES, U> cols(r.C, lane);
    float gamma[IN_LDS ? 1 : V][8], at_gamma[V][8], at_beta[V][8], gamma1 = 1.f, at_gamma1 = 0.f, at_beta1 = 0.f;
#pragma unroll
    for (int u = 0; u < U; ++u) {
        if constexpr (IN_LDS) {
            float g[8];
            load_columns(r.gamma, cols.at(u), 8, 1.f, g);
#pragma unroll
            for (int k = 0; k < 8; ++k) lds_gamma[cols.group(u) * 8 + k] = g[k];       // (read by this thread only)
        } else
            load_columns(r.gamma, cols.at(u), 8, 1.f, gamma[u]);
#pragma unroll
        for (int k = 0; k < 8; ++k) at_gamma[u][k] = at_beta[u][k] = 0.f;
    }
    if (r.gamma) gamma1 = r.gamma[cols.at_rest()];
    auto gamma_of = [&](int u, int k) __attribute__((always_inline)) { return IN_LDS ? lds_gamma[cols.group(u) * 8 + k] : gamma[IN_LDS ? 0 : u][k]; };
    const float scale = r.drop.state ? r.drop.scale : 1.f, each = 1.f / (float)r.C;
    int turn = 0;
    Eight<T> xs[V];
    Eight<G> gs[V];
    const T *from_x;
    const G *from_g;
    T one_x;
    G one_g;
    auto aim = [&](int row) __attribute__((always_inline)) {
        const size_t at = row < r.N ? row : r.N - 1;
        from_x = x + at * r.ldx;
        from_g = dy + at * r.ldy;
    };
    aim(blockIdx.x * TEAMS + team);
#pragma unroll
    for (int u = 0; u < U; ++u) {
        xs[u].load(from_x + cols.at(u), 8);
        gs[u].load(from_g + cols.at(u), 8);
    }
    one_x = from_x[cols.at_rest()];
    one_g = from_g[cols.at_rest()];
    for (int base = blockIdx.x * TEAMS; base < r.N; base += row_blocks * TEAMS, turn ^= 1) {
        const int row = base + team;
        const bool there = row < r.N;
        unsigned kept[(U + 4) / 4] = {};         // eight bits a group
        const size_t row_there = there ? row : r.N - 1;
        const float mean = r.stats[2 * row_there], rstd = r.stats[2 * row_there + 1];
        float s1 = 0.f, s2 = 0.f;
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const unsigned keep = !there ? 0 : r.drop.state ? Philox(r.drop).kept(cols.group(u), row, r.drop) : 0xff;
            kept[u / 4] |= keep << 8 * (u % 4);
            if constexpr (U > 1) {
                xs[u].forget();
                gs[u].forget();
                __builtin_amdgcn_sched_barrier(0);
            }
            float t1 = 0.f, t2 = 0.f;
#pragma unroll
            for (int k = 0; k < 8; ++k) {
                const Share s = share_of(xs[u].get(k), gs[u].get(k), gamma_of(u, k), mean, rstd, keep >> k & 1, scale);
                at_beta[u][k] += s.g;
                at_gamma[u][k] = __builtin_fmaf(s.g, s.xh, at_gamma[u][k]);
                t1 += s.gg;
                t2 = __builtin_fmaf(s.gg, s.xh, t2);
            }
            s1 += cols.has(u) ? t1 : 0.f;
            s2 += cols.has(u) ? t2 : 0.f;
            if constexpr (U > 1) {
                settle(at_gamma[u]);
                settle(at_beta[u]);
                settle(s1, s2);
            }
        }
        Share rest = {};
        const float v1 = Elem<T>::load(&one_x);
        if (cols.rest) {
            const unsigned bits = bits_of_rest(cols, r.drop, row, [&](int u) { return kept[u / 4] >> 8 * (u % 4); }), keep = there ? bits : 0;
            rest = share_of(v1, Elem<G>::load(&one_g), gamma1, mean, rstd, keep >> (lane & 7) & 1, scale);
            at_beta1 += rest.g;
            at_gamma1 = __builtin_fmaf(rest.g, rest.xh, at_gamma1);
            s1 += cols.has_rest() ? rest.gg : 0.f;
            s2 += cols.has_rest() ? rest.gg * rest.xh : 0.f;
        }
        team_sums<LANES>(s1, s2, turn, reinterpret_cast<float2 *>(lds));
        s1 *= each;
        s2 *= each;
        aim(row + row_blocks * TEAMS);
        G *to = dx + row_there * r.lddx;
#pragma unroll
        for (int u = 0; u < U; ++u) {
            Eight<G> out;
            float o[8];
            xs[u].forget();
            gs[u].forget();
            if constexpr (U > 1) __builtin_amdgcn_sched_barrier(0);
#pragma unroll
            for (int k = 0; k < 8; ++k) {
                const float v = xs[u].get(k);
                const Share s = share_of(v, gs[u].get(k), gamma_of(u, k), mean, rstd, kept[u / 4] >> (8 * (u % 4) + k) & 1, scale);
                const float d = rstd * (s.gg - s1 - s.xh * s2);
                o[k] = !relu_mask || v > 0.f ? d : 0.f;
            }
            out.set(o);
            xs[u].load(from_x + cols.at(u), 8);          // the next row's values, while this one's leave
            gs[u].load(from_g + cols.at(u), 8);
            if (there && cols.has(u)) out.store(to + cols.at(u), 8);
        }
        if (cols.rest) {
            const float d = rstd * (rest.gg - s1 - rest.xh * s2);
            one_x = from_x[cols.at_rest()];
            one_g = from_g[cols.at_rest()];
            if (there && cols.has_rest()) Elem<G>::store(to + cols.at_rest(), !relu_mask || v1 > 0.f ? d : 0.f);
        }
    }
    if (row_blocks < (int)gridDim.x || (!part && !dgamma && !dbeta)) return;
    float *to_gamma = part ? part + (size_t)blockIdx.x * 2 * r.C : dgamma, *to_beta = part ? part + (size_t)blockIdx.x * 2 * r.C + r.C : dbeta;
    if constexpr (TEAMS == 1) {
#pragma unroll
        for (int u = 0; u < U; ++u) {
            if (!cols.has(u)) continue;
            Eight<float> e;
            e.set(at_gamma[u]);
            if (to_gamma) e.store(to_gamma + cols.at(u), 8);
            e.set(at_beta[u]);
            if (to_beta) e.store(to_beta + cols.at(u), 8);
        }
        if (cols.has_rest()) {
            if (to_gamma) to_gamma[cols.at_rest()] = at_gamma1;
            if (to_beta) to_beta[cols.at_rest()] = at_beta1;
        }
    } else {
        constexpr int COLS = LANES * U * 8 + 8;     // [TEAMS][2][COLS], the columns behind the last group in the last eight
        float *mine = lds + team * 2 * COLS;
#pragma unroll
        for (int u = 0; u < U; ++u)
#pragma unroll
            for (int k = 0; k < 8; k += 4) {
                const int c = cols.group(u) * 8 + k;
                *reinterpret_cast<f32x4 *>(mine + c) = f32x4{at_gamma[u][k], at_gamma[u][k + 1], at_gamma[u][k + 2], at_gamma[u][k + 3]};
                *reinterpret_cast<f32x4 *>(mine + COLS + c) = f32x4{at_beta[u][k], at_beta[u][k + 1], at_beta[u][k + 2], at_beta[u][k + 3]};
            }
        if (lane < 8) {
            mine[COLS - 8 + lane] = at_gamma1;
            mine[2 * COLS - 8 + lane] = at_beta1;
        }
        __syncthreads();
        for (int c = threadIdx.x; c < 2 * COLS; c += kBlock<LANES>) {
            const int in = c < COLS ? c : c - COLS, behind = in - (COLS - 8);
            const bool there = behind >= 0 ? behind < cols.rest : in < cols.groups * 8;
            float s = 0.f;
#pragma unroll
            for (int t = 0; t < TEAMS; ++t) s += lds[t * 2 * COLS + c];
            float *to = c < COLS ? to_gamma : to_beta;
            if (to && there) to[behind >= 0 ? cols.groups * 8 + behind : in] = s;
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
            const unsigned keep = r.drop.state ? Philox(r.drop).kept(c / 8, row, r.drop) : 0xff;
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
__global__ __launch_bounds__(256) void layer_norm_bwd_long_kernel(Rows r, const T *x, const G *dy, G *dx, const float *__restrict__ sums, float *part,
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
        const unsigned keep = r.drop.state ? Philox(r.drop).kept(c / 8, row, r.drop) : 0xff;
        float o[8];
#pragma unroll
        for (int k = 0; k < 8; ++k) {
            const float v = xs.get(k);
            const Share s = share_of(v, gs.get(k), gamma[k], mean, rstd, keep >> k & 1, scale);
            at_beta[k] += s.g;
            at_gamma[k] = __builtin_fmaf(s.g, s.xh, at_gamma[k]);
            const float d = rstd * (s.gg - s1 - s.xh * s2);
            o[k] = !relu_mask || v > 0.f ? d : 0.f;
        }
        out.set(o);
        out.store(dx + (size_t)row * r.lddx + c, n);
    }
    if (!part || n == 0) return;
    Eight<float> e;
    e.set(at_gamma);
    e.store(part + (size_t)range * 2 * r.C + c, n);
    e.set(at_beta);
    e.store(part + (size_t)range * 2 * r.C + r.C + c, n);
}

// part [parts][2][C] added up in order: 16 columns to a workgroup at a time, 64 ranges of parts, then these.
constexpr int kJoinBlocks = 1 << 16;     // (of 1024 threads: a launch has less than 2^32, rows up to 2^30 columns)
__global__ __launch_bounds__(1024) void layer_norm_join_kernel(const float *__restrict__ part, int parts, int C, float *dgamma, float *dbeta)
{
    __shared__ float sums[64][17];
    const int at = threadIdx.x & 15, slice = threadIdx.x >> 4;
    const long all = 2l * C;
    for (long first = (long)blockIdx.x * 16; first < all; first += (long)gridDim.x * 16) {
        const long col = first + at;
        float s = 0.f;
        if (col < all)
            for (int p = slice; p < parts; p += 64) s += part[(size_t)p * all + col];
        sums[slice][at] = s;
        __syncthreads();
        // a wave's 64 lanes have a column's 64 ranges
        const long mine = first + (threadIdx.x >> 6);
        s = team_sum<64>(sums[threadIdx.x & 63][threadIdx.x >> 6]);
        float *to = mine < C ? dgamma : dbeta;
        if (!(threadIdx.x & 63) && mine < all && to) to[mine < C ? mine : mine - C] = s;
        __syncthreads();
    }
}

// A thread has UNITS groups of eight columns, 256 apart, all loaded before the first block of numbers.  Memory bounds it where rows begin at whole 16
// bytes (8192 x 25088 bf16: 150 to 165 us, 5.0 to 5.5 TB/s); 3001 x 4099 fp32 17.7 us, 100 x 4096 bf16 4.7 with the launch.
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
        const unsigned keep = drop.state ? Philox(drop).kept(group[u], row[u], drop) : 0xff;
        float o[8];
#pragma unroll
        for (int k = 0; k < 8; ++k) o[k] = !(keep >> k & 1) ? 0.f : drop.state ? v[u].get(k) * drop.scale : v[u].get(k);
        v[u].set(o);
        v[u].store(y + (size_t)row[u] * ldy + (size_t)group[u] * 8, n[u]);
    }
}

// Which team a row of C values takes: the smallest that holds it.
constexpr int kLongest = 28672;

template <typename F> int by_team(int C, F f)
{
    if (C < 8) return f(std::integral_constant<int, 8>{}, std::integral_constant<int, 0>{});
    if (C <= 64) return f(std::integral_constant<int, 8>{}, std::integral_constant<int, 1>{});
    if (C <= 128) return f(std::integral_constant<int, 16>{}, std::integral_constant<int, 1>{});
    if (C <= 256) return f(std::integral_constant<int, 32>{}, std::integral_constant<int, 1>{});
    if (C <= 512) return f(std::integral_constant<int, 64>{}, std::integral_constant<int, 1>{});
    if (C <= 1024) return f(std::integral_constant<int, 64>{}, std::integral_constant<int, 2>{});
    if (C <= 2048) return f(std::integral_constant<int, 256>{}, std::integral_constant<int, 1>{});
    if (C <= 4096) return f(std::integral_constant<int, 256>{}, std::integral_constant<int, 2>{});
    if (C <= 8192) return f(std::integral_constant<int, 512>{}, std::integral_constant<int, 2>{});
    if (C <= 16384) return f(std::integral_constant<int, 512>{}, std::integral_constant<int, 4>{});
    return f(std::integral_constant<int, 512>{}, std::integral_constant<int, 7>{});
}
// Workgroups that run at once: four of 256 threads to a compute unit, or one of 512.
inline int blocks_at_once(int block) { return block == 256 ? 1024 : 256; }
inline int lanes_of(int C) { return C <= 64 ? 8 : C <= 128 ? 16 : C <= 256 ? 32 : C <= 1024 ? 64 : C <= 4096 ? 256 : 512; }
inline int least(long a, long b) { return (int)(a < b ? a : b); }

// Parts that a backward call's gradients of gamma and beta are summed in.
bool bwd_is_long(int dtype, int g_dtype, int C) { return C > kLongest || (C > 16384 && (dtype == VGG_F32 || g_dtype == VGG_F32)); }
// ... and whether they are taken by columns, in the rows' launch (not where dx takes the place of what they read).
bool bwd_by_columns(int dtype, int g_dtype, int N, int C) { return N <= kFewRows && C <= 4096 && !bwd_is_long(dtype, g_dtype, C); }
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
    const bool sums = dgamma || dbeta, columns = sums && dx != dy && dx != x && bwd_by_columns(dtype, g_dtype, r.N, r.C), is_long = bwd_is_long(dtype, g_dtype, r.C);
    const int parts = bwd_parts(dtype, g_dtype, r.N, r.C);
    float *row_sums = static_cast<float *>(ws), *part = sums && !columns && (parts > 1 || is_long) ? row_sums + (is_long ? 2 * (size_t)((r.N + 1) & ~1) : 0) : nullptr;
    int rc = VGG_OK;
    if (is_long) {
        const int tiles = (r.C + 2047) / 2048;
        layer_norm_bwd_sums_kernel<T, G><<<least(r.N, 512), 1024, 0, s>>>(r, from, dyp, row_sums);
        if ((rc = launch_status()) != VGG_OK) return rc;
        layer_norm_bwd_long_kernel<T, G><<<tiles * parts, 256, 0, s>>>(r, from, dyp, dxp, row_sums, part, relu_mask, tiles);
    } else
        rc = by_team(r.C, [&](auto lanes, auto u) {
            constexpr int LANES = decltype(lanes)::value, U = decltype(u)::value, TEAMS = kBlock<LANES> / LANES;
            if constexpr (U == 7 && (sizeof(T) == 4 || sizeof(G) == 4)) return (int)VGG_ERR_UNSUPPORTED;     // (is_long)
            else {
                auto *kernel = &layer_norm_bwd_kernel<T, G, LANES, U>;
                size_t lds = (TEAMS > 1 ? (size_t)TEAMS * 2 * (LANES * U * 8 + 8) : kPlace + (U == 7 ? kLongest : 0)) * 4;
                if (lds > 65536 && !raise_lds_limit(reinterpret_cast<const void *>(kernel))) return (int)VGG_ERR_LAUNCH;
                if (columns && lds < (size_t)kColumnsLds) lds = kColumnsLds;
                const int grid = parts + (columns ? (r.C + 63) / 64 : 0);
                kernel<<<grid, kBlock<LANES>, lds, s>>>(r, from, dyp, dxp, part ? nullptr : dgamma, part ? nullptr : dbeta, part, relu_mask, parts);
                return (int)VGG_OK;
            }
        });
    if (rc != VGG_OK || (rc = launch_status()) != VGG_OK || !part) return rc;
    layer_norm_join_kernel<<<least((2l * r.C + 15) / 16, kJoinBlocks), 1024, 0, s>>>(part, parts, r.C, dgamma, dbeta);
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
