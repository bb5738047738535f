// Class scores to log probabilities: of given classes, with every row's entropy and most likely alternatives, and the
// gradient of the first two with respect to the scores.
//
// One pass over a row keeps, with d = z - m and m the largest score so far, E = sum exp(d) over all scores but one of the largest,
// and T = sum d exp(d); a larger score rescales both (S = 1 + E; E' = r S, T' = r (T + (m - m') S), r = exp(m - m')).  Then
//     log p_j = (z_j - m) - log S,   log S = log1p(E),   entropy = log S - T / S,
// E without the largest's own 1, so that the log probability of a class that is all but certain, -E, keeps its digits.  m and
// log S are kept apart (stats): their sum would round what the gradient takes the exponential of.
// All sums are fp32.  A score of -inf has d = -inf, which is raised to kNothing: exp(d) = 0, and its product with d no NaN.
// A NaN makes E, and it or a +inf everything of its row NaN.
#include "common.h"
#include "exp_of.h"
#include "wave.h"

#include <type_traits>

namespace vgg {

namespace {

constexpr int kMaxTop = 64;   // one alternative to a lane

struct Sums { float m, e, t; };   // of no scores: -inf, 0, 0

// E and T of sums that are not the largest's (or are, but count its 1), brought over to the maximum M.
__device__ __forceinline__ void rebase(Sums &a, float M)
{
    const float d = a.m == M ? 0.f : fmaxf(a.m - M, kNothing), r = expf(d), s = a.e + (a.m > -INFINITY ? 1.f : 0.f);
    a.t = r * __builtin_fmaf(d, s, a.t);
    a.e = r * s;
    a.m = M;
}
__device__ __forceinline__ Sums joined(Sums a, Sums b)
{
    if (b.m > a.m) { const Sums c = a; a = b; b = c; }
    rebase(b, a.m);
    return {a.m, a.e + b.e, a.t + b.t};
}

__device__ __forceinline__ Sums wave_joined(Sums a, int lane)
{
    const float M = all_max(a.m);
    if (lane != __builtin_ctzll(__ballot(a.m == M) | 1ull << 63)) rebase(a, M);   // (the first with the largest keeps its E)
    return {M, all_sum(a.e), all_sum(a.t)};
}

// V scores, `most` the largest, into a thread's sums.
template <int V> __device__ __forceinline__ void add_scores(Sums &a, const float (&z)[V], float most)
{
    bool fresh = most > a.m;
    if (fresh) rebase(a, most);
    const float base = a.m == -INFINITY ? 0.f : a.m;
    if (__any(fresh)) {
#pragma unroll
        for (int j = 0; j < V; ++j) {
            const float d = below(z[j] - base), e = exp_of(d);
            const bool it = fresh && z[j] == a.m;      // one of the new largest does not count
            a.e += it ? 0.f : e;
            a.t = __builtin_fmaf(d, e, a.t);
            fresh = fresh && !it;
        }
    } else
#pragma unroll
        for (int j = 0; j < V; ++j) {
            const float d = below(z[j] - base), e = exp_of(d);
            a.e += e;
            a.t = __builtin_fmaf(d, e, a.t);
        }
}

// The same where there is none yet.
template <int V> __device__ __forceinline__ void first_scores(Sums &a, const float (&z)[V], float most)
{
    bool fresh = most > -INFINITY;
    const float base = fresh ? most : 0.f;
    a.m = most;
#pragma unroll
    for (int j = 0; j < V; ++j) {
        const float d = below(z[j] - base), e = exp_of(d);
        const bool it = fresh && z[j] == most;
        a.e += it ? 0.f : e;
        a.t = __builtin_fmaf(d, e, a.t);
        fresh = fresh && !it;
    }
}

// A score and its class as one number: the better, the larger; equal scores: the lower class.  0: none.
typedef unsigned long long Key;
__device__ __forceinline__ Key key_of(float v, int id)
{
    const unsigned b = __float_as_uint(v + 0.f);         // (-0 is 0)
    return (Key)(b ^ ((unsigned)((int)b >> 31) | 0x80000000u)) << 32 | (unsigned)~id;
}
__device__ __forceinline__ float score_of(Key k)
{
    const unsigned b = (unsigned)(k >> 32);
    return __uint_as_float(b & 0x80000000u ? b ^ 0x80000000u : ~b);
}
__device__ __forceinline__ int class_of(Key k) { return (int)~(unsigned)k; }

// The best scores that a wave has seen.  Those that may be among them are put into a list in LDS, which, when it is nearly full
// and at the end, is cut down to the best `top` by counting for each how many are better.  What is not better than the last of
// them (or, before that, than the top-th of the lanes' first scores) is passed over without more than a comparison.
constexpr int kList = 256;
struct Best {
    Key *list;         // [kList], this wave's
    int count, top;
    float worst_v;
    int worst_id;
};
__device__ __forceinline__ bool may_enter(const Best &b, float v, int id) { return v > b.worst_v || (v == b.worst_v && id < b.worst_id); }

// What the wave's lanes have written to LDS is there for all of them.
__device__ __forceinline__ void wave_sync()
{
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
    __builtin_amdgcn_wave_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
}
template <int I> __device__ __forceinline__ void cut_list(Key *list, int count, int top, int lane)
{
    Key mine[I];
    int rank[I];
#pragma unroll
    for (int i = 0; i < I; ++i) {
        mine[i] = lane + 64 * i < count ? list[lane + 64 * i] : 0;
        rank[i] = 0;
    }
    if constexpr (I == 1) {                          // one key to a lane: registers are nearer than LDS
        for (int q = 0; q < count; ++q) {
            const Key k = (Key)(unsigned)__builtin_amdgcn_readlane((int)(mine[0] >> 32), q) << 32 | (unsigned)__builtin_amdgcn_readlane((int)mine[0], q);
            rank[0] += k > mine[0];
        }
    } else {
        int q = 0;
        for (; q + 4 <= count; q += 4) {
            Key k[4];
#pragma unroll
            for (int j = 0; j < 4; ++j) k[j] = list[q + j];
#pragma unroll
            for (int j = 0; j < 4; ++j)
#pragma unroll
                for (int i = 0; i < I; ++i) rank[i] += k[j] > mine[i];
        }
        for (; q < count; ++q) {
            const Key k = list[q];
#pragma unroll
            for (int i = 0; i < I; ++i) rank[i] += k > mine[i];
        }
    }
    wave_sync();
#pragma unroll
    for (int i = 0; i < I; ++i)
        if (mine[i] && rank[i] < top) list[rank[i]] = mine[i];
    wave_sync();
}
__device__ __noinline__ void cut_lists(Key *list, int count, int top, int lane)
{
    if (count <= 64) cut_list<1>(list, count, top, lane);
    else if (count <= 128) cut_list<2>(list, count, top, lane);
    else cut_list<4>(list, count, top, lane);
}
__device__ __forceinline__ void cut(Best &b, int lane)
{
    wave_sync();
    cut_lists(b.list, b.count, b.top, lane);
    if (b.count >= b.top) {
        b.count = b.top;
        const Key last = b.list[b.top - 1];
        b.worst_v = score_of(last);
        b.worst_id = class_of(last);
    }
}
__device__ __forceinline__ void offer(Best &b, float v, int id, int lane)
{
    if (!__any(v >= b.worst_v)) return;
    const Key mask = __ballot(may_enter(b, v, id));
    if (!mask) return;
    const int at = b.count + __builtin_amdgcn_mbcnt_hi((unsigned)(mask >> 32), __builtin_amdgcn_mbcnt_lo((unsigned)mask, 0));
    if (mask >> lane & 1) b.list[at] = key_of(v, id);
    b.count += __builtin_popcountll(mask);
    if (b.count > kList - 64) cut(b, lane);
}
// A bar that at least `top` of a first lot's scores reach, so of all: halvings between the least of the lanes' best
// and the largest bring it near the top-th.  For up to 32 alternatives only the lanes' best are counted, which leaves some 44 scores
// that reach the bar at most.
template <int V> __device__ __forceinline__ void expect(Best &b, const float (&z)[V], float most)
{
    const int lanes = __builtin_popcountll(__ballot(most > -INFINITY));
    if (lanes < b.top) return;
    float lo = all_min(most > -INFINITY ? most : INFINITY), hi = all_max(most);   // (`lanes` scores at least reach lo)
    if (!(hi < INFINITY)) return;                    // (the row's results are NaN)
#pragma unroll 1
    for (int k = 0; k < 8; ++k) {
        const float t = 0.5f * lo + 0.5f * hi;
        int count = 0;
        if (b.top > 32) {
#pragma unroll
            for (int j = 0; j < V; ++j) count += __builtin_popcountll(__ballot(z[j] >= t));
        } else
            count = __builtin_popcountll(__ballot(most >= t));
        const bool enough = count >= b.top;
        lo = enough ? t : lo;
        hi = enough ? hi : t;
    }
    b.worst_v = lo;
    b.worst_id = 0x7fffffff;
}

template <typename T> constexpr int kVec = 16 / (int)sizeof(T);   // scores of a 16-byte load
__device__ __forceinline__ void load_scores(const float *p, float (&z)[4])
{
    const f32x4 v = *reinterpret_cast<const f32x4 *>(p);
#pragma unroll
    for (int j = 0; j < 4; ++j) z[j] = v[j];
}
__device__ __forceinline__ void load_scores(const bf16_t *p, float (&z)[8])
{
    typedef unsigned u32x4 __attribute__((ext_vector_type(4)));
    const u32x4 v = *reinterpret_cast<const u32x4 *>(p);
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        z[2 * j] = __uint_as_float(v[j] << 16);
        z[2 * j + 1] = __uint_as_float(v[j] & 0xffff0000u);
    }
}

struct ScoreArgs {
    int N, K, top, parts, span;   // span: scores of a part
    size_t ldz;
    const int32_t *labels;
    float *logp, *entropy, *top_logp, *stats;
    int32_t *top_idx;
    float *part_sums;             // [N][parts][3]
    Key *part_best;               // [N][parts][top], best first, 0 where there are fewer
};

// Log of a row's sum: -inf where it has no class, NaN with a NaN or +inf.
__device__ __forceinline__ float log_sum(const Sums &r) { return r.m == -INFINITY && r.e == 0.f ? -INFINITY : r.m < INFINITY ? log1pf(r.e) : NAN; }
__device__ __forceinline__ void write_row(const ScoreArgs &a, const Sums &r, float log_s, float z_label, int y, int row)
{
    const bool empty = log_s == -INFINITY;
    if (a.logp) a.logp[row] = y < 0 || y >= a.K ? 0.f : empty ? -INFINITY : (z_label - r.m) - log_s;
    if (a.entropy) a.entropy[row] = empty ? 0.f : log_s - r.t / (1.f + r.e);
    if (a.stats) { a.stats[2 * (size_t)row] = r.m; a.stats[2 * (size_t)row + 1] = log_s; }
}
// Alternative i of a row: `k`, or none.
__device__ __forceinline__ void write_best(const ScoreArgs &a, const Sums &r, float log_s, int row, int i, Key k)
{
    const bool there = k && log_s > -INFINITY;       // (not with a NaN either)
    const size_t at = (size_t)row * a.top + i;
    a.top_logp[at] = there ? (score_of(k) - r.m) - log_s : log_s == log_s ? -INFINITY : log_s;
    a.top_idx[at] = there ? class_of(k) : -1;
}
// The best of W waves' lists, each in order: a thread finds its key's place among all by halving, in every list at a time.
template <int W, typename F> __device__ __forceinline__ void merge_lists(const Key (*lists)[kList], const int *counts, int top, F write)
{
    const int i = threadIdx.x, w = i / top, at = i - w * top;
    int count[W], all = 0;
#pragma unroll
    for (int k = 0; k < W; ++k) all += count[k] = counts[k];
    if (w < W && at < counts[w]) {
        const Key mine = lists[w][at];
        int before[W] = {};
        for (int step = 64; step > 0; step >>= 1) {
            if (step > top) continue;
#pragma unroll
            for (int k = 0; k < W; ++k) {
                const int next = before[k] + step;
                if (next <= count[k] && lists[k][next - 1] > mine) before[k] = next;
            }
        }
        int rank = 0;
#pragma unroll
        for (int k = 0; k < W; ++k) rank += before[k];
        if (rank < top) write(rank, mine);
    }
    if (i < top && i >= all) write(i, (Key)0);
}

// W waves to a row or to a part of one; W == 1: four rows to a workgroup.  A score is read once, in 16-byte loads,
// and lives in registers from there on; long rows are bound by the read and the exponentials beside it (4096 x
// 32768, bf16, four such tensors in turn: 67 us, 4.0 TB/s; 61 us with exponents rounded to fp32), short ones by the launch, one trip to
// memory, and the alternatives: listing and ranking them is a chain of LDS and ballots that nothing hides (100 x 1000, fp32: 3.2 us
// without, 5.5 us with the best five; 4 x 200003, bf16: 7.1 us, 15.3 us with the best twenty).  Rows in order are the slowest, since nearly
// every lot then offers all it has, or the first one all of the best (4 x 200003, bf16, rising or falling: 32 us; 512 x 50001, fp32: 399 us
// rising, 32 us falling, 44 us in any order).
template <typename T, int W, bool TOP>
__global__ __launch_bounds__(256) void log_probs_kernel(const T *__restrict__ z, ScoreArgs a)
{
    constexpr int V = kVec<T>, U = 16 / V;   // sixteen scores a lane at a time
    __shared__ Sums sums[4];
    __shared__ Key lists[TOP ? 4 : 1][kList];
    __shared__ int counts[4];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int unit = W == 1 ? blockIdx.x * 4 + wave : blockIdx.x;
    const int row = a.parts == 1 ? unit : unit / a.parts, part = unit - row * a.parts;
    if (row >= a.N) return;              // (W == 1 only: there is no barrier there)
    const T *zr = z + (size_t)row * a.ldz;
    const int y = a.logp ? a.labels[row] : -1;
    const float z_label = y >= 0 && y < a.K ? Elem<T>::load(zr + y) : 0.f;
    const int k0 = part * a.span, k1 = a.K - k0 < a.span ? a.K : k0 + a.span;
    // whole 16-byte vectors between a head and a tail of fewer scores
    const int off = (int)((reinterpret_cast<uintptr_t>(zr + k0) & 15) / sizeof(T));
    int head = off ? V - off : 0;
    if (head > k1 - k0) head = k1 - k0;
    const int v0 = k0 + head, nvec = (k1 - v0) / V, tail0 = v0 + nvec * V;
    const int ti = W == 1 ? lane : threadIdx.x, tn = W * 64;

    Sums mine = {-INFINITY, 0.f, 0.f};
    Best b = {lists[TOP ? wave : 0], 0, a.top, -INFINITY, -1};
    // head and tail: fewer than 2 V scores, one to a lane of the first wave
    float ends = -INFINITY;
    const int end_k = lane < head ? k0 + lane : tail0 + lane - head;
    if ((W == 1 || wave == 0) && (lane < head || end_k < k1)) ends = Elem<T>::load(zr + end_k);
    // The first lot has the ends among it and no sums before it.  (A short row's time is largely its instructions' own way from memory:
    // with the first lot in the loop, the ends after it and the log of the sum taken twice, 100 x 1000, top 5, took 7.2 us, not 5.4.)
    auto lot = [&](auto is_first, int i0) __attribute__((always_inline)) {
        constexpr bool FIRST = decltype(is_first)::value;
        constexpr int E = U * V + FIRST;
        float x[E];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int i = i0 + u * tn;
            float v[V];
            if (i < nvec) load_scores(zr + v0 + (size_t)i * V, v);
            else
#pragma unroll
                for (int j = 0; j < V; ++j) v[j] = -INFINITY;
#pragma unroll
            for (int j = 0; j < V; ++j) x[u * V + j] = v[j];
        }
        if constexpr (FIRST) x[E - 1] = ends;
        float most = -INFINITY;
#pragma unroll
        for (int j = 0; j < E; ++j) most = fmaxf(most, x[j]);
        if constexpr (TOP && FIRST) expect(b, x, most);
        if constexpr (FIRST) first_scores(mine, x, most);
        else add_scores(mine, x, most);
        if constexpr (TOP)
            if (__any(most >= b.worst_v && most > -INFINITY)) {
                // (a loop over the most that a lane has, its scores read again: 16 offers in a row are more instructions than a
                // short row waits for)
                unsigned some = 0;
#pragma unroll
                for (int j = 0; j < E; ++j) some |= (x[j] >= b.worst_v && x[j] > -INFINITY ? 1u : 0u) << j;
                while (__any(some)) {
                    const int j = some ? __builtin_ctz(some) : 0, k = j < U * V ? v0 + (i0 + j / V * tn) * V + j % V : end_k;
                    offer(b, some ? Elem<T>::load(zr + k) : -INFINITY, k, lane);
                    some &= some - 1;
                }
                if (b.count > b.top + 24 && i0 - ti + U * tn < nvec) cut(b, lane);   // (what follows meets a higher bar)
            }
    };
    lot(std::true_type{}, ti);
    if constexpr (W > 1)                 // (one wave's row is one lot)
        for (int i0 = ti + U * tn; i0 - ti < nvec; i0 += U * tn) lot(std::false_type{}, i0);
    mine = wave_joined(mine, lane);
    if constexpr (TOP) cut(b, lane);

    if constexpr (W == 1) {
        const float log_s = log_sum(mine);
        if (lane == 0) write_row(a, mine, log_s, z_label, y, row);
        if (TOP && lane < a.top) write_best(a, mine, log_s, row, lane, lane < b.count ? b.list[lane] : 0);
    } else {
        if (lane == 0) {
            sums[wave] = mine;
            counts[wave] = b.count;
        }
        __syncthreads();
        mine = sums[0];
        for (int w = 1; w < W; ++w) mine = joined(mine, sums[w]);
        const float log_s = log_sum(mine);
        const size_t at = (size_t)row * a.parts + part;
        if (threadIdx.x == 0) {
            if (a.parts == 1) write_row(a, mine, log_s, z_label, y, row);
            else { a.part_sums[at * 3] = mine.m; a.part_sums[at * 3 + 1] = mine.e; a.part_sums[at * 3 + 2] = mine.t; }
        }
        if constexpr (TOP)
            merge_lists<W>(lists, counts, a.top, [&](int i, Key k) __attribute__((always_inline)) {
                if (a.parts == 1) write_best(a, mine, log_s, row, i, k);
                else a.part_best[at * a.top + i] = k;
            });
    }
}

// The parts of a row: a wave to each row, a part to a lane.  The parts' lists are in order: where no part's r-th best may enter, no
// later one may.  Bound by the launch and by the lists' way from memory, 256 entries at a time (2.5 us; 5.5 us for 4 rows of 49 parts with
// the best twenty; 512 x 50001, top 20, in two parts: 46 us, 58 us with one rank of the parts at a time).
template <typename T, bool TOP>
__global__ __launch_bounds__(64) void log_probs_join_kernel(const T *__restrict__ z, ScoreArgs a)
{
    __shared__ Key list[TOP ? kList : 1];
    const int lane = threadIdx.x, row = blockIdx.x;
    const int y = a.logp ? a.labels[row] : -1;
    const float z_label = y >= 0 && y < a.K ? Elem<T>::load(z + (size_t)row * a.ldz + y) : 0.f;
    const Key *keys = a.part_best + (size_t)row * a.parts * a.top;
    Sums mine = {-INFINITY, 0.f, 0.f};
    for (int p = lane; p < a.parts; p += 64) {
        const float *s = a.part_sums + ((size_t)row * a.parts + p) * 3;
        mine = joined(mine, {s[0], s[1], s[2]});
    }
    Best b = {list, 0, a.top, -INFINITY, -1};
    if constexpr (TOP) {
        const int all = a.parts * a.top;             // (entry e: of part e % parts, its (e / parts)-th)
        auto entry = [&](int e) __attribute__((always_inline)) {
            return e < all ? keys[(size_t)(e % a.parts) * a.top + e / a.parts] : 0;
        };
        constexpr int U = 4;                         // entries of a lane on their way
        for (int e0 = 0, without = 0; e0 < all && without < a.parts; e0 += 64 * U) {
            Key k[U];
            float v[U], most = -INFINITY;
#pragma unroll
            for (int u = 0; u < U; ++u) k[u] = entry(e0 + 64 * u + lane);
#pragma unroll
            for (int u = 0; u < U; ++u) {
                v[u] = k[u] ? score_of(k[u]) : -INFINITY;
                most = fmaxf(most, v[u]);
            }
            if (e0 == 0) expect(b, v, most);
#pragma unroll
            for (int u = 0; u < U; ++u) {
                without = __any(may_enter(b, v[u], class_of(k[u]))) ? 0 : without + 64;
                offer(b, v[u], class_of(k[u]), lane);
            }
            if (b.count >= a.top + 32) cut(b, lane);
        }
        cut(b, lane);
    }
    mine = wave_joined(mine, lane);
    const float log_s = log_sum(mine);
    if (lane == 0) write_row(a, mine, log_s, z_label, y, row);
    if (TOP && lane < a.top) write_best(a, mine, log_s, row, lane, lane < b.count ? list[lane] : 0);
}

// dz_j = g (1[j = y] - p_j) - h p_j (log p_j + entropy); g (1 - p) of the label itself from expm1(log p), which keeps its digits where p is
// all but 1.
struct GradArgs {
    int N, K, span, parts;
    size_t ldz, lddz;
    const int32_t *labels;
    const float *stats, *entropy, *g_logp, *g_entropy;
};
// W waves to a row or to a part of one.  Bound by one read and one write of the scores (4096 x 32768, bf16, four such tensors in turn: 107 us, 5.0 TB/s).
template <typename T, int W>
__global__ __launch_bounds__(256) void log_probs_bwd_kernel(const T *z, T *dz, GradArgs a)
{
    constexpr int V = kVec<T>, TN = W * 64;
    const int tid = threadIdx.x % TN, unit = blockIdx.x * (4 / W) + threadIdx.x / TN;
    const int row = a.parts == 1 ? unit : unit / a.parts, part = unit - row * a.parts;
    if (row >= a.N) return;
    const T *zr = z + (size_t)row * a.ldz;
    T *dr = dz + (size_t)row * a.lddz;
    const int k0 = part * a.span, k1 = a.K - k0 < a.span ? a.K : k0 + a.span;
    int y = a.g_logp ? a.labels[row] : -1;
    if (y < 0 || y >= a.K) y = -1;
    const float g = y >= 0 ? a.g_logp[row] : 0.f;
    const float h = a.g_entropy ? a.g_entropy[row] : 0.f, ent = a.g_entropy ? a.entropy[row] : 0.f;
    const float m = a.stats[2 * (size_t)row], log_s = a.stats[2 * (size_t)row + 1];
    const bool none = m == -INFINITY && log_s == -INFINITY;
    const bool zero = none || (g == 0.f && h == 0.f);
    auto grad = [&](float zj) __attribute__((always_inline)) {
        const float lp = (zj - m) - log_s, p = expf(lp);
        return -p * __builtin_fmaf(h, fmaxf(lp, kNothing) + ent, g);
    };
    auto grad_of_label = [&](float zj) __attribute__((always_inline)) {      // (masked: zero)
        const float lp = (zj - m) - log_s;
        return zj == -INFINITY ? grad(zj) : -__builtin_fmaf(g, expm1f(lp), expf(lp) * h * (fmaxf(lp, kNothing) + ent));
    };
    const int off = (int)((reinterpret_cast<uintptr_t>(zr + k0) & 15) / sizeof(T));
    const bool together = ((reinterpret_cast<uintptr_t>(zr) ^ reinterpret_cast<uintptr_t>(dr)) & 15) == 0;
    int head = together ? (off ? V - off : 0) : k1 - k0;   // scores before the first 16-byte vector; all, where dz has none there
    if (head > k1 - k0) head = k1 - k0;
    const int v0 = k0 + head, nvec = (k1 - v0) / V, tail0 = v0 + nvec * V;
    for (int i = tid; i < nvec; i += TN) {
        float x[V] = {};
        if (!zero) {
            load_scores(zr + v0 + (size_t)i * V, x);
#pragma unroll
            for (int j = 0; j < V; ++j) x[j] = grad(x[j]);
            const int at = y - (v0 + i * V);
            if (at >= 0 && at < V) {                     // (its score once more: this thread has not written it yet)
                const float of_label = grad_of_label(Elem<T>::load(zr + y));
#pragma unroll
                for (int j = 0; j < V; ++j) x[j] = j == at ? of_label : x[j];
            }
        }
#pragma unroll
        for (int j = 0; j < V; j += 4) store4(dr + v0 + (size_t)i * V + j, x[j], x[j + 1], x[j + 2], x[j + 3]);
    }
    for (int i = tid; i < head + (k1 - tail0); i += TN) {
        const int k = i < head ? k0 + i : tail0 + i - head;
        const float zk = zero ? 0.f : Elem<T>::load(zr + k);
        Elem<T>::store(dr + k, zero ? 0.f : k == y ? grad_of_label(zk) : grad(zk));
    }
}

constexpr int kOneWave = 1024;   // scores that one wave takes by itself (16 x 2048, top 5: 9.9 us so, 6.7 us with four waves; 4096 x 1000:
                                 // 9.2 us so, 24 us with four)
struct Split { int parts, span; };
// Rows that are too few to fill the chip are cut into parts of at least 4096 scores (1 x 50000, top 1: 9.7 us, 17.4 us in one part of
// sixteen waves).
Split split_rows(int N, int K)
{
    const int most = (K + 4095) / 4096, want = (1024 + N - 1) / N;
    int parts = want < most ? want : most;
    if (parts < 1) parts = 1;
    const int span = ((K + parts - 1) / parts + 7) / 8 * 8;
    return {(K + span - 1) / span, span};
}

}  // namespace

size_t log_probs_workspace(int N, int K, int top)
{
    const Split s = split_rows(N, K);
    if (s.parts == 1) return 0;
    return round_up((size_t)N * s.parts * (3 * sizeof(float) + top * sizeof(Key)) + sizeof(Key), 256);
}

template <typename T, bool TOP>
static int log_probs_of(const T *z, const ScoreArgs &a, hipStream_t s)
{
    const unsigned units = (unsigned)a.N * a.parts;
    if (a.K <= kOneWave) hipLaunchKernelGGL((log_probs_kernel<T, 1, TOP>), dim3((units + 3) / 4), dim3(256), 0, s, z, a);
    else hipLaunchKernelGGL((log_probs_kernel<T, 4, TOP>), dim3(units), dim3(256), 0, s, z, a);
    if (a.parts > 1) hipLaunchKernelGGL((log_probs_join_kernel<T, TOP>), dim3(a.N), dim3(64), 0, s, z, a);
    return launch_status();
}

int log_probs(int dtype, int N, int K, size_t ldz, const void *z, const int32_t *labels, int top, float *logp, float *entropy,
              float *top_logp, int32_t *top_idx, float *stats, void *ws, hipStream_t s)
{
    const Split c = split_rows(N, K);
    ScoreArgs a = {N, K, top, c.parts, c.span, ldz, labels, logp, entropy, top_logp, stats, top_idx, nullptr, nullptr};
    if (c.parts > 1) {
        const size_t n = (size_t)N * c.parts;
        a.part_sums = static_cast<float *>(ws);
        a.part_best = static_cast<Key *>(ws);
        a.part_sums = reinterpret_cast<float *>(a.part_best + n * top);
    }
    if (dtype == VGG_BF16) {
        const bf16_t *zb = static_cast<const bf16_t *>(z);
        return top ? log_probs_of<bf16_t, true>(zb, a, s) : log_probs_of<bf16_t, false>(zb, a, s);
    }
    const float *zf = static_cast<const float *>(z);
    return top ? log_probs_of<float, true>(zf, a, s) : log_probs_of<float, false>(zf, a, s);
}

template <typename T>
static int log_probs_bwd_of(const T *z, T *dz, const GradArgs &a, hipStream_t s)
{
    const unsigned units = (unsigned)a.N * a.parts;
    if (a.K <= 512) hipLaunchKernelGGL((log_probs_bwd_kernel<T, 1>), dim3((units + 3) / 4), dim3(256), 0, s, z, dz, a);
    else hipLaunchKernelGGL((log_probs_bwd_kernel<T, 4>), dim3(units), dim3(256), 0, s, z, dz, a);
    return launch_status();
}

int log_probs_bwd(int dtype, int N, int K, size_t ldz, const void *z, const int32_t *labels, const float *stats, const float *entropy,
                  const float *g_logp, const float *g_entropy, void *dz, size_t lddz, hipStream_t s)
{
    const Split c = split_rows(N, K);
    const GradArgs a = {N, K, c.span, c.parts, ldz, lddz, labels, stats, entropy, g_logp, g_entropy};
    if (dtype == VGG_BF16) return log_probs_bwd_of(static_cast<const bf16_t *>(z), static_cast<bf16_t *>(dz), a, s);
    return log_probs_bwd_of(static_cast<const float *>(z), static_cast<float *>(dz), a, s);
}

}  // namespace vgg
