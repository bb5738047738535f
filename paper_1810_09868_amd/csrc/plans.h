// Which variants of the 4-bit product's and the updates' kernels a call takes: rules on its sizes, kept apart from the kernels so that the
// host can look at them by itself.
#pragma once
#include <stddef.h>

#include "../../include/vgg_mi355x.h"

namespace vgg {

// ------------------------------------------------------------------------------------------ products with 4-bit weights
constexpr int kW4FewRows = 1;    // rows of a up to which the first kernel runs

// ... and the second: its workgroups of 16 outputs read all of a each, in pieces scattered over its rows, so that long rows are
// worth laying out first (25088 inputs, bf16: 5 rows 18.2 against 20.7 us, 10 rows 23.5 against 20.8; 4096 inputs, fp32, 16 rows:
// 11.5 against 11.7).
constexpr int kW4TileRows = 16;
constexpr size_t kW4TileBytes = 300000;

inline bool w4_one_tile(int dtype, int N, int In) { return N <= kW4TileRows && (size_t)N * In * (dtype == VGG_BF16 ? 2 : 4) <= kW4TileBytes; }

// Tiles of 64 outputs read the laid out activations least often, those of 16 begin and end soonest and need the fewest splits.  16
// where all workgroups run at once, 32 else, as long as the activations' way out of L2 is no more than this many bytes in all (32
// x 4096 x 4096, bf16: 8.3, 10.8, 12.1 us with 16, 32, 64; 100 x 4096 x 4096: 18.4, 14.6, 18.3; 64 x 25088 x 4096: 41.7, 32.7, 29.5).
constexpr size_t kW4ReadAgain = 160u << 20;

struct W4Plan { int nt, rt, tiles, splits, row_tiles; size_t lay_bytes; };
inline W4Plan w4_tiles_plan(int dtype, int N, int In, int Out)
{
    W4Plan t;
    t.nt = N <= 16 ? 1 : N <= 32 ? 2 : 4;
    t.tiles = (N + 16 * t.nt - 1) / (16 * t.nt) * t.nt;
    const int kb = (In + 127) / 128, most = (kb + 7) / 8;
    t.lay_bytes = (size_t)kb * t.tiles * 4 * (dtype == VGG_BF16 ? 1 : 3) * 1024;
    auto row_tiles = [&](int rt) { return (Out + 16 * rt - 1) / (16 * rt); };
    auto few = [&](int rt) { return t.lay_bytes * row_tiles(rt) <= kW4ReadAgain; };
    t.rt = few(1) && (long)row_tiles(1) * (t.tiles / t.nt) <= 256 ? 1 : few(2) ? 2 : 4;
    t.row_tiles = row_tiles(t.rt);
    const long units = (long)t.row_tiles * (t.tiles / t.nt);
    t.splits = (int)(units >= 256 ? 1 : (256 + units - 1) / units);
    if (t.splits > most) t.splits = most;
    return t;
}

// ------------------------------------------------------------------------------------------------ losses over many classes
// Whether fp32 products are short enough for 32 x 32 tiles of the fp32 matrix unit, in half the launches: their number, and each contraction, which a
// tile's waves go along while others wait (loss and gradients in us, so and by large tiles: 64 x 64 x 64 32, 44; 100 x 1024 x 1000 59, 72; 500 x 500 x 500
// 71, 88; 2000 x 256 x 300 92, 78; 1000 x 300 x 1000 122, 80; 4000 x 64 x 1000 145, 95; 1 x 1024 x 2000 52, 62; 1 x 4096 x 1000 104, 76).
constexpr long kXentSmall = 9l << 24;
inline bool xent_is_small(int dtype, int N, int In, int K)
{
    const long n = (N + 31) / 32 * 32, k = (K + 31) / 32 * 32;
    return dtype == VGG_F32 && N <= 4096 && In <= 1024 && K <= 2048 && n * k * In <= kXentSmall;
}

// Other products: tiles of 256 rows (classes for the scores, inputs for da and dw) and 64, 128 or 256 columns.
constexpr int kTA = 256;      // rows of C in a tile
constexpr int kParts = 2048;  // workgroups that seek an fp32 operand's largest exponent, at the most
constexpr int kStep = 64;     // contractions are whole multiples of this many indices
constexpr size_t kPieceBytes = 512u << 20;   // what dz and laid out weights of a piece of the classes may take of the workspace,
constexpr long kPieceClasses = 1 << 20;      // and how many there are (a tile's 256 rows of dz by offsets of 31 bits)
// bf16 rows up to which what rounding leaves of dz enters dw, as a contraction twice as long.  Off by 2^-9 of each term, dw is as exact as its own
// rounding to bf16 on the average of many rows; the fewer there are, the more hangs on single ones.
constexpr int kRestRows = 512;
// fp32 rows up to which, and classes from which on, scores are formed from weights where they are, by the loss and by its gradients alike: m and log_s of one product with
// the scores of another would give a nearly certain label the difference of the two (loss in us, so and with weights laid out: 1 x 4096 x 131072 498, 1842; 64 x 4096 x 131072 909, 1890; 4 x 1024 x 10007 65, 49; with four times 32 rows to a wave 100 x 4096 x 25000 949, 357).
constexpr int kDirectRows = 64, kDirectClasses = 1 << 14;
constexpr int kOuterRows = 16;               // rows up to which dw is written by its own kernel

inline int up(long v, int to) { return (int)((v + to - 1) / to * to); }
inline long div_up(long a, long b) { return (a + b - 1) / b; }

// Columns of a tile, of examples for the scores and da, of classes for dw: as many as leave no half of it empty, and give every compute unit a tile
// of its own where that can be.  Scores in one go: half of the compute units, since tiles of half the width in two rounds read w twice (bf16 128 x 2048 x
// 40000 34 us for 49; of less than half, narrower ones are faster: 1000 x 1024 x 5000 22 us in 128 columns, 31 in 256, 28 in 64).
inline int tile_of(int cols, long row_tiles, int least = 256)
{
    int tn = cols > 128 ? 256 : cols > 64 ? 128 : 64;
    while (tn > 64 && row_tiles * div_up(cols, tn) < least) tn /= 2;
    return tn;
}
// Whether the contraction of few tiles of scores is split.  All of them have to be kept for a moment then, and read again, which takes the longer the more
// classes and rows there are, while a contraction in one goes on for 0.6 us (fp32 1.1) a stage.  (Loss and gradients in us, split and not: bf16 100 x 4096 x
// 1000 63, 98; 1000 x 4096 x 4000 229, 262; 100 x 4096 x 8192 130, 155; 100 x 4096 x 12000 194, 175; 1000 x 1024 x 1000 98, 73; 100 x 1024 x 1000 53, 54; fp32 100 x
// 4096 x 1000 95, 192; 100 x 4096 x 16000 734, 767; 100 x 4096 x 25000 1100, 1067; 100 x 1024 x 2500 90, 103; 1000 x 1024 x 2500 244, 207.)
inline bool scores_are_split(int dtype, int N, int K, int steps)
{
    const long work = dtype == VGG_BF16 ? steps : 2l * steps;
    return work >= 16 && work >= K / 144 + N / 64;
}
// Ranges of a contraction of `steps` stages, where `tiles` do not fill the chip: at least 256 indices of bf16 operands each, or 128 of
// fp32 ones, which take three times as long.
inline int splits_of(int dtype, long tiles, int steps)
{
    const long most = div_up(steps, dtype == VGG_BF16 ? 4 : 2), want = tiles >= 256 ? 1 : div_up(256, tiles);
    return (int)(want < most ? want : most);
}

struct XentPlan {
    int PL, In, InP, NP, tn, grad_tn;
    bool direct_w, direct_a;      // read where they are (bf16, whole stages)
    bool few_rows;                // scores by the fp32 matrix unit, from operands where they are
    int classes, pieces;          // of a piece (the last has what is left)
    int z_splits;                 // 0: scores' tiles end in their sums or gradients; else their parts are added up (then one piece)
    int ld_dz, rest_rows;
    size_t ld_z;
    // forward
    size_t a_at, w_at, ea_at, most_at, z_at, sums_at, label_at, forward_bytes;
    // backward
    int da_splits, da_tn, dw_splits, dw_tn, db_parts;
    size_t a2_at, eg_at, rest_at, tail_at, dz_at, da_at, dw_at, db_at, backward_bytes;
};

inline XentPlan xent_plan(int dtype, int N, int In, int K)
{
    XentPlan p;
    p.PL = dtype == VGG_BF16 ? 1 : 2;
    p.In = In; p.InP = up(In, kStep); p.NP = up(N, kStep);
    const int steps = p.InP / kStep;
    const long k_tiles = div_up(K, kTA);
    // (where the contraction of scores is split: their columns by what that leaves idle)
    p.tn = tile_of(N, k_tiles * splits_of(dtype, k_tiles, steps));
    p.z_splits = scores_are_split(dtype, N, K, steps) && k_tiles * div_up(N, p.tn) < 128 ? splits_of(dtype, k_tiles * div_up(N, p.tn), steps) : 0;
    if (p.z_splits <= 1) {
        p.z_splits = 0;
        p.tn = tile_of(N, k_tiles, 128);
    }
    p.grad_tn = p.PL == 2 && p.tn == 256 ? 128 : p.tn;     // (256: more registers than there are)
    p.direct_w = p.direct_a = dtype == VGG_BF16 && In % kStep == 0;
    p.few_rows = dtype == VGG_F32 && !p.z_splits && N <= kDirectRows && K >= kDirectClasses;
    const long n_tiles = div_up(N, p.tn), d_tiles = div_up(In, kTA);
    p.rest_rows = p.PL == 1 && N <= kRestRows ? p.NP : 0;
    const size_t per_class = (size_t)p.PL * 2 * (p.NP + p.rest_rows + (p.direct_w ? 0 : p.InP));
    long classes = (long)(kPieceBytes / per_class) / kTA * kTA;
    if (classes < kTA) classes = kTA;
    if (classes > kPieceClasses) classes = kPieceClasses;
    if (p.z_splits || classes > K) classes = up(K, kTA);      // (z_splits: one piece)
    // as large as they may be, and of the 64 largest sizes the one whose tiles leave least of the chip idle in their last rounds
    const long all = div_up(K, kTA), largest = classes / kTA < all ? classes / kTA : all;
    auto rounds = [&](long tiles) { return div_up(tiles * n_tiles, 256); };
    long best = 0, best_rounds = 0;
    for (long t = largest; t > 0 && t > largest - (p.z_splits ? 1 : 64); --t) {
        const long r = all / t * rounds(t) + (all % t ? rounds(all % t) : 0);
        if (!best || r < best_rounds) { best = t; best_rounds = r; }
    }
    p.classes = (int)(best * kTA);
    p.pieces = (int)div_up(K, p.classes);
    const int most = p.classes < K ? p.classes : K;
    p.ld_dz = up(most, kStep);
    p.ld_z = up(K, 4);
    size_t at = 0;
    auto take = [&](size_t bytes) { const size_t here = at; at += (bytes + 255) / 256 * 256; return here; };
    // (the gradients take the activations laid out in any case: rows without a label have to be zeros)
    p.a_at = take((size_t)p.PL * 2 * p.NP * p.InP);
    p.w_at = take(p.direct_w ? 0 : (size_t)p.PL * 2 * up(most, kStep) * p.InP);
    p.ea_at = take(p.PL == 2 ? (size_t)N * 4 : 0);
    p.most_at = take(p.PL == 2 ? (size_t)(2 + 2 * kParts) * 4 : 0);
    p.z_at = take(p.z_splits ? (size_t)p.z_splits * N * p.ld_z * 4 : 0);
    const size_t both = at;
    p.sums_at = take(p.z_splits ? 0 : (size_t)div_up(K, kTA) * N * 8);
    p.label_at = take(p.z_splits ? 0 : (size_t)N * 4);
    p.forward_bytes = at;
    at = both;
    p.a2_at = take(p.PL == 2 ? (size_t)4 * p.NP * p.InP : 0);
    p.eg_at = take(p.PL == 2 ? (size_t)N * 4 : 0);
    p.tail_at = take(p.direct_w ? (size_t)kStep * In * 2 : 0);
    p.rest_at = take(p.PL == 1 ? (size_t)N * 4 : 0);
    p.dz_at = take((size_t)p.PL * 2 * (p.NP + p.rest_rows) * p.ld_dz);
    p.da_tn = tile_of(N, d_tiles * splits_of(dtype, d_tiles, (int)div_up(most, kStep)));
    p.da_splits = splits_of(dtype, div_up(N, p.da_tn) * d_tiles, (int)div_up(most, kStep));
    p.da_at = take((size_t)p.da_splits * N * p.InP * 4);
    p.dw_tn = tile_of(most, d_tiles);
    p.dw_splits = splits_of(dtype, d_tiles * div_up(most, p.dw_tn), (p.NP + p.rest_rows) / kStep);
    p.dw_at = take(p.dw_splits == 1 || N <= kOuterRows ? 0 : (size_t)p.dw_splits * most * p.InP * 4);
    // rows' ranges that db is summed in
    p.db_parts = (int)(p.z_splits ? div_up(N, N < 256 ? 4 : div_up(N, 64)) : div_up(N, p.grad_tn));
    p.db_at = take(p.db_parts == 1 ? 0 : (size_t)p.db_parts * p.ld_dz * 4);
    p.backward_bytes = at;
    return p;
}

// ------------------------------------------------------------------------------------------------ orthogonalised updates
inline int round_to(int v, int to) { return (v + to - 1) / to * to; }

// Matrices of few rows (of X): the bytes of 64 elements in LDS (16 more: rows start in different banks), and what a workgroup with
// `blocks` of 32 columns has there.
constexpr int kFewRows = 64, kLds = 160 * 1024;
constexpr int row_stride(int planes) { return 128 * planes + 16; }
inline size_t few_lds(int planes, int blocks) { return (size_t)(blocks * 32 + 2 * kFewRows) * row_stride(planes) + 3 * 256; }
// Column blocks of a wave in one workgroup, 0 where a matrix is too large: its planes' room in LDS (448 columns of two), and at most 640
// columns of one plane (updates of 64 x 576: 48.4 us, and 51.1 in three workgroups and seven launches; 64 x 640: 50.0, 51.2; 64 x 768: 53.9,
// 51.5).
inline int small_blocks(int planes, int rows, int cols)
{
    const int m = rows < cols ? rows : cols, n = rows < cols ? cols : rows, blocks = (n + 31) / 32, cb = (blocks + 7) / 8;
    return m <= kFewRows && blocks <= 20 && few_lds(planes, blocks) <= kLds ? cb : 0;
}
// With more columns: 256 columns to a workgroup while that makes at most 16, whose shares each of them adds up, else as many as LDS has
// room for, up to 512.
struct FewPlan { int cb, each, wgs; };
inline FewPlan few_plan(int planes, int rows, int cols)
{
    const int blocks = ((rows < cols ? cols : rows) + 31) / 32;
    FewPlan w;
    w.cb = blocks <= 16 * 8 ? 1 : 2;
    w.each = w.cb * 8;
    while (few_lds(planes, w.each) > kLds) --w.each;
    w.wgs = (blocks + w.each - 1) / w.each;
    return w;
}
// ... as long as a matrix's workgroups run at once: they all add up all shares, so that what is read grows with their square, and products
// by tiles are faster then (fp32 update of 64 x 98304: 280 us, 384 by tiles; 64 x 131072, 293 workgroups: 622, 498; 64 x 1000000: 14.6 ms,
// 3.4 ms).
inline bool is_wide(int planes, int rows, int cols)
{
    return (rows <= kFewRows || cols <= kFewRows) && few_plan(planes, rows, cols).wgs <= 256;
}

// Tiles of an update's products, X of m x n, m <= n: 256 x 256 where the product with X takes no more of the chip's rounds with them (a
// tile is four times the work of a 128 x 128 one, in about 3.4 times its time), and the contraction over m is long beside what a tile begins and ends with
// (fp32 updates: 7 x 512 x 4608: 831 us with them, 775 us without; 1024 x 4096: 605, 375; 4096 x 4096: 3.94 ms, 4.40 ms; 1088 x 10944, where
// they are taken: 1.03 ms, 0.99 ms).
inline int muon_tile(long batch, int m, int n)
{
    auto rounds = [&](int t) { return (batch * (round_to(m, t) / t) * (round_to(n, t) / t) + 255) / 256; };
    return m >= 1024 && 3.4 * rounds(256) <= rounds(128) ? 256 : 128;
}

}  // namespace vgg
