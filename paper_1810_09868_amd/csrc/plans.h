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
// tile's waves go along while others wait (loss and gradients in us, so and by large tiles: 64 x 64 x 64 33, 50; 100 x 1024 x 1000 61, 95; 500 x 500 x 500 73,
// 133; 1000 x 300 x 1000 124, 138; 2000 x 256 x 2000 232, 160; 100 x 100 x 4000 99, 92; 1 x 4096 x 1000 107, 83).
constexpr long kXentSmall = 5l << 26;
inline bool xent_is_small(int dtype, int N, int In, int K)
{
    const long n = (N + 31) / 32 * 32, k = (K + 31) / 32 * 32;
    return dtype == VGG_F32 && N <= 4096 && In <= 1024 && K <= 2048 && n * k * In <= kXentSmall;
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
