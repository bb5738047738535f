// A dense layer over many classes and its softmax cross entropy, without the scores [N][K] in memory (but where there are few and their contraction is split).
//
// z = a w^T + b.  Forward: every tile of scores leaves its rows' largest score m and E, the sum of the exponentials of the others above it;
// joined over a row's tiles, loss = log(1 + E) - (z_label - m).  Backward, for a piece of the classes at a time: the same scores again, bit for bit, from them
// dz = g (softmax - 1[label]), and with it da += dz w, dw = dz^T a, db = sum_n dz.  E is kept without the largest's own 1, and the label's
// dz is g expm1(log p), so that a label that is all but certain keeps its digits.
//
// The three products are one kernel: C[col][row] = sum_k A[row][k] B[col][k], where an operand lies by its rows or by the contraction
// index (which is then read transposed out of LDS).  bf16 operands are multiplied as they are, fp32 ones in two f16 parts, 22 bits: their
// products without those of two second parts are off by 2^-22, and are three where three bf16 parts need six.  f16 has few exponents, so
// operands are laid out in units of powers of two, in which the largest is between 2^14 and 2^15; what is 2^17 times smaller has 22 bits still, and
// below that 2^-39 of the largest is left out.  Activations have units of their own in every row, weights one in all of a piece, W:
//     a = a' 2^(ea[n] - 14),  w = w' 2^(W - 14),  z = sum_i a' w' 2^(ea[n] + W - 28).
// A contraction needs units that do not depend on its index.  With 2^eg[n] <= |g_loss[n]| < 2 2^eg[n] and A = max (ea + eg),
//     D = dz 2^(14 - eg[n]),      da = sum_k D w' 2^(eg[n] + W - 28),
//     a" = a 2^(eg[n] - A + 14),  dw = sum_n D a" 2^(A - 28):
// a row's da has its digits however small its weight in the loss, and dw loses those of rows that add next to nothing to it.  (With weights in
// units of their rows, D would have to make up for them: a class of small weights would lose its dw.)
#include "common.h"
#include "dropout.h"
#include "exp_of.h"
#include "plans.h"
#include "wave.h"
#include "xent.h"

#include <limits.h>

#include <type_traits>

namespace vgg {

namespace {

constexpr int kTileStride = 528;             // bytes from row to row of 256 bf16 numbers in LDS

enum { kStore, kStats, kGrad };

struct Operand {
    const char *p;
    size_t ld;            // bytes from row to row
    int rows;             // by rows: of these; by the contraction index: bytes of a row that are there (a multiple of 16)
    const char *tail;     // by the contraction index: where the last stage's 64 rows lie, if not with the others
};

struct Sums { float m, e; };   // largest score, and the exponentials of the others above it; of none: -inf, 0
__device__ __forceinline__ Sums joined(Sums a, Sums b)
{
    if (b.m > a.m) { const Sums c = a; a = b; b = c; }
    const float d = a.m == b.m ? 0.f : below(b.m - a.m), one = b.m > -INFINITY ? 1.f : 0.f;
    return {a.m, a.e + exp_of(d) * (b.e + one)};
}

struct Product {
    Operand a, b;
    int rows, cols, steps, splits;   // of C; the contraction's indices in whole 64s; ranges of them
    // fp32: C's units, 2^(ea[col] + *most - 28), each where it is given
    const int *ea, *most;
    // kStore: C[col][row], a row of C^T every ld elements, fp32 or bf16; a range's every `part` elements, added to what is there if asked
    void *out;
    size_t ld, part;
    int bf16, add;
    // kStats, kGrad: classes are rows of C, examples its columns
    const float *bias;
    const int32_t *labels;
    int class0, classes, all_classes;   // of this piece: the first, how many; of all
    Sums *sums;                          // kStats: [tiles of classes, of all pieces][N]
    float *z_label;                      // [N]
    const float *stats, *g;              // kGrad: [N][2], [N]
    const int *eg;                       // fp32
    bf16_t *dz;                          // [N ...][ld_dz], parts side by side
    int ld_dz;                           // classes of a row
    int rest_rows;                       // bf16: what rounding leaves of dz lies so many rows on; 0: it is not kept
    float *rest_of_label;                // bf16: [N], ... of dz at the labels
    int wrap;                            // contraction indices, in whole 64s, after which A begins again; 0: never
    float *db;                           // [tiles of examples][ld_db]
    size_t ld_db;
};

typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x4 __attribute__((ext_vector_type(4)));
typedef unsigned short u16x4 __attribute__((ext_vector_type(4)));

// Where column c of a row in PL parts lies, in 16-bit numbers: parts of 32 columns side by side.
template <int PL> __host__ __device__ __forceinline__ size_t column_at(int c, int part) { return PL == 1 ? c : (size_t)(c >> 5) * 64 + part * 32 + (c & 31); }
// Four numbers in the unit 2^-e, in two f16 parts; of what is not finite the first says it all.
__device__ __forceinline__ void two_parts(const f32x4 &v, int e, f16x4 (&part)[2])
{
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        const float x = ldexpf(v[k], e);
        part[0][k] = (_Float16)x;
        const float rest = x - (float)part[0][k];
        part[1][k] = (_Float16)(__builtin_fabsf(rest) < INFINITY ? rest : 0.f);
    }
}
// What rounding to bf16 leaves (of infinities and NaN: nothing).
__device__ __forceinline__ float rest_of(float v)
{
    const float r = v - bf16_to_f32(f32_to_bf16(v));
    return __builtin_fabsf(r) < INFINITY ? r : 0.f;
}
// e with 2^e <= |v| < 2 2^e; 0 for zeros and what is not finite.
__device__ __forceinline__ int exponent_of(float v) { return v != 0.f && __builtin_fabsf(v) < INFINITY ? ilogbf(v) : 0; }

typedef __attribute__((address_space(3))) char lds_char;

// Workgroups go round the eight XCDs; each takes a run of the work, so that neighbours share their operands in its L2.
__device__ __forceinline__ int spread(int id, int count)
{
    const int per = count >> 3, more = count & 7, xcd = id & 7, at = id >> 3;
    return xcd * per + (xcd < more ? xcd : more) + at;
}

__device__ __forceinline__ bf16x8 read_transposed(const char *at)
{
    typedef short s16x4 __attribute__((ext_vector_type(4)));
    typedef __attribute__((address_space(3))) s16x4 *lp;
    const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lp)at);
    const s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lp)(at + 4 * 128));
    return __builtin_bit_cast(bf16x8, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
}

__device__ __forceinline__ void wave_sync()
{
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
    __builtin_amdgcn_wave_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
}

// A stage is 128 bytes of a row: 64 contraction indices of bf16 operands, or both parts of 32 of fp32 ones, which lie side by side.
__host__ __device__ constexpr int stage_lds(int tn) { return (kTA + tn) * 128; }
__host__ __device__ constexpr int stages_of(int tn) { return tn == 256 ? 2 : 3; }
// LDS of a tile: its stages, or what its end turns round in it
struct Example { float m, log_s, g; int label, ea, eg; };   // what the end of a tile knows of a column
__host__ __device__ constexpr int main_lds_of(int tn, int mode, int stages)
{
    const int run = (stages < stages_of(tn) ? stages : stages_of(tn)) * stage_lds(tn), stored = 8 * 32 * (tn == 64 ? 144 : tn == 128 ? 272 : 528);
    const int end = mode == kStore ? stored : mode == kGrad ? tn * kTileStride : 8 * tn * (int)sizeof(Sums);
    return run > end ? run : end;
}
// ... and behind that the tile's biases and examples
__host__ __device__ constexpr int lds_of(int tn, int mode, int stages) { return main_lds_of(tn, mode, stages) + (mode == kStore ? 0 : kTA * 4 + tn * (int)sizeof(Example)); }

// A tile of 256 rows by TN columns of C: eight waves of 32 x 32 blocks, stages copied straight into LDS, two or three of them, the next under way while one is
// multiplied.  Columns are 256 where they fill the chip, since each operand of a stage is then met 256 times; few examples take as few columns as hold
// them.  The matrix unit bounds large ones, at the power it draws: of 8192 x 2048 x 131072 bf16 a fourth of the classes takes 936 us with the scores' sums, 1003
// with dz, 852 for da and 863 for dw (1.10 to 1.29 PFLOP/s); 1000 x 1001 x 50001 fp32 333, 371 (in 128 columns: 256 have no registers for their end), 263 and 343
// (0.81 to 1.14 PFLOP/s of f16).  The read of w bounds few rows: 4 x 4096 x 200003 bf16 380 us with the sums, 345 with dz, 260 for da (4.3, 4.8 and 6.3 TB/s).
template <bool A_TR, bool B_TR, int TN, int PL, int MODE>
__global__ __launch_bounds__(512) void xent_product_kernel(Product p)
{
    extern __shared__ __align__(16) char lds[];   // [STAGES][A, B]
    // eight waves, WA x WB of them, BX x BY blocks of 32 x 32 each
    constexpr int KS = kStep / PL, STAGES = stages_of(TN), WB = TN == 256 ? 4 : TN == 128 ? 2 : 1, WA = 8 / WB, BX = kTA / 32 / WA, BY = TN / 32 / WB;
    constexpr int HALF = kTA * 128, STAGE = stage_lds(TN), CA = kTA / 64, CB = TN / 64, COPIES = CA + CB;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int mt = (p.rows + kTA - 1) / kTA, nt = (p.cols + TN - 1) / TN;
    const int unit = spread(blockIdx.x, gridDim.x), split = unit / (mt * nt), in_all = unit - split * (mt * nt);
    // eight tiles down, then one to the right
    const int wide = 8 * nt, group = in_all / wide, in = in_all - group * wide, down = mt - group * 8 < 8 ? mt - group * 8 : 8;
    const int ti = group * 8 + in % down, tj = in / down;
    const int s0 = (int)((long)p.steps * split / p.splits), total = ((int)((long)p.steps * (split + 1) / p.splits) - s0) * PL;

    // Where this thread's copies come from, within a stage; rows and columns that are not there are others that are (what they give is not
    // used).  By rows: [rows][128 bytes], the 16-byte segments of a row in an order that puts sixteen rows of one segment in different banks.  By the
    // contraction index: [128 bytes of columns][KS][128 bytes], the halves of every other pair of rows exchanged.
    unsigned from_a[CA], from_b[CB];
    auto source = [&](const Operand &o, bool tr, int tile0, int q) __attribute__((always_inline)) {
        const int at = (q * 512 + (int)threadIdx.x) * 16;
        if (!tr) {
            const int r = at >> 7, seg = ((at >> 4) & 7) ^ (r >> 1 & 7);
            return (unsigned)((tile0 + r < o.rows ? r : o.rows - 1 - tile0) * (long)o.ld) + seg * 16;
        }
        const int k = (at >> 7) % KS, col = tile0 * 2 * PL + at / (KS * 128) * 128 + ((at & 127) ^ (k >> 1 & 1) << 6);
        return (unsigned)(k * (long)o.ld) + (col < o.rows ? col : o.rows - 16);
    };
#pragma unroll
    for (int q = 0; q < CA; ++q) from_a[q] = source(p.a, A_TR, ti * kTA, q);
#pragma unroll
    for (int q = 0; q < CB; ++q) from_b[q] = source(p.b, B_TR, tj * TN, q);
    const size_t step_a = A_TR ? KS * p.a.ld : 128, step_b = B_TR ? KS * p.b.ld : 128;
    const char *at_a = p.a.p + (A_TR ? 0 : (size_t)ti * kTA * p.a.ld) + (size_t)(A_TR && PL == 1 && p.wrap ? s0 % p.wrap : s0) * PL * step_a;
    const char *at_b = p.b.p + (B_TR ? 0 : (size_t)tj * TN * p.b.ld) + (size_t)s0 * PL * step_b;
    const unsigned lds0 = __builtin_amdgcn_readfirstlane((unsigned)(uintptr_t)(lds_char *)lds + wave * 1024);
    // the stage that is copied next
    int slot = 0, to_come = p.steps - s0;
    auto aim = [&]() __attribute__((always_inline)) {
        if (A_TR && PL == 1 && p.a.tail && to_come == 1) at_a = p.a.tail;
        if (A_TR && PL == 1 && p.wrap && to_come == p.steps - p.wrap) at_a = p.a.p;
    };
    aim();
    auto copy_one = [&](int n) __attribute__((always_inline)) {      // of a stage's COPIES
        const bool is_a = n < CA;
        const unsigned to = lds0 + slot * STAGE + n * 8192, off = is_a ? from_a[is_a ? n : 0] : from_b[is_a ? 0 : n - CA];
        const char *base = is_a ? at_a : at_b;
        asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2" : : "s"(to), "v"(off), "s"(base) : "m0", "memory");
        if (n == COPIES - 1) {
            slot = slot + 1 == STAGES ? 0 : slot + 1;
            at_a += step_a;
            at_b += step_b;
            --to_come;
            aim();
        }
    };

    // What the tile's end needs of its classes and examples: asked for now, put into LDS then.
    float own_bias = -INFINITY;
    float own_m = 0.f, own_log_s = 0.f, own_g = 0.f;
    int own_label = -1, own_ea = 0, own_eg = 0;
    if constexpr (MODE != kStore) {
        const int row = ti * kTA + (int)threadIdx.x, col = tj * TN + (int)threadIdx.x;
        if (threadIdx.x < kTA && row < p.classes) own_bias = p.bias ? p.bias[p.class0 + row] : 0.f;
        if (threadIdx.x < TN && col < p.cols) {
            const int label = p.labels[col];
            own_label = (int)((unsigned)label - p.class0);
            if constexpr (PL == 2) own_ea = p.ea[col] + *p.most - 28;
            if constexpr (MODE == kGrad) {
                own_m = p.stats[2 * (size_t)col];
                own_log_s = p.stats[2 * (size_t)col + 1];
                own_g = label >= 0 && label < p.all_classes ? p.g[col] : 0.f;
                if constexpr (PL == 2) own_eg = p.eg[col];
            }
        }
    }
    f32x16 acc[BX][BY] = {};
    const int wi = wave / WB * (BX * 32), wj = wave % WB * (BY * 32);
    const int rx = lane >> 1 & 7;
    const int s16 = lane & 15, tr_k = 8 * (lane >> 5) + (s16 >> 2), tr_x = s16 >> 3, tr_at = (lane >> 4 & 1) * 32 + (s16 & 3) * 8;
    // A stage is KK steps of 16 contraction indices.  Between a step's products the next step's fragments are read, and in a stage's last
    // step, after the barrier, the next stage's first fragments and the copies of a stage to come.
    constexpr int KK = 4 / PL, M = (PL == 2 ? 3 : 1) * BX * BY, R = PL * (BX + BY);
    struct Fragments { bf16x8 a[PL][BX], b[PL][BY]; };
    auto read_one = [&](int use, int k, int n, Fragments &f) __attribute__((always_inline)) {
        const int part = n / (BX + BY), m = n % (BX + BY);
        const bool is_a = m < BX;
        const int q = is_a ? m : m - BX, w0 = is_a ? wi : wj;
        const char *from = lds + use * STAGE + (is_a ? 0 : HALF);
        bf16x8 v;
        if (is_a ? A_TR : B_TR) {
            const int c = ((w0 >> 5) + q) * PL + part;                 // 64-byte block of a row
            v = read_transposed(from + (c >> 1) * (KS * 128) + (k * 16 + tr_k) * 128 + (((c & 1) ^ tr_x) << 6) + tr_at);
        } else
            v = *reinterpret_cast<const bf16x8 *>(from + (w0 + (lane & 31) + q * 32) * 128 + (((part * 4 + k * 2 + (lane >> 5)) ^ rx) << 4));
        if (is_a) f.a[part][is_a ? q : 0] = v;
        else f.b[part][is_a ? 0 : q] = v;
    };
    Fragments f[2];
    int use = 0;
    // One stage; READ: there is a next one, COPY: there is one to be copied.
    auto stage = [&](auto READ, auto COPY) __attribute__((always_inline)) {
        constexpr bool reads = decltype(READ)::value, copies = decltype(COPY)::value;
#pragma unroll
        for (int k = 0; k < KK; ++k) {
            const bool last = k + 1 == KK;
            const int lead = last ? M / 3 : 0, tasks = last ? (reads ? R : 0) + (copies ? COPIES : 0) : R;
            const Fragments &g = f[k & 1];
            Fragments &next = f[(k + 1) & 1];
#pragma unroll
            for (int i = 0; i < M; ++i) {
                // (fp32: the small terms first; a sum's next product waits for its last, so the blocks take turns)
                const int term = PL == 2 ? i / (BX * BY) : 2, x = i % (BX * BY) / BY, y = i % BY;
                if (last && reads && i == lead) {
                    // The next stage's copies have landed (those of later ones may be on their way), and all waves have read what they need
                    // of this one, whose place the next copies take.
                    asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" : : "n"(copies ? (STAGES - 2) * COPIES : 0) : "memory");
                    use = use + 1 == STAGES ? 0 : use + 1;
                }
                const bf16x8 ga = g.a[term == 0 ? PL - 1 : 0][x], gb = g.b[term == 1 ? PL - 1 : 0][y];
                if constexpr (PL == 2) acc[x][y] = __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(f16x8, ga), __builtin_bit_cast(f16x8, gb), acc[x][y], 0, 0, 0);
                else acc[x][y] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(ga, gb, acc[x][y], 0, 0, 0);
                if (i >= lead)
#pragma unroll
                    for (int n = (i - lead) * tasks / (M - lead); n < (i - lead + 1) * tasks / (M - lead); ++n) {
                        if (!last) read_one(use, k + 1, n, next);
                        else if (reads && n < R) read_one(use, 0, n, next);
                        else copy_one(reads ? n - R : n);
                    }
                __builtin_amdgcn_sched_barrier(0);
            }
        }
    };
#pragma unroll
    for (int k = 0; k < STAGES; ++k)
        if (k < total)
#pragma unroll
            for (int n = 0; n < COPIES; ++n) copy_one(n);
    if (total >= STAGES) asm volatile("s_waitcnt vmcnt(%0)\n\ts_barrier" : : "n"((STAGES - 1) * COPIES) : "memory");
    else asm volatile("s_waitcnt vmcnt(0)\n\ts_barrier" : : : "memory");
#pragma unroll
    for (int n = 0; n < R; ++n) read_one(0, 0, n, f[0]);
    int st = 0;
    for (; st + STAGES < total; ++st) stage(std::true_type{}, std::true_type{});
    for (; st + 1 < total; ++st) stage(std::true_type{}, std::false_type{});
    stage(std::false_type{}, std::false_type{});
    // Value v of a block: row 8 (v / 4) + 4 (lane / 32) + v % 4, column lane % 32.
    asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" : : : "memory");   // no wave reads operands any more
    if constexpr (MODE == kStore) {
        // A wave's 32 columns and all its rows go through a place of its own in LDS: then a lane has eight consecutive rows.
        constexpr int ROWS = BX * 32, STRIDE = ROWS * 4 + 16, LANES = ROWS / 8;
        char *turned = lds + wave * (32 * STRIDE);
        const int r8 = lane % LANES * 8, row = ti * kTA + wi + r8;
        int of_col[BY] = {};     // the exponent of column lane % 32 of a block
        if constexpr (PL == 2) {
            const int all = (p.most ? *p.most : 0) - 28;
#pragma unroll
            for (int y = 0; y < BY; ++y) {
                const int col = tj * TN + wj + y * 32 + (lane & 31);
                of_col[y] = all + (p.ea && col < p.cols ? p.ea[col] : 0);
            }
        }
#pragma unroll
        for (int y = 0; y < BY; ++y) {
#pragma unroll
            for (int x = 0; x < BX; ++x)
#pragma unroll
                for (int q = 0; q < 4; ++q)
                    *reinterpret_cast<f32x4 *>(turned + (lane & 31) * STRIDE + (x * 32 + 8 * q + 4 * (lane >> 5)) * 4) =
                        f32x4{acc[x][y][4 * q], acc[x][y][4 * q + 1], acc[x][y][4 * q + 2], acc[x][y][4 * q + 3]};
            wave_sync();
#pragma unroll 2      // (a tile of a short contraction waits for code)
            for (int i = 0; i < LANES / 2; ++i) {
                const int c = i * (64 / LANES) + lane / LANES, col = tj * TN + wj + y * 32 + c, n = p.rows - row;
                const f32x4 *here = reinterpret_cast<const f32x4 *>(turned + c * STRIDE + r8 * 4);
                f32x4 lo = here[0], hi = here[1];
                if constexpr (PL == 2) {
                    const int e = __shfl(of_col[y], c);
#pragma unroll
                    for (int k = 0; k < 4; ++k) {
                        lo[k] = ldexpf(lo[k], e);
                        hi[k] = ldexpf(hi[k], e);
                    }
                }
                if (col < p.cols && n > 0) {
                    const size_t at = (size_t)split * p.part + (size_t)col * p.ld + row;
                    float v[8];
#pragma unroll
                    for (int k = 0; k < 4; ++k) { v[k] = lo[k]; v[k + 4] = hi[k]; }
                    if (p.bf16) {
                        Eight<bf16_t> e;
                        e.set(v);
                        e.store(static_cast<bf16_t *>(p.out) + at, n);
                    } else {
                        float *to = static_cast<float *>(p.out) + at;
                        Eight<float> e, old;
                        if (p.add) {
                            old.load(to, n);
#pragma unroll
                            for (int k = 0; k < 8; ++k) v[k] += old.get(k);
                        }
                        e.set(v);
                        e.store(to, n);
                    }
                }
            }
            wave_sync();
        }
    } else {
        // scores of this lane: example tj TN + wj + 32 y + lane % 32, class row0 + 32 x + 8 (v / 4) + v % 4 of the piece
        float *bias = reinterpret_cast<float *>(lds + main_lds_of(TN, MODE, stages_of(TN)));
        Example *examples = reinterpret_cast<Example *>(bias + kTA);
        if (threadIdx.x < kTA) bias[threadIdx.x] = own_bias;
        if (threadIdx.x < TN) {
            Example &e = examples[threadIdx.x];
            e.label = own_label;
            if constexpr (PL == 2) e.ea = own_ea;
            if constexpr (MODE == kGrad) { e.m = own_m; e.log_s = own_log_s; e.g = own_g; }
            if constexpr (MODE == kGrad && PL == 2) e.eg = own_eg;
        }
        __syncthreads();
        const int row0 = wi + 4 * (lane >> 5);          // of the tile
#pragma unroll
        for (int x = 0; x < BX; ++x)
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                const f32x4 b = *reinterpret_cast<const f32x4 *>(bias + row0 + 32 * x + 8 * q);     // (-inf past the last class)
#pragma unroll
                for (int y = 0; y < BY; ++y) {
                    const int ea = PL == 2 ? examples[wj + 32 * y + (lane & 31)].ea : 0;
#pragma unroll
                    for (int k = 0; k < 4; ++k) acc[x][y][4 * q + k] = b[k] + (PL == 2 ? ldexpf(acc[x][y][4 * q + k], ea) : acc[x][y][4 * q + k]);
                }
            }
        // the score of this lane's label, if it is among the lane's
        auto score_at = [&](int y, int label) __attribute__((always_inline)) {
            float z = -INFINITY;
            const int rel = label - row0;
#pragma unroll
            for (int x = 0; x < BX; ++x)
#pragma unroll
                for (int v = 0; v < 16; ++v) z = rel == 32 * x + 8 * (v >> 2) + (v & 3) ? acc[x][y][v] : z;
            return z;
        };
        auto is_here = [&](int label) __attribute__((always_inline)) {
            const int rel = label - row0;
            return rel >= 0 && rel < 32 * BX && !(rel & 4);
        };
        if constexpr (MODE == kStats) {
            Sums *all = reinterpret_cast<Sums *>(lds);    // [WA][TN]
#pragma unroll
            for (int y = 0; y < BY; ++y) {
                if constexpr (TN == 64) if (tj * TN + 32 * y >= p.cols) continue;     // (few rows)
                const int at = wj + 32 * y + (lane & 31), label = (int)((unsigned)examples[at].label - ti * kTA);
                const bool here = is_here(label);
                if (__any(here)) {
                    const float z = score_at(y, label);
                    if (here) p.z_label[tj * TN + at] = z;       // (no label: past the last class or column)
                }
                Sums s = {-INFINITY, 0.f};
#pragma unroll
                for (int x = 0; x < BX; ++x)
#pragma unroll
                    for (int v = 0; v < 16; ++v) s.m = fmaxf(s.m, acc[x][y][v]);
                bool fresh = s.m > -INFINITY;               // one of the largest does not count
                const float base = fresh ? s.m : 0.f;
#pragma unroll
                for (int x = 0; x < BX; ++x)
#pragma unroll
                    for (int v = 0; v < 16; ++v) {
                        const float z = acc[x][y][v], e = exp_of(below(z - base));
                        const bool it = fresh && z == s.m;
                        s.e += it ? 0.f : e;
                        fresh = fresh && !it;
                    }
                s = joined(s, Sums{__shfl_xor(s.m, 32), __shfl_xor(s.e, 32)});
                if (lane < 32) all[wave / WB * TN + wj + 32 * y + lane] = s;
            }
            __syncthreads();
            if (threadIdx.x < TN) {
                Sums s = all[threadIdx.x];
#pragma unroll
                for (int w = 1; w < WA; ++w) s = joined(s, all[w * TN + threadIdx.x]);
                const int col = tj * TN + threadIdx.x;
                if (col < p.cols) p.sums[(size_t)(p.class0 / kTA + ti) * p.cols + col] = s;
            }
        } else {
            float sum[BX][16] = {};
#pragma unroll
            for (int y = 0; y < BY; ++y) {
                if constexpr (TN == 64) if (tj * TN + 32 * y >= p.cols) continue;     // (few rows)
                const Example &e = examples[wj + 32 * y + (lane & 31)];
                const int label = (int)((unsigned)e.label - ti * kTA);
                const bool here = is_here(label), none = e.g == 0.f || e.log_s == -INFINITY;     // (-inf: a row without a class)
                float fixed = 0.f;
                const bool any = __any(here);
                if (any) {
                    const float z = score_at(y, label);
                    fixed = none || z == -INFINITY ? 0.f : e.g * expm1f((z - e.m) - e.log_s);
                    if constexpr (PL == 1)
                        if (here && tj * TN + wj + 32 * y + (lane & 31) < p.cols) p.rest_of_label[tj * TN + wj + 32 * y + (lane & 31)] = rest_of(fixed);
                }
#pragma unroll
                for (int x = 0; x < BX; ++x)
#pragma unroll
                    for (int v = 0; v < 16; ++v) {
                        // (bf16: off by |d| 2^-24 of a share that is rounded to 2^-9, either way)
                        const float d = below((acc[x][y][v] - e.m) - e.log_s), share = PL == 1 ? __builtin_amdgcn_exp2f(d * 1.44269504f) : exp_of(d);
                        acc[x][y][v] = none ? 0.f : e.g * share;
                    }
                if (any) {
                    const int rel = label - row0;
#pragma unroll
                    for (int x = 0; x < BX; ++x)
#pragma unroll
                        for (int v = 0; v < 16; ++v) acc[x][y][v] = rel == 32 * x + 8 * (v >> 2) + (v & 3) ? fixed : acc[x][y][v];
                }
#pragma unroll
                for (int x = 0; x < BX; ++x)
#pragma unroll
                    for (int v = 0; v < 16; ++v) sum[x][v] += acc[x][y][v];
            }
            // dz, a part (bf16: it, and what rounding leaves of it) at a time: [example][class] in LDS, then runs of 512 (fp32: 64) bytes
            const int parts = PL == 1 && p.rest_rows ? 2 : PL;
#pragma unroll
            for (int part = 0; part < 2; ++part) {
                if (part >= parts) continue;
#pragma unroll
                for (int y = 0; y < BY; ++y) {
                    const int eg = PL == 2 ? examples[wj + 32 * y + (lane & 31)].eg : 0;
#pragma unroll
                    for (int x = 0; x < BX; ++x) {
                        // (the second parts anew, not all of them kept from the first ones' turn on)
                        if (PL == 2 || part == 1) asm volatile("" : "+v"(acc[x][y]));
#pragma unroll
                        for (int q = 0; q < 4; ++q) {
                            f32x4 w = {acc[x][y][4 * q], acc[x][y][4 * q + 1], acc[x][y][4 * q + 2], acc[x][y][4 * q + 3]};
                            char *to = lds + (wj + 32 * y + (lane & 31)) * kTileStride + (row0 + 32 * x + 8 * q) * 2;
                            if constexpr (PL == 1) {
                                if (part == 1) w = f32x4{rest_of(w[0]), rest_of(w[1]), rest_of(w[2]), rest_of(w[3])};
                                store4(reinterpret_cast<bf16_t *>(to), w[0], w[1], w[2], w[3]);
                            } else {
                                if (part == 0) {
#pragma unroll
                                    for (int k = 0; k < 4; ++k) acc[x][y][4 * q + k] = w[k] = ldexpf(w[k], 14 - eg);
                                }
                                f16x4 h[2];
                                two_parts(w, 0, h);
                                *reinterpret_cast<f16x4 *>(to) = h[part];
                            }
                        }
                    }
                }
                __syncthreads();
#pragma unroll
                for (int k = 0; k < TN / 16; ++k) {
                    const int at = k * 512 + threadIdx.x, col = tj * TN + (at >> 5), row = ti * kTA + (at & 31) * 8;
                    if (col < p.cols && row < p.ld_dz)
                        *reinterpret_cast<f32x4 *>(p.dz + (size_t)(col + (PL == 1 ? part * p.rest_rows : 0)) * p.ld_dz * PL + column_at<PL>(row, part)) =
                            *reinterpret_cast<const f32x4 *>(lds + (at >> 5) * kTileStride + (at & 31) * 16);
                }
                __syncthreads();
            }
            // db: over the 32 lanes that have an example each, then over the waves that share classes.  Sixteen sums to a lane become one: at each step a
            // lane hands half of them to its partner and adds up the other half.
            float *all = reinterpret_cast<float *>(lds);    // [WB][256]
            const bool odd8 = lane & 8, odd2 = lane & 2, odd1 = lane & 1;
#pragma unroll
            for (int x = 0; x < BX; ++x) {
                float h8[8], h4[4], h2[2];
#pragma unroll
                for (int v = 0; v < 8; ++v) {
                    const auto q = __builtin_amdgcn_permlane16_swap(__float_as_uint(sum[x][v]), __float_as_uint(sum[x][v + 8]), false, false);
                    const unsigned q0 = q[0], q1 = q[1];
                    h8[v] = __uint_as_float(q0) + __uint_as_float(q1);
                }
#pragma unroll
                for (int v = 0; v < 4; ++v) h4[v] = (odd8 ? h8[v + 4] : h8[v]) + row_ror<8>(odd8 ? h8[v] : h8[v + 4]);
#pragma unroll
                for (int v = 0; v < 2; ++v) h2[v] = (odd2 ? h4[v + 2] : h4[v]) + dpp<0x4E>(odd2 ? h4[v] : h4[v + 2]);
                float h = (odd1 ? h2[1] : h2[0]) + dpp<0xB1>(odd1 ? h2[0] : h2[1]);
                h += __shfl_xor(h, 4);
                const int v = (lane & 16 ? 8 : 0) + (odd8 ? 4 : 0) + (odd2 ? 2 : 0) + (odd1 ? 1 : 0);
                if (!(lane & 4)) all[wave % WB * kTA + row0 + 32 * x + 8 * (v >> 2) + (v & 3)] = h;
            }
            __syncthreads();
            if (p.db && threadIdx.x < kTA) {
                float s = 0.f;
#pragma unroll
                for (int w = 0; w < WB; ++w) s += all[w * kTA + threadIdx.x];
                const int row = ti * kTA + threadIdx.x;
                if (row < p.classes) p.db[(size_t)tj * p.ld_db + row] = s;
            }
        }
    }
}

// ------------------------------------------------------------------------------------------ before and after the products
// A bf16 matrix [rows][cols] as the products take it: [rows_p][cols_p], zeros past its end, and, where there are labels, in rows that have
// none or whose weight is zero.
__device__ __forceinline__ bool row_counts(int row, const int32_t *labels, const float *g, int classes)
{
    if (!labels) return true;
    const int y = labels[row];
    return y >= 0 && y < classes && (!g || g[row] != 0.f);
}
__global__ __launch_bounds__(256) void xent_lay_kernel(const bf16_t *__restrict__ from, int rows, int cols, bf16_t *to, int rows_p, int cols_p, const int32_t *labels,
                                                       const float *g, int classes)
{
    const int groups = cols_p / 8;
    for (size_t at = (size_t)blockIdx.x * 256 + threadIdx.x; at < (size_t)rows_p * groups; at += (size_t)gridDim.x * 256) {
        const int row = (int)(at / groups), c = (int)(at - (size_t)row * groups) * 8;
        const bool there = row < rows && row_counts(row, labels, g, classes);
        Eight<bf16_t> v;
        v.load(there ? from + (size_t)row * cols + c : from, there ? cols - c : 0);
        *reinterpret_cast<Eight<bf16_t>::u32x4 *>(to + (size_t)row * cols_p + c) = v.w;
    }
}
// An fp32 matrix in two f16 parts: [rows][cols] becomes [rows_p][cols_p], rows that do not count (as above, or masked by a bias) zeros.  kMost only seeks
// the rows' largest exponent; kOwn lays rows in units of their own, which go into e (and the exponents of g into eg), and seeks the largest of both.
// Every workgroup leaves the largest it met in part [blocks].  The next launch makes one of the n_part of them, which it leaves in *most: kShared takes
// units of what eg[row] leaves of it, kAll takes it as it is.  (The largest is the same in any order.)
enum { kMost, kOwn, kShared, kAll };
struct Lay32 {
    const float *from;
    int rows, cols;
    bf16_t *to;
    int rows_p, cols_p;
    const int32_t *labels;
    const float *g;
    int classes;
    const float *bias;
    int *e, *eg, *part, n_part, *most;
    int blocks;
};
template <int KIND, int U, int W>      // W waves to a row, U groups of eight columns a lane in registers; U = 0: rows of any length, met twice
__device__ __forceinline__ void lay32_rows(const Lay32 &l, int block)
{
    const float *from = l.from;
    const int rows = l.rows, cols = l.cols, rows_p = l.rows_p, cols_p = l.cols_p;
    constexpr int LANES = 64 * W, ROWS = 4 / W;
    __shared__ float waves[2][4];
    __shared__ int most_of_wave[4];
    const int lane = threadIdx.x % LANES, groups = cols_p / 8;
    auto most_of_all = [&](int most) __attribute__((always_inline)) {
#pragma unroll
        for (int d = 32; d; d >>= 1) most = max(most, __shfl_xor(most, d));
        if ((threadIdx.x & 63) == 0) most_of_wave[threadIdx.x >> 6] = most;
        __syncthreads();
        return max(max(most_of_wave[0], most_of_wave[1]), max(most_of_wave[2], most_of_wave[3]));
    };
    int largest = INT_MIN, turn = 0, most = 0;
    if constexpr (KIND == kShared || KIND == kAll) {
        most = INT_MIN;
        for (int k = threadIdx.x; k < l.n_part; k += 256) most = max(most, l.part[k]);
        most = most_of_all(most);
        if (most == INT_MIN) most = 0;        // of zeros only
        if (block == 0 && threadIdx.x == 0) *l.most = most;
    }
    auto magnitude = [](const Eight<float> &v) __attribute__((always_inline)) {
        float m = 0.f;
#pragma unroll
        for (int k = 0; k < 8; ++k) {
            const float x = __builtin_fabsf(v.get(k));
            m = x < INFINITY ? fmaxf(m, x) : m;
        }
        return m;
    };
    for (int row = block * ROWS + threadIdx.x / LANES; row < rows_p; row += l.blocks * ROWS) {
        const bool there = row < rows && row_counts(row, l.labels, l.g, l.classes) && (!l.bias || l.bias[row] > -INFINITY);
        const float *src = from + (size_t)(there ? row : 0) * cols;
        Eight<float> kept[U ? U : 1];
        auto group_of = [&](int u) __attribute__((always_inline)) { return u * LANES + lane; };
#pragma unroll
        for (int u = 0; u < U; ++u) kept[u].load(there && group_of(u) * 8 < cols ? src + group_of(u) * 8 : from, there ? cols - group_of(u) * 8 : 0);
        int unit;
        if constexpr (KIND == kShared) unit = there ? l.eg[row] - most + 14 : 0;
        else if constexpr (KIND == kAll) unit = 14 - most;
        else {
            float m = 0.f;
            if constexpr (U > 0)
#pragma unroll
                for (int u = 0; u < U; ++u) m = fmaxf(m, magnitude(kept[u]));
            else if (there)
                for (int c = lane * 8; c < cols; c += LANES * 8) {
                    Eight<float> v;
                    v.load(src + c, cols - c);
                    m = fmaxf(m, magnitude(v));
                }
            m = all_max(m);
            if constexpr (W == 4) {
                if ((threadIdx.x & 63) == 0) waves[turn][threadIdx.x >> 6] = m;
                __syncthreads();
                m = fmaxf(fmaxf(waves[turn][0], waves[turn][1]), fmaxf(waves[turn][2], waves[turn][3]));
                turn ^= 1;
            }
            const int mine = exponent_of(m), of_g = there && l.g ? exponent_of(l.g[row]) : 0;
            unit = 14 - mine;
            if (KIND == kOwn && lane == 0 && row < rows) {
                l.e[row] = mine;
                if (l.eg) l.eg[row] = of_g;
            }
            if (m > 0.f && mine + of_g > largest) largest = mine + of_g;
        }
        if constexpr (KIND == kMost) continue;
        auto write = [&](int c, const Eight<float> &v) __attribute__((always_inline)) {
            f16x4 lo[2], hi[2];
            two_parts(v.lo, unit, lo);
            two_parts(v.hi, unit, hi);
#pragma unroll
            for (int part = 0; part < 2; ++part)
                *reinterpret_cast<f16x8 *>(l.to + (size_t)row * cols_p * 2 + column_at<2>(c, part)) = __builtin_shufflevector(lo[part], hi[part], 0, 1, 2, 3, 4, 5, 6, 7);
        };
        if constexpr (U > 0) {
#pragma unroll
            for (int u = 0; u < U; ++u)
                if (group_of(u) < groups) write(group_of(u) * 8, kept[u]);
        } else
            for (int group = lane; group < groups; group += LANES) {
                Eight<float> v;
                v.load(there && group * 8 < cols ? src + group * 8 : from, there ? cols - group * 8 : 0);
                write(group * 8, v);
            }
    }
    if constexpr (KIND == kMost || KIND == kOwn)
        if (l.part) {
            largest = most_of_all(largest);
            if (threadIdx.x == 0) l.part[block] = largest;
        }
}

// Zeros where the contraction over examples reads past the last of them, `count` 16 bytes of dz (and of what rounding leaves of it), and in rows
// whose label no piece holds.
struct Clear { bf16_t *dz, *dz_rest; size_t count; float *rest_of_label; int N, blocks; };
__device__ __forceinline__ void clear(const Clear &c, int block)
{
    for (size_t at = (size_t)block * 256 + threadIdx.x; at < c.count; at += (size_t)c.blocks * 256) {
        *reinterpret_cast<f32x4 *>(c.dz + at * 8) = f32x4{};
        if (c.dz_rest) *reinterpret_cast<f32x4 *>(c.dz_rest + at * 8) = f32x4{};
    }
    if (c.rest_of_label)
        for (int at = block * 256 + threadIdx.x; at < c.N; at += c.blocks * 256) c.rest_of_label[at] = 0.f;
}
__global__ __launch_bounds__(256) void xent_clear_kernel(Clear c) { clear(c, blockIdx.x); }

// What comes before the first product of fp32 operands, in two launches: bytes bound them (50001 x 1001: 49 and 80 us, 4.1 and 5.1 TB/s), or, where there
// are few, a chain of loads each (100 x 4096 x 1000, loss and gradients: 97 us in all; 111 with each of the five parts in a launch of its own).
template <int U, int W> __global__ __launch_bounds__(256) void xent_first_kernel(Lay32 a, Lay32 w, Clear c)
{
    const int block = blockIdx.x;
    if (block < a.blocks) lay32_rows<kOwn, U, W>(a, block);
    else if (block < a.blocks + w.blocks) lay32_rows<kMost, U, W>(w, block - a.blocks);
    else clear(c, block - a.blocks - w.blocks);
}
template <int U, int W> __global__ __launch_bounds__(256) void xent_second_kernel(Lay32 a, Lay32 w)
{
    const int block = blockIdx.x;
    if (block < a.blocks) lay32_rows<kShared, U, W>(a, block);
    else lay32_rows<kAll, U, W>(w, block - a.blocks);
}

__device__ __forceinline__ void write_loss(Sums s, float z_label, int label, int classes, float *loss, float *stats, int row)
{
    const float log_s = s.m == -INFINITY && s.e == 0.f ? -INFINITY : s.m < INFINITY ? log1pf(s.e) : NAN;
    if (loss) loss[row] = label < 0 || label >= classes ? 0.f : log_s != log_s ? log_s : z_label == -INFINITY ? INFINITY : log_s - (z_label - s.m);
    if (stats) { stats[2 * (size_t)row] = s.m; stats[2 * (size_t)row + 1] = log_s; }
}

// The tiles' sums [tiles][N] of a row: ROWS rows to a workgroup, 256 / ROWS runs of tiles each.
template <int ROWS>
__global__ __launch_bounds__(256) void xent_join_kernel(const Sums *__restrict__ sums, int tiles, int N, int classes, const int32_t *__restrict__ labels,
                                                        const float *__restrict__ z_label, float *loss, float *stats)
{
    constexpr int RUNS = 256 / ROWS;
    __shared__ Sums all[RUNS][ROWS];
    const int at = threadIdx.x % ROWS, run = threadIdx.x / ROWS, row = blockIdx.x * ROWS + at;
    Sums s = {-INFINITY, 0.f};
    if (row < N)
#pragma unroll 4
        for (int t = run; t < tiles; t += RUNS) s = joined(s, sums[(size_t)t * N + row]);
    all[run][at] = s;
#pragma unroll
    for (int half = RUNS / 2; half > 0; half /= 2) {
        __syncthreads();
        if (run < half) all[run][at] = s = joined(s, all[run + half][at]);
    }
    if (run || row >= N) return;
    const int y = labels[row];
    write_loss(s, y >= 0 && y < classes ? z_label[row] : 0.f, y, classes, loss, stats, row);
}

// WAVES waves to a row, 1 or 4.
template <int WAVES>
__global__ __launch_bounds__(256) void xent_rows_kernel(Scores z, const int32_t *__restrict__ labels, float *loss, float *stats)
{
    __shared__ Sums all[4];
    __shared__ float z_labels[4];
    const int wave = threadIdx.x >> 6, row = WAVES == 4 ? blockIdx.x : blockIdx.x * 4 + wave, at = threadIdx.x % (64 * WAVES);
    if (row >= z.N) return;                 // (one wave to a row: no barrier)
    const int y = labels[row];
    float z_label = -INFINITY;
    Sums s = {-INFINITY, 0.f};
    for (int k = at * 4; k < z.classes; k += 256 * WAVES) {
        const f32x4 v = z.at(row, k);
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            s = v[j] == v[j] ? joined(s, Sums{v[j], 0.f}) : Sums{s.m, v[j]};
            z_label = k + j == y ? v[j] : z_label;
        }
    }
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) {
        s = joined(s, Sums{__shfl_xor(s.m, o), __shfl_xor(s.e, o)});
        const float other = __shfl_xor(z_label, o);
        z_label = z_label == -INFINITY ? other : z_label;       // (a masked label's is -inf in any case)
    }
    if constexpr (WAVES == 4) {
        if ((threadIdx.x & 63) == 0) { all[wave] = s; z_labels[wave] = z_label; }
        __syncthreads();
        for (int w = 1; w < 4; ++w) {
            s = joined(s, all[w]);
            z_label = z_label == -INFINITY ? z_labels[w] : z_label;
        }
    }
    if (at == 0) write_loss(s, z_label, y, z.classes, loss, stats, row);
}
// dz [PL][N][ld_dz] of all classes, and db of a range of rows: 256 classes to a workgroup, four rows at a time.
template <int PL>
__global__ __launch_bounds__(256) void xent_grad_kernel(Scores z, const int32_t *__restrict__ labels, const float *__restrict__ stats, const float *__restrict__ g,
                                                        bf16_t *dz, int ld_dz, float *db, size_t ld_db, const int *__restrict__ eg, int rest_rows, float *rest_of_label)
{
    __shared__ f32x4 sums[4][64];
    const int k = blockIdx.x * 256 + (threadIdx.x & 63) * 4, r = threadIdx.x >> 6;
    const int r0 = (int)((long)z.N * blockIdx.y / gridDim.y), r1 = (int)((long)z.N * (blockIdx.y + 1) / gridDim.y);
    f32x4 sum = {};
    if (k < ld_dz)
        for (int row = r0 + r; row < r1; row += 4) {
            const int y = labels[row];
            const float w = y >= 0 && y < z.classes ? g[row] : 0.f, m = stats[2 * (size_t)row], log_s = stats[2 * (size_t)row + 1];
            f32x4 out = {};
            if (k < z.classes && w != 0.f && log_s != -INFINITY) {
                const f32x4 v = z.at(row, k);
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const float d = (v[j] - m) - log_s;
                    out[j] = w * (k + j != y ? exp_of(below(d)) : v[j] == -INFINITY ? 0.f : expm1f(d));
                }
            }
            sum += out;
            bf16_t *to = dz + (size_t)row * ld_dz * PL;
            if constexpr (PL == 1) {
                store4(to + k, out[0], out[1], out[2], out[3]);
                if (rest_rows) store4(to + (size_t)rest_rows * ld_dz + k, rest_of(out[0]), rest_of(out[1]), rest_of(out[2]), rest_of(out[3]));
#pragma unroll
                for (int j = 0; j < 4; ++j)
                    if (k + j == y && k + j < z.classes) rest_of_label[row] = rest_of(out[j]);
            } else {
#pragma unroll
                for (int j = 0; j < 4; ++j) out[j] = ldexpf(out[j], 14 - eg[row]);
                f16x4 h[2];
                two_parts(out, 0, h);
#pragma unroll
                for (int part = 0; part < 2; ++part) *reinterpret_cast<f16x4 *>(to + column_at<2>(k, part)) = h[part];
            }
        }
    sums[r][threadIdx.x & 63] = sum;
    __syncthreads();
    if (r || !db) return;
#pragma unroll
    for (int q = 1; q < 4; ++q) sum += sums[q][threadIdx.x];
#pragma unroll
    for (int j = 0; j < 4; ++j)
        if (k + j < z.classes) db[(size_t)blockIdx.y * ld_db + k + j] = sum[j];
}

// Scores of few fp32 rows, from weights where they are, and what becomes of them: their sums, or dz and db.  Seeking the weights' exponent, laying them out and
// reading that back would pass memory four times instead of once.  Both come from here, bit for bit the same scores: the gradient of a label that is all but
// certain is what z - m and log s leave of each other, and scores of another product, off by their own rounding, would leave that instead.  A wave: 32 classes and R times 32 rows, by the fp32 matrix unit; a lane has a class (and a row) of its own and, of 8
// contraction indices, four; U times 8 of them at once and the next on their way.  The read bounds one group of 32 rows (sums, 1 x 4096 x 131072: 496 us, 4.3 TB/s),
// the way of the rows out of L2 two (64 rows 914).
struct Few {
    const float *a, *w, *bias;       // w and bias of class0 on
    const int32_t *labels;
    int N, In, class0, classes, all_classes;
    Sums *sums;                      // kStats: [tiles of classes][N]
    float *z_label;                  // [N]
    const float *stats, *g;          // kGrad, and as in Product:
    const int *eg;
    bf16_t *dz;
    int ld_dz;
    float *db;
};
// (gradients: pieces of the classes, in workgroups that fill the chip sooner.  Loss and gradients of 64 x 4096 x 131072 5502 us with eight waves, 4473 with four, 4812 with two)
constexpr int few_waves(int mode) { return mode == kStats ? kTA / 32 : 4; }
template <int R, int U, int MODE>
__global__ __launch_bounds__(64 * few_waves(MODE)) void xent_few_kernel(Few p)
{
    const float *a = p.a, *w = p.w, *bias = p.bias;
    const int N = p.N, In = p.In, K = p.classes;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, half = lane >> 5, k0 = (blockIdx.x * few_waves(MODE) + wave) * 32;
    const float *of_w = w + (size_t)(k0 + (lane & 31) < K ? k0 + (lane & 31) : K - 1) * In, *of_a[R];
#pragma unroll
    for (int r = 0; r < R; ++r) of_a[r] = a + (size_t)(32 * r + (lane & 31) < N ? 32 * r + (lane & 31) : N - 1) * In;
    f32x16 acc[R] = {};
    f32x4 vw[2][U], va[2][R][U];
    auto fetch = [&](int c0, f32x4 (&to_w)[U], f32x4 (&to_a)[R][U]) __attribute__((always_inline)) {
        if (c0 + 8 * U <= In) {
#pragma unroll
            for (int u = 0; u < U; ++u) __builtin_memcpy(&to_w[u], of_w + c0 + 8 * u + 4 * half, 16);
#pragma unroll
            for (int r = 0; r < R; ++r)
#pragma unroll
                for (int u = 0; u < U; ++u) __builtin_memcpy(&to_a[r][u], of_a[r] + c0 + 8 * u + 4 * half, 16);
        } else
#pragma unroll
            for (int u = 0; u < U; ++u)
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    const int c = c0 + 8 * u + 4 * half + k, at = c < In ? c : In - 1;
                    const float x = of_w[at];
                    to_w[u][k] = c < In ? x : 0.f;
#pragma unroll
                    for (int r = 0; r < R; ++r) {
                        const float y = of_a[r][at];
                        to_a[r][u][k] = c < In ? y : 0.f;
                    }
                }
    };
    auto multiply = [&](const f32x4 (&by_w)[U], const f32x4 (&by_a)[R][U]) __attribute__((always_inline)) {
#pragma unroll
        for (int u = 0; u < U; ++u)
#pragma unroll
            for (int k = 0; k < 4; ++k)
#pragma unroll
                for (int r = 0; r < R; ++r) acc[r] = __builtin_amdgcn_mfma_f32_32x32x2f32(by_w[u][k], by_a[r][u][k], acc[r], 0, 0, 0);
    };
    fetch(0, vw[0], va[0]);
    for (int c = 0; c < In; c += 16 * U) {
        if (c + 8 * U < In) fetch(c + 8 * U, vw[1], va[1]);
        multiply(vw[0], va[0]);
        if (c + 8 * U >= In) break;
        if (c + 16 * U < In) fetch(c + 16 * U, vw[0], va[0]);
        multiply(vw[1], va[1]);
    }
    // value v of a lane: class 8 (v / 4) + 4 (lane / 32) + v % 4, row lane % 32
    float b[16];
#pragma unroll
    for (int v = 0; v < 16; ++v) {
        const int k = k0 + 8 * (v >> 2) + 4 * half + (v & 3);
        b[v] = k >= K ? -INFINITY : bias ? bias[k] : 0.f;
    }
    if constexpr (MODE == kStats) {
        __shared__ Sums all[8][R * 32];
#pragma unroll
        for (int r = 0; r < R; ++r) {
            const int row = 32 * r + (lane & 31), label = row < N ? p.labels[row] : -1;
            Sums s = {-INFINITY, 0.f};
            bool here = false;
            float z_of = 0.f;
#pragma unroll
            for (int v = 0; v < 16; ++v) {
                const int k = k0 + 8 * (v >> 2) + 4 * half + (v & 3);
                const float z = b[v] == -INFINITY ? -INFINITY : acc[r][v] + b[v];
                acc[r][v] = z;
                s.m = fmaxf(s.m, z);
                if (k == label && k < K) { here = true; z_of = z; }
            }
            if (here) p.z_label[row] = z_of;
            bool fresh = s.m > -INFINITY;               // one of the largest does not count
            const float base = fresh ? s.m : 0.f;
#pragma unroll
            for (int v = 0; v < 16; ++v) {
                const float e = exp_of(below(acc[r][v] - base));
                const bool it = fresh && acc[r][v] == s.m;
                s.e += it ? 0.f : e;
                fresh = fresh && !it;
            }
            s = joined(s, Sums{__shfl_xor(s.m, 32), __shfl_xor(s.e, 32)});
            if (half == 0) all[wave][row] = s;
        }
        __syncthreads();
        const int row = threadIdx.x;
        if (row >= R * 32 || row >= N) return;
        Sums s = all[0][row];
#pragma unroll
        for (int q = 1; q < 8; ++q) s = joined(s, all[q][row]);
        p.sums[(size_t)blockIdx.x * N + row] = s;
    } else {
        float sum[16] = {};
#pragma unroll
        for (int r = 0; r < R; ++r) {
            const int row = 32 * r + (lane & 31), label = row < N ? p.labels[row] : -1;
            const bool counts = label >= 0 && label < p.all_classes;
            const float g = counts ? p.g[row] : 0.f, m = counts ? p.stats[2 * row] : 0.f, log_s = counts ? p.stats[2 * row + 1] : 0.f;
            const bool none = g == 0.f || log_s == -INFINITY;      // (-inf: a row without a class)
            const int own = counts ? label - p.class0 : -1, unit = row < N ? 14 - p.eg[row] : 0;
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                const int k = k0 + 8 * q + 4 * half;
                f32x4 out;
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const int v = 4 * q + j;
                    const float z = b[v] == -INFINITY ? -INFINITY : acc[r][v] + b[v], d = (z - m) - log_s;
                    float share = exp_of(below(d));
                    if (k + j == own) share = z == -INFINITY ? 0.f : expm1f(d);
                    out[j] = none || k + j >= K ? 0.f : g * share;
                    sum[v] += out[j];
                    out[j] = ldexpf(out[j], unit);
                }
                f16x4 h[2];
                two_parts(out, 0, h);
                if (row < N && k < p.ld_dz)
#pragma unroll
                    for (int part = 0; part < 2; ++part) *reinterpret_cast<f16x4 *>(p.dz + (size_t)row * p.ld_dz * 2 + column_at<2>(k, part)) = h[part];
            }
        }
        if (!p.db) return;
#pragma unroll
        for (int v = 0; v < 16; ++v) {
            const float s = team_sum<32>(sum[v]);
            const int k = k0 + 8 * (v >> 2) + 4 * half + (v & 3);
            if ((lane & 31) == 0 && k < K) p.db[k] = s;
        }
    }
}

// dw of few rows, a sum of up to NMAX outer products: a thread's eight columns of the activations stay in registers, dz is the same for all
// threads, and what is left is the write (4 rows, 200003 x 4096 bf16: 284 us, 5.8 TB/s of writes; in 256 x 256 tiles 432, in narrower ones 558).
template <int PL, int NMAX, typename G>
__global__ __launch_bounds__(256) void xent_outer_kernel(const bf16_t *__restrict__ a, int cols_a, const bf16_t *__restrict__ dz, int ld_dz, int rest_rows, int N, int cols, int classes,
                                                         const int *__restrict__ most, G *dw)
{
    const int c = (blockIdx.x * 256 + threadIdx.x) * 8, n = cols - c < 0 ? 0 : cols - c < 8 ? cols - c : 8;
    if (n == 0) return;
    // eight numbers of a row in PL parts
    auto numbers = [](const bf16_t *row, int at, float (&v)[8]) __attribute__((always_inline)) {
        if constexpr (PL == 1) {
            Eight<bf16_t> e;
            e.load(row + at, 8);
#pragma unroll
            for (int k = 0; k < 8; ++k) v[k] = e.get(k);
        } else {
            const f16x8 h = *reinterpret_cast<const f16x8 *>(row + column_at<2>(at, 0)), l = *reinterpret_cast<const f16x8 *>(row + column_at<2>(at, 1));
#pragma unroll
            for (int k = 0; k < 8; ++k) v[k] = (float)h[k] + (float)l[k];
        }
    };
    float v[NMAX][8];
#pragma unroll
    for (int r = 0; r < NMAX; ++r) {
        numbers(a + (size_t)(r < N ? r : 0) * cols_a * PL, c, v[r]);        // (laid out in whole stages)
#pragma unroll
        for (int k = 0; k < 8; ++k) v[r][k] = r < N ? v[r][k] : 0.f;
    }
    const int groups = (classes + 7) / 8, g0 = (int)((long)groups * blockIdx.y / gridDim.y), g1 = (int)((long)groups * (blockIdx.y + 1) / gridDim.y);
    const int units = PL == 2 ? *most - 28 : 0;
    for (int group = g0; group < g1; ++group) {
        float w[NMAX][8];
#pragma unroll
        for (int r = 0; r < NMAX; ++r) {
            numbers(dz + (size_t)(r < N ? r : 0) * ld_dz * PL, group * 8, w[r]);
            if constexpr (PL == 1) {
                float rest[8];
                numbers(dz + (size_t)(rest_rows + (r < N ? r : 0)) * ld_dz, group * 8, rest);
#pragma unroll
                for (int k = 0; k < 8; ++k) w[r][k] += rest[k];
            }
        }
#pragma unroll
        for (int k = 0; k < 8; ++k) {
            if (group * 8 + k >= classes) break;
            float out[8] = {};
#pragma unroll
            for (int r = 0; r < NMAX; ++r)
#pragma unroll
                for (int q = 0; q < 8; ++q) out[q] = __builtin_fmaf(w[r][k], v[r][q], out[q]);
            if constexpr (PL == 2) {
#pragma unroll
                for (int q = 0; q < 8; ++q) out[q] = ldexpf(out[q], units);
            }
            Eight<G> e;
            e.set(out);
            e.store(dw + (size_t)(group * 8 + k) * cols + c, n);
        }
    }
}

// out [rows][cols] = the sum of `parts` matrices [rows][ld], `part` elements apart, in order; da of bf16 operands: and of what rounding left of dz
// at a row's label, times the label's weights.  That one number is most of a row's dz: without it da would be off by as much again as by
// its own rounding to bf16, with one sign for the whole row.  Where relu_of is given, 0 where that is not above 0.
template <typename T>
__global__ __launch_bounds__(256) void xent_add_kernel(const float *__restrict__ from, int parts, size_t part, size_t ld, int rows, int cols, T *out,
                                                       const float *__restrict__ rest_of_label, const int32_t *__restrict__ labels, const bf16_t *__restrict__ w,
                                                       const void *relu_of, int relu_dtype)
{
    const int groups = (cols + 3) / 4;
    for (size_t at = (size_t)blockIdx.x * 256 + threadIdx.x; at < (size_t)rows * groups; at += (size_t)gridDim.x * 256) {
        const size_t row = at / groups;
        const int c = (int)(at - row * groups) * 4;
        f32x4 s = {};
        for (int q = 0; q < parts; ++q) s += *reinterpret_cast<const f32x4 *>(from + q * part + row * ld + c);     // (ld is a multiple of 4)
        if (rest_of_label)
            if (const float r = rest_of_label[row]; r != 0.f) {
                const bf16_t *of = w + (size_t)labels[row] * cols + c;
#pragma unroll
                for (int k = 0; k < 4; ++k)
                    if (c + k < cols) s[k] = __builtin_fmaf(r, bf16_to_f32(of[k]), s[k]);
            }
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            if (c + k >= cols) continue;
            const size_t to = row * cols + c + k;
            const bool open = !relu_of || (relu_dtype == VGG_BF16 ? bf16_to_f32(static_cast<const bf16_t *>(relu_of)[to]) : static_cast<const float *>(relu_of)[to]) > 0.f;
            Elem<T>::store(out + to, open ? s[k] : 0.f);
        }
    }
}

// ------------------------------------------------------------------------------------------------------ launches
static_assert(lds_of(256, kGrad, 2) <= 160 * 1024 && lds_of(256, kStore, 2) <= 160 * 1024 && lds_of(128, kGrad, 3) <= 160 * 1024, "LDS of a compute unit");
template <bool A_TR, bool B_TR, int TN, int PL, int MODE> int launch_product(const Product &p, hipStream_t s)
{
    auto *kernel = &xent_product_kernel<A_TR, B_TR, TN, PL, MODE>;
    // (a short contraction has no more stages: more workgroups to a compute unit)
    const int lds = lds_of(TN, MODE, MODE == kStore ? PL * (p.steps / p.splits + 1) : stages_of(TN));
    if (lds > 65536 && !raise_lds_limit(reinterpret_cast<const void *>(kernel))) return VGG_ERR_LAUNCH;
    const long grid = div_up(p.rows, kTA) * div_up(p.cols, TN) * p.splits;
    kernel<<<(int)grid, 512, lds, s>>>(p);
    return launch_status();
}
template <bool A_TR, bool B_TR, int MODE> int product(int PL, int tn, const Product &p, hipStream_t s)
{
    if (PL == 2)
        return tn == 256   ? launch_product<A_TR, B_TR, MODE == kGrad ? 128 : 256, 2, MODE>(p, s)
               : tn == 128 ? launch_product<A_TR, B_TR, 128, 2, MODE>(p, s)
                           : launch_product<A_TR, B_TR, 64, 2, MODE>(p, s);
    return tn == 256   ? launch_product<A_TR, B_TR, 256, 1, MODE>(p, s)
           : tn == 128 ? launch_product<A_TR, B_TR, 128, 1, MODE>(p, s)
                       : launch_product<A_TR, B_TR, 64, 1, MODE>(p, s);
}

template <int PL, typename G> int outer(const Product &q, const bf16_t *a, int cols_a, const bf16_t *dz, int ld_dz, int rest_rows, int N, hipStream_t s)
{
    const long across = div_up(q.rows, 2048), down = div_up(2048, across), most = div_up(q.cols, 8);
    const dim3 grid((unsigned)across, (unsigned)(down < most ? down : most));
    G *to = static_cast<G *>(q.out);
    if (N <= 4) xent_outer_kernel<PL, 4, G><<<grid, 256, 0, s>>>(a, cols_a, dz, ld_dz, rest_rows, N, q.rows, q.cols, q.most, to);
    else if (N <= 8) xent_outer_kernel<PL, 8, G><<<grid, 256, 0, s>>>(a, cols_a, dz, ld_dz, rest_rows, N, q.rows, q.cols, q.most, to);
    else xent_outer_kernel<PL, 16, G><<<grid, 256, 0, s>>>(a, cols_a, dz, ld_dz, rest_rows, N, q.rows, q.cols, q.most, to);
    return launch_status();
}

int lay(const void *from, int rows, int cols, void *to, int rows_p, int cols_p, const int32_t *labels, const float *g, int classes, hipStream_t s)
{
    const long blocks = div_up((long)rows_p * (cols_p / 8), 256);
    xent_lay_kernel<<<(int)(blocks < 8192 ? blocks : 8192), 256, 0, s>>>(static_cast<const bf16_t *>(from), rows, cols, static_cast<bf16_t *>(to), rows_p, cols_p, labels, g,
                                                                         classes);
    return launch_status();
}
// fp32: a row's waves and its groups in registers, for activations and weights alike, which are as long; f takes both as constants.
template <typename F> int by_length(int cols, F f)
{
    const std::integral_constant<int, 0> any{};
    const std::integral_constant<int, 1> one{};
    const std::integral_constant<int, 2> two{};
    const std::integral_constant<int, 4> four{};
    if (cols <= 512) f(one, one);
    else if (cols <= 1024) f(two, one);
    else if (cols <= 2048) f(one, four);
    else if (cols <= 4096) f(two, four);
    else if (cols <= 8192) f(four, four);
    else f(any, four);
    return launch_status();
}
int lay32_blocks(int rows, int cols)
{
    const long blocks = cols <= 1024 ? div_up(rows, 4) : rows;
    return (int)(blocks < kParts ? blocks : kParts);
}
int lay32_first(Lay32 a, Lay32 w, Clear clear, hipStream_t s)      // each where it has blocks
{
    return by_length(a.cols, [&](auto u, auto waves) {
        xent_first_kernel<decltype(u)::value, decltype(waves)::value><<<a.blocks + w.blocks + clear.blocks, 256, 0, s>>>(a, w, clear);
    });
}
int lay32_second(Lay32 a, Lay32 w, hipStream_t s)
{
    return by_length(w.cols, [&](auto u, auto waves) { xent_second_kernel<decltype(u)::value, decltype(waves)::value><<<a.blocks + w.blocks, 256, 0, s>>>(a, w); });
}
int add_parts(int dtype, const float *from, int parts, size_t part, size_t ld, int rows, int cols, void *out, hipStream_t s, const float *rest = nullptr,
              const int32_t *labels = nullptr, const void *w = nullptr, const void *relu_of = nullptr, int relu_dtype = 0)
{
    const bf16_t *w16 = static_cast<const bf16_t *>(w);
    const long blocks = div_up((long)rows * div_up(cols, 4), 256);
    const int grid = (int)(blocks < 8192 ? blocks : 8192);
    if (dtype == VGG_BF16) xent_add_kernel<bf16_t><<<grid, 256, 0, s>>>(from, parts, part, ld, rows, cols, static_cast<bf16_t *>(out), rest, labels, w16, relu_of, relu_dtype);
    else xent_add_kernel<float><<<grid, 256, 0, s>>>(from, parts, part, ld, rows, cols, static_cast<float *>(out), rest, labels, w16, relu_of, relu_dtype);
    return launch_status();
}

struct Call {
    int dtype, N, In, K;
    const void *a, *w;
    const float *bias;
    const int32_t *labels;
    char *ws;
    hipStream_t s;
};
template <typename T> T *at(const Call &c, size_t offset) { return reinterpret_cast<T *>(c.ws + offset); }

// fp32: activations, and a piece's weights (of `here` classes), as they are laid out; exponents behind another: those of all, the parts of them.
Lay32 activations(const Call &c, const XentPlan &pl)
{
    Lay32 l = {};
    l.from = static_cast<const float *>(c.a); l.rows = c.N; l.cols = c.In; l.rows_p = pl.NP; l.cols_p = pl.InP;
    l.to = at<bf16_t>(c, pl.a_at);
    l.e = at<int>(c, pl.ea_at);
    l.most = at<int>(c, pl.most_at); l.part = l.most + 2;
    l.blocks = l.n_part = lay32_blocks(l.rows_p, c.In);
    return l;
}
Lay32 weights(const Call &c, const XentPlan &pl, int class0, int here)
{
    Lay32 l = {};
    l.from = static_cast<const float *>(c.w) + (size_t)class0 * c.In; l.rows = l.rows_p = here; l.cols = c.In; l.cols_p = pl.InP;
    l.to = at<bf16_t>(c, pl.w_at);
    l.bias = c.bias ? c.bias + class0 : nullptr;
    l.most = at<int>(c, pl.most_at) + 1; l.part = l.most + 1 + kParts;
    l.blocks = l.n_part = lay32_blocks(here, c.In);
    return l;
}

// The product that gives the scores of a piece: classes are the rows of C, examples its columns.  fp32: `first`, `clear`: what goes with the search for
// its weights' largest exponent, `second`: with laying them out.
int scores_product(const Call &c, const XentPlan &pl, int piece, bool laid_a, const Lay32 &first, const Clear &clear, const Lay32 &second, Product &p)
{
    const int es = c.dtype == VGG_BF16 ? 2 : 4, class0 = piece * pl.classes, here = c.K - class0 < pl.classes ? c.K - class0 : pl.classes;
    const char *w = static_cast<const char *>(c.w) + (size_t)class0 * c.In * es;
    const size_t ld = (size_t)pl.InP * 2 * pl.PL;
    p = Product{};
    p.rows = here; p.cols = c.N; p.steps = pl.InP / kStep; p.splits = 1;
    if (pl.direct_w) p.a = {w, ld, here, nullptr};
    else {
        const int rows_p = up(here, kStep);
        int rc;
        if (pl.PL == 2) {
            Lay32 of_w = weights(c, pl, class0, here);
            if ((rc = lay32_first(first, of_w, clear, c.s))) return rc;
            of_w.rows_p = rows_p;
            of_w.blocks = lay32_blocks(rows_p, c.In);
            rc = lay32_second(second, of_w, c.s);
        } else
            rc = lay(w, here, c.In, c.ws + pl.w_at, rows_p, pl.InP, nullptr, nullptr, 0, c.s);
        if (rc) return rc;
        p.a = {c.ws + pl.w_at, ld, here, nullptr};
    }
    p.b = {laid_a ? c.ws + pl.a_at : static_cast<const char *>(c.a), ld, c.N, nullptr};
    if (pl.PL == 2) { p.ea = at<int>(c, pl.ea_at); p.most = at<int>(c, pl.most_at) + 1; }
    p.bias = c.bias; p.labels = c.labels;
    p.class0 = class0; p.classes = here; p.all_classes = c.K;
    return VGG_OK;
}
int scores_in_parts(const XentPlan &pl, const Call &c, Product &p, Scores &z)
{
    p.splits = pl.z_splits;
    p.out = c.ws + pl.z_at; p.ld = pl.ld_z; p.part = (size_t)c.N * pl.ld_z;
    z = {static_cast<const float *>(p.out), pl.z_splits, c.N, c.K, pl.ld_z, c.bias};
    return product<false, false, kStore>(pl.PL, pl.tn, p, c.s);
}

Few few_rows(const Call &c, int class0, int here)
{
    Few p = {};
    p.a = static_cast<const float *>(c.a); p.w = static_cast<const float *>(c.w) + (size_t)class0 * c.In; p.bias = c.bias ? c.bias + class0 : nullptr;
    p.labels = c.labels;
    p.N = c.N; p.In = c.In; p.class0 = class0; p.classes = here; p.all_classes = c.K;
    return p;
}
template <int MODE> int few_scores(const Few &p, hipStream_t s)
{
    constexpr int W = few_waves(MODE);
    const int tiles = (int)div_up(p.classes, 32 * W);
    if (p.N <= 32) xent_few_kernel<1, 8, MODE><<<tiles, 64 * W, 0, s>>>(p);
    else xent_few_kernel<2, 4, MODE><<<tiles, 64 * W, 0, s>>>(p);
    return launch_status();
}

int forward(const Call &c, float *loss, float *stats)
{
    const XentPlan pl = xent_plan(c.dtype, c.N, c.In, c.K);
    int rc;
    Sums *sums = at<Sums>(c, pl.sums_at);
    float *z_label = at<float>(c, pl.label_at);
    const int tiles = (int)div_up(c.K, kTA);
    auto join = [&] {
        if (c.N <= 512) xent_join_kernel<1><<<c.N, 256, 0, c.s>>>(sums, tiles, c.N, c.K, c.labels, z_label, loss, stats);
        else xent_join_kernel<16><<<(int)div_up(c.N, 16), 256, 0, c.s>>>(sums, tiles, c.N, c.K, c.labels, z_label, loss, stats);
        return launch_status();
    };
    if (pl.few_rows) {
        Few p = few_rows(c, 0, c.K);
        p.sums = sums; p.z_label = z_label;
        if ((rc = few_scores<kStats>(p, c.s))) return rc;
        return join();
    }
    if (pl.PL == 1 && !pl.direct_a && (rc = lay(c.a, c.N, c.In, c.ws + pl.a_at, pl.NP, pl.InP, nullptr, nullptr, 0, c.s))) return rc;
    Lay32 of_a = {};
    if (pl.PL == 2) {
        of_a = activations(c, pl);
        of_a.part = nullptr;
    }
    Lay32 none = {};
    none.cols = c.In;
    for (int piece = 0; piece < pl.pieces; ++piece) {
        Product p;
        if ((rc = scores_product(c, pl, piece, !pl.direct_a, of_a, {}, none, p))) return rc;
        if (pl.z_splits) {
            Scores z;
            if ((rc = scores_in_parts(pl, c, p, z))) return rc;
            return xent_rows(z, c.labels, loss, stats, c.s);
        }
        of_a = none;
        p.sums = sums; p.z_label = z_label;
        if ((rc = product<false, false, kStats>(pl.PL, pl.tn, p, c.s))) return rc;
    }
    return join();
}

int backward(const Call &c, int g_dtype, const float *stats, const float *g, void *da, void *dw, float *db, int relu_mask)
{
    const XentPlan pl = xent_plan(c.dtype, c.N, c.In, c.K);
    const int gs = g_dtype == VGG_BF16 ? 2 : 4;
    const bool two = pl.PL == 2;
    bf16_t *dz = at<bf16_t>(c, pl.dz_at);
    int *eg = two ? at<int>(c, pl.eg_at) : nullptr;
    float *rest = two ? nullptr : at<float>(c, pl.rest_at);
    int rc;
    Clear clear = {};
    clear.dz = dz + (size_t)c.N * pl.ld_dz * pl.PL;
    clear.count = (size_t)(pl.NP - c.N) * pl.ld_dz * pl.PL / 8;
    clear.dz_rest = pl.rest_rows ? clear.dz + (size_t)pl.rest_rows * pl.ld_dz : nullptr;
    clear.rest_of_label = rest;
    clear.N = c.N;
    const size_t most = clear.count > (size_t)c.N || !rest ? clear.count : c.N;
    clear.blocks = (int)(most < 256 * 1024 ? div_up(most, 256) : 1024);
    bf16_t *a_of_dw = at<bf16_t>(c, two ? pl.a2_at : pl.a_at);
    Lay32 first = {}, second = {}, none = {};
    none.cols = c.In;
    if (two) {
        first = activations(c, pl);
        first.labels = c.labels; first.g = g; first.classes = c.K; first.eg = eg;
        second = dw ? first : none;
        second.to = a_of_dw;
    } else {
        if (clear.blocks) {
            xent_clear_kernel<<<clear.blocks, 256, 0, c.s>>>(clear);
            if ((rc = launch_status())) return rc;
        }
        if ((rc = lay(c.a, c.N, c.In, c.ws + pl.a_at, pl.NP, pl.InP, c.labels, g, c.K, c.s))) return rc;
    }
    float *da_part = at<float>(c, pl.da_at), *dw_part = at<float>(c, pl.dw_at);
    for (int piece = 0; piece < pl.pieces; ++piece) {
        Product p;
        if ((rc = scores_product(c, pl, piece, true, first, clear, second, p))) return rc;
        first = second = none;
        clear.blocks = 0;
        const Operand w = p.a;
        const int class0 = p.class0, here = p.classes;
        float *db_to = db ? pl.db_parts == 1 ? db + class0 : at<float>(c, pl.db_at) : nullptr;
        if (pl.z_splits) {
            Scores z;
            if ((rc = scores_in_parts(pl, c, p, z))) return rc;
            const dim3 grid((unsigned)div_up(pl.ld_dz, 256), (unsigned)pl.db_parts);
            if (two) xent_grad_kernel<2><<<grid, 256, 0, c.s>>>(z, c.labels, stats, g, dz, pl.ld_dz, db_to, pl.ld_dz, eg, 0, nullptr);
            else xent_grad_kernel<1><<<grid, 256, 0, c.s>>>(z, c.labels, stats, g, dz, pl.ld_dz, db_to, pl.ld_dz, eg, pl.rest_rows, rest);
            if ((rc = launch_status())) return rc;
        } else if (pl.few_rows) {
            Few q = few_rows(c, class0, here);
            q.stats = stats; q.g = g; q.eg = eg;
            q.dz = dz; q.ld_dz = pl.ld_dz;
            q.db = db_to;      // (of 64 rows at the most: one part)
            if ((rc = few_scores<kGrad>(q, c.s))) return rc;
        } else {
            p.stats = stats; p.g = g; p.eg = eg;
            p.dz = dz; p.ld_dz = pl.ld_dz; p.rest_rows = pl.rest_rows; p.rest_of_label = rest;
            p.db = db_to; p.ld_db = pl.ld_dz;
            if ((rc = product<false, false, kGrad>(pl.PL, pl.grad_tn, p, c.s))) return rc;
        }
        if (db && pl.db_parts > 1 && (rc = add_parts(VGG_F32, db_to, pl.db_parts, pl.ld_dz, pl.ld_dz, 1, here, db + class0, c.s))) return rc;
        const size_t ld_dz = (size_t)pl.ld_dz * 2 * pl.PL;
        // (a last piece's gradients beyond its classes: zeros up to the contraction's next stage)
        if (da) {
            Product q = {};
            const int steps = (int)div_up(here, kStep);
            q.a = w;
            q.a.rows = (int)w.ld;
            if (pl.direct_w && here % kStep) {
                const int from = here / kStep * kStep;
                if ((rc = lay(w.p + (size_t)from * w.ld, here - from, c.In, c.ws + pl.tail_at, kStep, c.In, nullptr, nullptr, 0, c.s))) return rc;
                q.a.tail = c.ws + pl.tail_at;
            }
            q.b = {reinterpret_cast<const char *>(dz), ld_dz, c.N, nullptr};
            q.rows = c.In; q.cols = c.N; q.steps = steps; q.splits = pl.da_splits < steps ? pl.da_splits : steps;
            q.ea = eg; q.most = p.most;
            q.out = da_part; q.ld = pl.InP; q.part = (size_t)c.N * pl.InP; q.add = piece > 0;
            if ((rc = product<true, false, kStore>(pl.PL, pl.da_tn, q, c.s))) return rc;
        }
        if (dw) {
            Product q = {};
            q.a = {reinterpret_cast<const char *>(a_of_dw), (size_t)pl.InP * 2 * pl.PL, pl.InP * 2 * pl.PL, nullptr};
            q.b = {reinterpret_cast<const char *>(dz), ld_dz, (int)ld_dz, nullptr};
            q.rows = c.In; q.cols = here; q.steps = (pl.NP + pl.rest_rows) / kStep; q.splits = pl.dw_splits;
            q.wrap = pl.rest_rows / kStep;
            q.most = two ? at<int>(c, pl.most_at) : nullptr;
            void *out = static_cast<char *>(dw) + (size_t)class0 * c.In * gs;
            q.out = out;
            if (c.N <= kOuterRows) {
                rc = two                  ? outer<2, float>(q, a_of_dw, pl.InP, dz, pl.ld_dz, pl.rest_rows, c.N, c.s)
                     : g_dtype == VGG_F32 ? outer<1, float>(q, a_of_dw, pl.InP, dz, pl.ld_dz, pl.rest_rows, c.N, c.s)
                                          : outer<1, bf16_t>(q, a_of_dw, pl.InP, dz, pl.ld_dz, pl.rest_rows, c.N, c.s);
                if (rc) return rc;
                continue;
            }
            if (q.splits == 1) { q.ld = c.In; q.bf16 = g_dtype == VGG_BF16; }
            else { q.out = dw_part; q.ld = pl.InP; q.part = (size_t)here * pl.InP; }
            if ((rc = product<true, true, kStore>(pl.PL, pl.dw_tn, q, c.s))) return rc;
            if (q.splits > 1 && (rc = add_parts(g_dtype, dw_part, q.splits, q.part, pl.InP, here, c.In, out, c.s))) return rc;
        }
    }
    if (da) return add_parts(g_dtype, da_part, pl.da_splits, (size_t)c.N * pl.InP, pl.InP, c.N, c.In, da, c.s, rest, c.labels, c.w, relu_mask ? c.a : nullptr, c.dtype);
    return VGG_OK;
}

}  // namespace

int xent_rows(const Scores &z, const int32_t *labels, float *loss, float *stats, hipStream_t s)
{
    if (z.classes <= 1024 && z.parts == 1) xent_rows_kernel<1><<<(z.N + 3) / 4, 256, 0, s>>>(z, labels, loss, stats);
    else xent_rows_kernel<4><<<z.N, 256, 0, s>>>(z, labels, loss, stats);
    return launch_status();
}

size_t fc_xent_workspace(int dtype, int N, int In, int K)
{
    return xent_is_small(dtype, N, In, K) ? fc_xent_small_workspace(N, K) : xent_plan(dtype, N, In, K).forward_bytes;
}
size_t fc_xent_bwd_workspace(int dtype, int N, int In, int K)
{
    return xent_is_small(dtype, N, In, K) ? fc_xent_small_workspace(N, K) : xent_plan(dtype, N, In, K).backward_bytes;
}

int fc_xent(int dtype, int N, int In, int K, const void *a, const void *w, const float *bias, const int32_t *labels, float *loss, float *stats, void *ws,
            hipStream_t s)
{
    if (xent_is_small(dtype, N, In, K)) 
        return fc_xent_small(N, In, K, static_cast<const float *>(a), static_cast<const float *>(w), bias, labels, loss, stats, ws, s);
    return forward(Call{dtype, N, In, K, a, w, bias, labels, static_cast<char *>(ws), s}, loss, stats);
}

int fc_xent_bwd(int dtype, int g_dtype, int N, int In, int K, const void *a, const void *w, const float *bias, const int32_t *labels, const float *stats,
                const float *g_loss, void *da, void *dw, float *db, int relu_mask, void *ws, hipStream_t s)
{
    if (xent_is_small(dtype, N, In, K)) 
        return fc_xent_small_bwd(N, In, K, static_cast<const float *>(a), static_cast<const float *>(w), bias, labels, stats, g_loss, static_cast<float *>(da),
                                 static_cast<float *>(dw), db, relu_mask, ws, s);
    return backward(Call{dtype, N, In, K, a, w, bias, labels, static_cast<char *>(ws), s}, g_dtype, stats, g_loss, da, dw, db, relu_mask);
}

}  // namespace vgg
