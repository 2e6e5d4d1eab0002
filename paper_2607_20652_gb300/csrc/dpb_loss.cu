// dpb_loss.cu -- softmax cross entropy over a vocabulary from the hidden rows,
// and its gradient, on the tcgen05 tensor cores.
//
//   z = H W^T,  lse_t = log sum_v exp z_tv,  loss_t = lse_t - z_t,y
//   dz_tv = g_t (exp(z_tv - lse_t) - [v = y]),  dH = dz W,  dW = dz^T H
//
// z is never in memory: the forward reduces each 256 x 256 tile of it to a
// maximum and a sum per row while the next tile is multiplied. The gradient
// forms the tiles again, a piece of the vocabulary at a time, and writes dz of
// the piece in bf16, which the two other products then read; with T tokens, V
// words and d columns that is 2 T V d operations forward and 6 T V d for the
// gradient, where keeping z would save 2 T V d and cost T V values.
//
// What bf16 costs: of dH nothing beyond its own rounding (0.0017 of its norm) in
// rows whose targets' entries are the largest, as these have what rounding leaves of
// them added (Before, rest_of). Of dW 0.0018 with one gradient for all tokens and 0.0023 to
// 0.0024 with one for each, where rounding dW alone gives 0.0017: two bf16 would
// double its products, a third of the work. Up to 512 tokens dz has two bf16.
//
// All of it is one kernel of matrix products (product_kernel). Pairs of blocks
// take units, tiles of 256 x 256 of one of the products, from a counter: the pair
// shares each product (each block loads its 128 rows of A and half of B, so an
// operand byte is fetched for 128 products, where single blocks of 128 x 256
// would need half as many bytes again). In a block a warp copies, one issues (in
// the first block of the pair), one takes units, and eight take the sums out of
// TMEM, two accumulators in turn, so that a unit's results are formed while the
// next unit is multiplied.
//
// What bounds it, at 8192 tokens, 50257 words, 768 columns: forward the products
// (500 cycles of 512 a slot of 64 columns; 327 us at once, 1930 TFLOP/s, 355 to
// 375 us for as long as one likes, when the power limit holds the clock at 1.6 GHz; the
// library's product of these sizes, which writes the scores, 350 and 395 us). The
// gradient's units take 650 (dz: its stores and the products' operands share the
// shared memory), 670 (dH) and 560 cycles (dW) a slot, 1155 us at once and 1300 us
// at the power limit, 1460 TFLOP/s, where three library products take 1190.
// Measured and not taken: dz and dW stored by the row warps themselves, with
// seven slots in place of the rows on their way (dz 760 cycles a slot); two
// places for a warp's rows with five slots (710, 750 and 620); a kernel for each
// piece (14 launches: 1460 us); pieces of 2048 words (1430 us) or 8192 (as 4096).
//
// Tokens that take no part are not multiplied: their places are closed up
// first (prepare_kernel, gather_kernel), which also keeps whatever their rows
// hold out of the sums.
#include <cuda_bf16.h>
#include <math_constants.h>

#include <algorithm>
#include <cstring>
#include <type_traits>

#include "dpb_checks.h"
#include "dpb_device.cuh"
#include "dpb_rows.cuh"
#include "dpb_tensor_core.cuh"

namespace dpb {
namespace {

using namespace tc;
using bf16 = __nv_bfloat16;

constexpr uint32_t kTries = 1u << 20;  // polls of a wait before it gives up
constexpr int kTile = 256;             // rows and columns of a unit
constexpr int kStages = 6;             // slots of the operands' ring
constexpr int kStageBytes = 32768;     // 128 x 64 of A and of B
constexpr int kStore = 4096;           // a warp's rows on their way to memory: 32 of 64 bf16
constexpr int kRowWarps = 8;
constexpr int kThreads = 128 + 32 * kRowWarps;
constexpr int kAhead = 4;              // units taken ahead, at most
constexpr int kBuffers = 3;            // pieces of dz held, where there are many tokens
constexpr int kMostPieces = 160;
enum Exact { kAsMultiplied = 0, kInJoin = 1, kBeside = 2 };  // where the loss takes its targets' scores from
constexpr int kGroup = 32;             // tiles of rows that pass a tile of the vocabulary before the next
constexpr float kLog2e = 1.4426950408889634f;
constexpr float kLowest = -3.402823466e38f;  // the maximum of no score: finite, so that it can be subtracted

enum Kind { kScores = 0, kGrad = 1, kDHidden = 2, kDWeight = 3, kEnd = 4 };

// What the tokens' pass leaves for the others.
struct Head {
    int count;     // tokens that take part
    int all;       // none is left out: rows are where they were
    float g_max;   // largest finite |grad_loss| (1 if all are 0)
    int next;      // units taken
    // of each piece, the row warps that are done with a unit of each kind (kGrad, kDHidden, kDWeight)
    int done[kMostPieces][4];
};
// Of the i-th token that takes part: its target, lse, grad_loss / g_max.
struct Token {
    int target;
    float lse, g;
    int row;
};

struct Args {
    CUtensorMap hidden, closed;  // rows as given, and closed up
    CUtensorMap weight;
    CUtensorMap dz, dz_out;  // loaded and stored: [rows, and their remainders][held pieces]
    CUtensorMap dw;
    const bf16 *h, *w;
    int64_t h_stride, w_stride;
    bf16 *closed_rows;
    Head *head;
    Token *tokens;
    int *place;  // of each token: where it went, or -1
    float2 *part;  // [tiles of the vocabulary][rows]
    float *z_target, *z_exact;  // the targets' scores: the tensor cores', and summed by themselves
    float *rest;  // of each token: what is left of its target's dz by rounding it to bf16
    float *loss, *lse;
    int *counted;
    CUtensorMap sums, w_sums;
    float *acc;  // sums of dH, where there are several pieces: [rows][dim], or (split) one for each piece, of T_pad rows
    float *w_acc;  // sums of dW over parts of the tokens, where these are several: [parts][V_pad][dim]
    bf16 *dh, *dw_rows;
    int64_t dh_stride, dw_stride;
    int64_t T, T_pad;
    int V, d, piece;  // piece: words of a piece
    int pieces, held;
    int parts, part_rows, V_pad;  // parts of the tokens that dW is summed over apart, and the rows of each
    bool split;  // each piece's sums of dH apart, added up by join_sums_kernel
    bool fine;   // dz as two bf16, the rounded value and the remainder
    bool want_h, want_w;
    int exact;
    bool few;  // rows that the tokens' cluster closes up itself
    uint32_t tries;  // polls of a unit's wait for others
    int32_t *status;
};

struct Unit {
    int kind, m0, n0, blocks;  // blocks: of 64 along K
    int piece, part;  // part: of the tokens (kDWeight)
};

// ---- units ------------------------------------------------------------------------

// Tiles of the vocabulary: groups of rows' tiles, so that the tiles under way
// share both operands.
__device__ __forceinline__ Unit score_unit(int kind, int u, int tiles_m, int tiles_n, int d, int piece) {
    const int group = u / (kGroup * tiles_n), in = u - group * kGroup * tiles_n;
    const int rows = min(kGroup, tiles_m - group * kGroup);
    return Unit{kind, (group * kGroup + in % rows) * kTile, in / rows * kTile, (d + 63) / 64, piece, 0};
}

// How many units each product has, and which is the u-th. The gradient's
// pieces overlap: dz of a piece comes before the products that read the piece
// before it, so that what a unit waits for was taken a piece's time ago:
//   dz 0, dz 1, dH 0, dW 0, dz 2, dH 1, dW 1, ..., dW last, dH last
// (in the last one the longer units come first, so that the pairs end together);
// where all of dz is held, all of it comes first.
struct List {
    int tiles_m, tiles_d, words;  // words of the vocabulary that a piece (the forward: all) has
    int count, last;              // tokens; words of the last piece
    __device__ __forceinline__ List(const Args &a, int count_) : count(count_) {
        tiles_m = (count + kTile - 1) / kTile, tiles_d = (a.d + kTile - 1) / kTile;
        words = a.loss ? a.V : a.piece;
        last = a.loss ? a.V : a.V - (a.pieces - 1) * a.piece;
    }
    __device__ __forceinline__ int words_of(const Args &a, int piece) const { return piece == a.pieces - 1 ? last : words; }
    __device__ __forceinline__ int grad_units(int w) const { return tiles_m * ((w + kTile - 1) / kTile); }
    __device__ __forceinline__ int weight_units(const Args &a, int w) const {
        return a.want_w ? (w + kTile - 1) / kTile * tiles_d * a.parts : 0;
    }
    __device__ __forceinline__ int hidden_units(const Args &a) const { return a.want_h ? tiles_m * tiles_d : 0; }
    __device__ __forceinline__ Unit reader(const Args &a, int u, int piece) const {
        const int w = words_of(a, piece), n_w = weight_units(a, w), n_h = hidden_units(a);
        const int rows = a.parts > 1 ? a.part_rows : count;  // that a unit of dW sums over
        const bool h_first = piece < a.pieces - 1 || w > rows;
        if (u >= n_w + n_h) return Unit{kEnd, 0, 0, 0, 0, 0};
        const bool is_h = h_first ? u < n_h : u >= n_w;
        u -= is_h && !h_first ? n_w : !is_h && h_first ? n_h : 0;
        const int each = is_h ? n_h : n_w / a.parts, part = is_h ? 0 : u / each;
        u -= part * each;
        const int blocks = ((is_h ? w : max(0, min(rows, count - part * rows))) + 63) / 64;
        return Unit{is_h ? kDHidden : kDWeight, u / tiles_d * kTile, u % tiles_d * kTile, a.fine ? 2 * blocks : blocks, piece, part};
    }
    __device__ __forceinline__ Unit at(const Args &a, int u) const {
        const int all = a.pieces, first = grad_units(words_of(a, 0));
        if (a.loss) return u < first ? score_unit(kScores, u, tiles_m, (a.V + kTile - 1) / kTile, a.d, 0) : Unit{kEnd, 0, 0, 0, 0, 0};
        int piece = 0;
        if (a.held == all) {
            const int dz = grad_units(words), total = dz * (all - 1) + grad_units(last);
            const bool reads = u >= total;
            if (reads) u -= total;
            const int each = reads ? weight_units(a, words) + hidden_units(a) : dz;
            if (each > 0) piece = min(u / each, all - 1);
            u -= piece * each;
            if (reads) return reader(a, u, piece);
        } else if (u >= first) {
            u -= first;
            const int readers = weight_units(a, words) + hidden_units(a), full = grad_units(words) + readers;
            // pieces 1 .. all - 2 are full, and so are the readers of those before them
            const int step = full > 0 ? max(0, min(u / full, all - 2)) : 0;
            u -= step * full;
            piece = step + 1;
            const int dz = piece < all ? grad_units(words_of(a, piece)) : 0;
            if (u >= dz) {
                u -= dz;
                if (piece < all) {
                    if (u < readers) return reader(a, u, piece - 1);
                    u -= readers;
                    ++piece;
                }
                return reader(a, u, piece - 1);
            }
        }
        return score_unit(kGrad, u, tiles_m, (words_of(a, piece) + kTile - 1) / kTile, a.d, piece);
    }
    // Where the row warps count units of a kind. Where all of dz is held, it is one count.
    __device__ __forceinline__ int *counter(const Args &a, const Unit &t) const {
        return &a.head->done[t.kind == kGrad && a.held == a.pieces ? 0 : t.piece][t.kind];
    }
    // One thread: what the unit waits for has been done: dz of its piece, and the
    // sums of dH before it; for dz, the products that read its place. `all_there`
    // (false at first): all of dz is held and has been waited for.
    __device__ __forceinline__ bool wait(const Args &a, const Unit &t, bool &all_there) const {
        const int each = 2 * kRowWarps;
        if (t.kind == kGrad) {
            const int before = t.piece - a.held;
            if (before < 0) return true;
            if (!reached(a, &a.head->done[before][kDWeight], each * weight_units(a, words)) ||
                !reached(a, &a.head->done[before][kDHidden], each * hidden_units(a)))
                return false;
        } else if (t.kind == kDHidden || t.kind == kDWeight) {
            const bool ordered = t.kind == kDHidden && t.piece > 0 && !a.split;
            if (all_there && !ordered) return true;
            const bool one = a.held == a.pieces;
            const int dz = one ? grad_units(words) * (a.pieces - 1) + grad_units(last) : grad_units(words_of(a, t.piece));
            if ((!all_there && !reached(a, counter(a, Unit{kGrad, 0, 0, 0, t.piece, 0}), each * dz)) ||
                (ordered && !reached(a, &a.head->done[t.piece - 1][kDHidden], each * hidden_units(a))))
                return false;
            all_there = one;
        } else {
            return true;
        }
        fence_cluster();  // for the blocks that it is handed to
        return true;
    }
    static __device__ __forceinline__ bool reached(const Args &a, const int *counter, int target) {
        for (uint32_t i = 0; i < a.tries; ++i) {
            int v;
            asm volatile("ld.acquire.gpu.global.s32 %0, [%1];" : "=r"(v) : "l"(counter) : "memory");
            if (v >= target) return true;
            __nanosleep(200);
        }
        return false;
    }
};

// One thread of a row warp: what it wrote for a unit is in memory.
__device__ __forceinline__ void count_done(int *counter) {
    asm volatile("red.release.gpu.global.add.s32 [%0], 1;" ::"l"(counter) : "memory");
}

// ---- shared memory ------------------------------------------------------------------

struct Shared {
    static constexpr int kData = kStages * kStageBytes, kBars = kData + kRowWarps * kStore;
    // barriers: full and empty of each slot, sums ready and read of each
    // accumulator, upper halves of the rows' sums there (of each accumulator and
    // quarter), units handed over and taken
    static constexpr int kFullBar = kBars, kEmptyBar = kFullBar + 8 * kStages, kReady = kEmptyBar + 8 * kStages,
                         kRead = kReady + 16, kUpper = kRead + 16, kHanded = kUpper + 64, kTaken = kHanded + 8 * kAhead,
                         kUnits = (kTaken + 8 * kAhead + 15) / 16 * 16, kTmem = kUnits + 16 * kAhead, kBytes = kTmem + 4;
    static constexpr int kMerge = kData;  // the upper halves: the forward has no rows on their way to memory
};
static_assert(kRowWarps == 8 && 2 * 128 * 8 <= kRowWarps * kStore, "two halves of a row");
constexpr int kSmem = Shared::kBytes + 1024;  // the data starts at a multiple of 1024

// Units in the order in which they are taken, seen by one role of one block.
// What a unit is, is worked out by the warp that takes them. Handing it over and
// giving its slot back order no plain writes: as releases at cluster scope the
// arrivals had every role wait for its writes (8 x 1024, forward: 410 us
// against 322).
struct Units {
    uint32_t base, taken;  // this block's barriers and slots; the first block's `taken`
    int i = 0;
    __device__ __forceinline__ bool ready() const { return bar_test(base + Shared::kHanded + 8 * (i % kAhead), (i / kAhead) & 1); }
    // All lanes (or one thread): the next unit; false after a wait that gave up.
    __device__ __forceinline__ bool next(Unit &t) {
        const int s = i % kAhead;
        if (!bar_wait(base + Shared::kHanded + 8 * s, (i / kAhead) & 1, kTries)) return false;
        int x;
        asm volatile("ld.shared.v4.u32 {%0, %1, %2, %3}, [%4];"
                     : "=r"(x), "=r"(t.m0), "=r"(t.n0), "=r"(t.blocks)
                     : "r"(base + Shared::kUnits + 16 * s)
                     : "memory");
        t.kind = x & 7, t.piece = x >> 3 & 0xff, t.part = x >> 11;
        ++i;
        return true;
    }
    // One thread of the first block: unit t into slot s of the block of `rank`.
    __device__ __forceinline__ void hand(const Unit &t, int s, uint32_t rank) const {
        const uint32_t bar = peer_addr(base + Shared::kHanded + 8 * s, rank);
        bar_arrive_expect_peer(bar, 16);
        store_peer(peer_addr(base + Shared::kUnits + 16 * s, rank), t.kind | t.piece << 3 | t.part << 11, t.m0, t.n0, t.blocks, bar);
    }
    // One thread: the unit has been read.
    __device__ __forceinline__ void done() const { bar_arrive_peer(taken + 8 * ((i - 1) % kAhead)); }
};

// ---- what becomes of a unit's sums ----------------------------------------------------

__device__ __forceinline__ uint32_t swizzled(uint32_t base, int row, int piece) {
    return base + row * 128 + ((piece ^ (row & 7)) << 4);
}
__device__ __forceinline__ void store_shared(uint32_t addr, uint32_t x, uint32_t y, uint32_t z, uint32_t w) {
    asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(addr), "r"(x), "r"(y), "r"(z), "r"(w) : "memory");
}

__device__ __forceinline__ float4 load_shared(uint32_t addr) {
    float4 x;
    asm volatile("ld.shared.v4.f32 {%0, %1, %2, %3}, [%4];" : "=f"(x.x), "=f"(x.y), "=f"(x.z), "=f"(x.w) : "r"(addr) : "memory");
    return x;
}

// What becomes of a row's target, where it is one of 32 columns: eight of them at a
// time, as a warp has few targets in a tile (65536 tokens, 1000 words, 256 columns,
// forward: 67 us, 71 with all 32).
template <typename F>
__device__ __forceinline__ void at_target(int column, F &&f) {
    if ((unsigned)column >= 32u) return;
#pragma unroll
    for (int k = 0; k < 32; k += 8)
        if (column / 8 == k / 8)
#pragma unroll
            for (int i = k; i < k + 8; ++i)
                if (column == i) f(i);
}

// A row's maximum and sum of exp(z - maximum) over 128 of its scores but the
// target's, which join_kernel adds. 32 of them are added in eight chains of four.
__device__ __forceinline__ float2 reduce_scores(uint32_t tmem, int columns, int target, float *z_target) {
    float top = kLowest, sum = 0.f;
    const uint64_t scale = pair(kLog2e, kLog2e);
#pragma unroll 1
    for (int c = 0; c < 128; c += 32) {
        uint32_t v[32];
        __syncwarp();
        tmem_load(tmem + c, v);
        load_wait(v);
        if (c + 32 > columns)
#pragma unroll
            for (int i = 0; i < 32; ++i)
                if (c + i >= columns) v[i] = 0xff800000u;
        at_target(target - c, [&](int i) { *z_target = __uint_as_float(v[i]), v[i] = 0xff800000u; });
        float m[4];
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            m[k] = __uint_as_float(v[8 * k]);
#pragma unroll
            for (int i = 1; i < 7; i += 2) m[k] = max3(m[k], __uint_as_float(v[8 * k + i]), __uint_as_float(v[8 * k + i + 1]));
            m[k] = fmaxf(m[k], __uint_as_float(v[8 * k + 7]));
        }
        const float now = max3(fmaxf(m[0], m[1]), fmaxf(m[2], m[3]), top);
        const uint64_t less = pair(-now, -now);
        uint64_t s[4] = {0, 0, 0, 0};
#pragma unroll
        for (int i = 0; i < 32; i += 2) {
            const float2 x = unpair(mul2(add2(pair_bits(v[i], v[i + 1]), less), scale));
            s[i / 2 % 4] = add2(s[i / 2 % 4], pair(exp2_approx(x.x), exp2_approx(x.y)));
        }
        const float2 t = unpair(add2(add2(s[0], s[1]), add2(s[2], s[3])));
        sum = fmaf(sum, exp2_approx((top - now) * kLog2e), t.x + t.y);
        top = now;
    }
    return make_float2(top, sum);
}

__device__ __forceinline__ float2 join(float2 a, float2 b) {
    const float top = fmaxf(a.x, b.x);
    return make_float2(top, a.y * exp2_approx((a.x - top) * kLog2e) + b.y * exp2_approx((b.x - top) * kLog2e));
}

// 64 columns of a row's dz as bf16 pairs, into the warp's rows on their way to
// memory; or what their rounding left over. lse is subtracted before the scaling to
// powers of 2, so that a row whose target is all of it gives 0 exactly: scaled by
// itself it would be rounded once more, 4e-5 at a score of 1000. `aim` is set to the
// target's, before it is rounded. `taken` is called once they have been read out of TMEM.
template <typename F>
__device__ __forceinline__ void grad_columns(uint32_t tmem, uint32_t stage, int lane, int columns, const Token &t,
                                             int target, float &aim, bool remainder, F &&taken) {
    const uint64_t scale = pair(kLog2e, kLog2e), less = pair(-t.lse, -t.lse);
    uint32_t both[2][32];
    __syncwarp();
    tmem_load(tmem, both[0]);
    tmem_load(tmem + 32, both[1]);
    load_wait(both[0]);
    load_wait(both[1]);
    taken();
#pragma unroll
    for (int c = 0; c < 64; c += 32) {
        const uint32_t(&v)[32] = both[c / 32];
        float p[32];
#pragma unroll
        for (int i = 0; i < 32; i += 2) {
            const float2 x = unpair(mul2(add2(pair_bits(v[i], v[i + 1]), less), scale));
            p[i] = exp2_approx(x.x), p[i + 1] = exp2_approx(x.y);
        }
        at_target(target - c, [&](int i) { p[i] -= 1.f, aim = p[i] * t.g; });
        if (c + 32 > columns)
#pragma unroll
            for (int i = 0; i < 32; ++i)
                if (c + i >= columns) p[i] = 0.f;
        uint32_t x[16];
#pragma unroll
        for (int i = 0; i < 16; ++i) {
            const float a = p[2 * i] * t.g, b = p[2 * i + 1] * t.g;
            x[i] = pack_bf16(a, b);
            if (remainder) x[i] = pack_bf16(a - __uint_as_float(x[i] << 16), b - __uint_as_float(x[i] & 0xffff0000u));
            if (t.row < 0) x[i] = 0;
        }
#pragma unroll
        for (int i = 0; i < 4; ++i)
            store_shared(swizzled(stage, lane, c / 8 + i), x[4 * i], x[4 * i + 1], x[4 * i + 2], x[4 * i + 3]);
    }
}

// What rounding dz of the target to bf16 leaves goes by itself into dH: four columns
// of its product with the target's row of the weight. As the largest entry of most
// rows it would set their error (a gradient for each of 8192 tokens: 0.0024 of dH's
// norm, 0.0017 with it, which is dH's own rounding).
__device__ __forceinline__ float rest_of(float aim) { return aim - __bfloat162float(__float2bfloat16_rn(aim)); }
__device__ __forceinline__ void add_rest(float4 &x, float rest, uint2 w) {
    x.x = fmaf(rest, __uint_as_float(w.x << 16), x.x);
    x.y = fmaf(rest, __uint_as_float(w.x & 0xffff0000u), x.y);
    x.z = fmaf(rest, __uint_as_float(w.y << 16), x.z);
    x.w = fmaf(rest, __uint_as_float(w.y & 0xffff0000u), x.w);
}

// Four columns of rows row, row + 4, ... of dH as the pieces before have summed
// them (other blocks' values, so not by way of this SM's own cache), and of the
// weight's rows of their targets (`target`: of the warp's row of this lane).
struct Before {
    float4 sums[8];
    uint2 w[8];
    __device__ __forceinline__ void load(const Args &a, bool first, int row, int count, int column, int target) {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const int y = __shfl_sync(kFull, target, (threadIdx.x & 31) / 8 + 4 * i);
            sums[i] = make_float4(0.f, 0.f, 0.f, 0.f);
            w[i] = make_uint2(0, 0);
            if (row + 4 * i >= count || column >= a.d) continue;
            if (!first) sums[i] = __ldcg(reinterpret_cast<const float4 *>(a.acc + (int64_t)(row + 4 * i) * a.d + column));
            if (!a.fine) w[i] = *reinterpret_cast<const uint2 *>(a.w + y * a.w_stride + column);
        }
    }
};

// The next slot of the ring, and how often the ring has been gone round.
struct Turn {
    int slot = 0;
    uint32_t round = 0;
    __device__ __forceinline__ void next() {
        if (++slot == kStages) slot = 0, round ^= 1;
    }
};

// One thread: d = the ring's next `blocks` slots multiplied and added up. A_ROWS,
// B_ROWS: that operand's rows run along K. The next slot is waited for while
// half of a slot's products are still to be issued, so that the tensor cores
// have work meanwhile.
template <bool A_ROWS, bool B_ROWS>
__device__ __forceinline__ bool multiply(uint32_t d, int blocks, uint32_t base, Turn &at) {
    auto wait = [&] { return bar_wait(base + Shared::kFullBar + 8 * at.slot, at.round, kTries); };
    if (!wait()) return false;
    for (int k = 0; k < blocks; ++k) {
        fence_after();
        const uint32_t from = base + at.slot * kStageBytes, done = base + Shared::kEmptyBar + 8 * at.slot;
        const uint64_t da = A_ROWS ? desc_k_rows(from, 8192) : desc_k_inside(from);
        const uint64_t db = B_ROWS ? desc_k_rows(from + 16384, 8192) : desc_k_inside(from + 16384);
        auto product = [&](int i) {
            mma_ss_pair(d, desc_at(da, A_ROWS ? 2048 * i : 32 * i), desc_at(db, B_ROWS ? 2048 * i : 32 * i),
                        mma_shape_pair(kTile, A_ROWS, B_ROWS), k > 0 || i > 0);
        };
        product(0);
        product(1);
        product(2);
        at.next();
        const bool ok = k + 1 == blocks || wait();
        product(3);
        mma_commit_pair(done);
        if (!ok) return false;
    }
    return true;
}

// A warp: the score of a token's target, its products added up in fp32 with each
// sum rounded, where the tensor cores cut off.
__device__ __forceinline__ float target_score(const Args &a, const Token &t) {
    const int lane = threadIdx.x & 31, pieces = a.d / 8;
    const bf16 *h = a.h + t.row * a.h_stride, *w = a.w + t.target * a.w_stride;
    float sum[2] = {0.f, 0.f};
#pragma unroll 4
    for (int i = lane; i < pieces; i += 32) {
        Piece<bf16, 8> x, y;
        load_piece(h + 8 * i, x);
        load_piece(w + 8 * i, y);
#pragma unroll
        for (int j = 0; j < 8; ++j) sum[j & 1] = fmaf(x.v[j], y.v[j], sum[j & 1]);
    }
    float z = sum[0] + sum[1];
#pragma unroll
    for (int i = 16; i > 0; i /= 2) z += __shfl_xor_sync(kFull, z, i);
    return z;
}

// ---- the kernel -------------------------------------------------------------------------

__global__ void __cluster_dims__(2, 1, 1) __launch_bounds__(kThreads, 1) product_kernel(const __grid_constant__ Args a) {
    extern __shared__ uint8_t raw[];
    const uint32_t base = (smem_addr(raw) + 1023) & ~1023u;
    uint8_t *const mem = raw + (base - smem_addr(raw));
    const int warp = threadIdx.x / 32, lane = threadIdx.x & 31;
    const uint32_t rank = cluster_rank();
    bool failed = false;

    auto full = [&](int s) { return base + Shared::kFullBar + 8 * s; };
    auto empty = [&](int s) { return base + Shared::kEmptyBar + 8 * s; };
    if (warp == 0 && elect_one()) {
        for (int s = 0; s < kStages; ++s) {
            bar_init(full(s), 1);
            bar_init(empty(s), 1);
        }
        for (int b = 0; b < 2; ++b) {
            bar_init(base + Shared::kReady + 8 * b, 1);
            bar_init(base + Shared::kRead + 8 * b, 2 * kRowWarps);
            for (int q = 0; q < 4; ++q) bar_init(base + Shared::kUpper + 8 * (4 * b + q), 1);
        }
        for (int s = 0; s < kAhead; ++s) {
            bar_init(base + Shared::kHanded + 8 * s, 1);
            bar_init(base + Shared::kTaken + 8 * s, 2 * kRowWarps + 3);
        }
        bar_init_fence();
    }
    if (warp == 1) tmem_alloc_pair(base + Shared::kTmem, 512);
    fence_before();
    __syncthreads();
    cluster_sync();
    fence_after();
    start_next();
    wait_previous();
    const int count = a.head->count;
    const List list(a, count);
    uint32_t tmem;
    asm volatile("ld.shared.u32 %0, [%1];" : "=r"(tmem) : "r"(base + Shared::kTmem) : "memory");

    Units units{base, peer_addr(base + Shared::kTaken, 0)};
    if (warp == 0) {
        // ---- copies
        if (elect_one()) {
            const CUtensorMap *rows = a.head->all ? &a.hidden : &a.closed;
            int at = 0;  // slots filled
            bool fenced = false;
            Unit t;
            while (true) {
                if ((failed = !units.next(t))) break;
                units.done();
                if (t.kind == kEnd) break;
                // other blocks' dz, which the first block has seen (List::wait), by way of copies
                if (t.kind > kGrad && !(fenced && a.held == a.pieces)) {
                    fence_cluster();
                    fence_async();
                    fenced = true;
                }
                const int v0 = t.piece * a.piece;
                const int dz0 = t.piece % a.held * a.piece;  // the piece's columns of dz
                const int first = t.kind > kGrad && a.fine ? t.blocks / 2 : t.blocks;  // blocks of rounded values
                for (int k = 0; k < t.blocks; ++k, ++at) {
                    const int s = at % kStages;
                    if (at >= kStages && !bar_wait(empty(s), ((at / kStages) & 1) ^ 1, kTries)) {
                        failed = true;
                        break;
                    }
                    const uint32_t bar = peer_addr(full(s), 0), to = base + s * kStageBytes;
                    if (rank == 0) bar_arrive_expect(full(s), 2 * kStageBytes);
                    const int m = t.m0 + 128 * rank, n = t.n0 + 128 * rank;
                    const int kk = t.part * a.part_rows + 64 * (k < first ? k : k - first), rest = k < first ? 0 : (int)a.T_pad;
#pragma unroll
                    for (int j = 0; j < 2; ++j) {
                        const uint32_t ta = to + 8192 * j, tb = ta + 16384;
                        if (t.kind <= kGrad) {
                            copy_box_pair(ta, rows, 64 * k, m + 64 * j, bar);
                            copy_box_pair(tb, &a.weight, 64 * k, v0 + n + 64 * j, bar);
                        } else if (t.kind == kDHidden) {
                            copy_box_pair(ta, &a.dz, dz0 + kk, rest + m + 64 * j, bar);
                            copy_box_pair(tb, &a.weight, n + 64 * j, v0 + kk, bar);
                        } else {
                            copy_box_pair(ta, &a.dz, dz0 + m + 64 * j, rest + kk, bar);
                            copy_box_pair(tb, rows, n + 64 * j, kk, bar);
                        }
                    }
                }
                if (failed) break;
            }
            // no copy is in flight when the pair ends, whatever gave up, and no
            // product's arrival at the second block
            for (int i = max(0, at - kStages); i < at; ++i)
                bar_wait(rank == 0 ? full(i % kStages) : empty(i % kStages), (i / kStages) & 1, kTries);
        }
    } else if (warp == 1) {
        // ---- products
        if (rank == 0 && elect_one()) {
            int sums = 0, slots = 0;
            Turn at;
            Unit t;
            while (true) {
                if ((failed = !units.next(t))) break;
                units.done();
                if (t.kind == kEnd) break;
                if (t.blocks == 0) continue;
                const int b = sums & 1;
                if (sums >= 2 && !bar_wait(base + Shared::kRead + 8 * b, ((sums / 2) & 1) ^ 1, kTries)) {
                    failed = true;
                    break;
                }
                fence_after();
                const uint32_t d = tmem + kTile * b;
                failed = !(t.kind == kDWeight   ? multiply<true, true>(d, t.blocks, base, at)
                           : t.kind == kDHidden ? multiply<false, true>(d, t.blocks, base, at)
                                                : multiply<false, false>(d, t.blocks, base, at));
                if (failed) break;
                mma_commit_pair(base + Shared::kReady + 8 * b);
                ++sums;
                slots = min(slots + t.blocks, kStages);
            }
            // every arrival of a product on a barrier of the pair has come before it ends
            for (int i = 0; i < slots; ++i) {
                at.slot = at.slot == 0 ? (at.round ^= 1, kStages - 1) : at.slot - 1;
                failed |= !bar_wait(empty(at.slot), at.round, kTries);
            }
            for (int i = max(0, sums - 2); i < sums; ++i)
                failed |= !bar_wait(base + Shared::kReady + 8 * (i & 1), (i / 2) & 1, kTries);
        }
    } else if (warp == 2) {
        // ---- units
        if (rank == 0 && elect_one()) {
            bool all_there = false;
            // Two ahead, as a long unit that a pair holds is one that others lack; four
            // where they are so short that taking them is what they wait for.
            int ahead = 2;
            for (int i = 0;; ++i) {
                const int s = i % kAhead, before = i - ahead;
                if (before >= 0 && !bar_wait(base + Shared::kTaken + 8 * (before % kAhead), (before / kAhead) & 1, kTries)) {
                    failed = true;
                    break;
                }
                Unit t = list.at(a, atomicAdd(&a.head->next, 1));
                ahead = t.blocks <= 8 ? kAhead : 2;
                // a wait that gives up ends the pair as the last unit does, with nothing under way
                if (!list.wait(a, t, all_there)) failed = true, t.kind = kEnd;
                units.hand(t, s, 0);
                units.hand(t, s, 1);
                if (t.kind == kEnd) break;
            }
        }
    } else if (warp == 3) {
        // ---- the targets' scores
        if (a.exact == kBeside)
            for (int i = blockIdx.x; i < count; i += gridDim.x) {
                const float z = target_score(a, a.tokens[i]);
                if (lane == 0) a.z_exact[i] = z;
            }
    } else if (warp >= 4) {
        // ---- sums: a row and 128 of its columns a thread
        const int quarter = warp & 3, half = (warp - 4) / 4;
        const uint32_t stage = base + Shared::kData + (warp - 4) * kStore;
        const uint32_t read_bar = peer_addr(base + Shared::kRead, 0);
        const float g = a.head->g_max;
        int sums = 0;
        Unit t;
        // Counts a unit once its copies are in memory, which they are when half of the
        // next unit's are under way (`later`), or before a wait: others may wait for
        // the count.
        int *pending = nullptr;
        auto settle = [&](auto later) {
            if (pending && lane == 0) {
                stores_done<decltype(later)::value>();
                fence_async();
                count_done(pending);
            }
            pending = nullptr;
            __syncwarp();
        };
        auto sums_read = [&](int b) {
            fence_before();
            __syncwarp();
            if (elect_one()) bar_arrive_peer(read_bar + 8 * b);
        };
        const std::integral_constant<int, 0> now{};
        const std::integral_constant<int, 1> later{};
        while (true) {
            if (!__all_sync(kFull, units.ready())) settle(now);
            if (!__all_sync(kFull, units.next(t))) {
                failed = true;
                break;
            }
            __syncwarp();
            if (elect_one()) units.done();
            if (t.kind == kEnd) break;
            const int row0 = t.m0 + 128 * rank + 32 * quarter, row = row0 + lane, column = t.n0 + 128 * half;
            const int b = sums & 1;
            const uint32_t from = tmem + ((uint32_t)quarter << 21) + kTile * b + 128 * half;
            Token token{-1, 0.f, 0.f, -1};
            if (t.kind != kDWeight && row < count) token = a.tokens[row];
            const int aimed = token.target - t.piece * a.piece - column;  // the target's column (kGrad)
            const bool ends = t.kind == kDHidden && t.piece == a.pieces - 1 && !a.split;
            float rest = 0.f;
            Before before;
            if (ends) {
                fence_cluster();  // other blocks' sums, which the first block has seen
                fence_async();
                if (!a.fine && row < count) rest = __ldcg(a.rest + row);
                before.load(a, t.piece == 0, row0 + lane / 8, count, column + 4 * (lane % 8), token.target);
            }
            if (t.blocks > 0) {
                if (!__all_sync(kFull, bar_test(base + Shared::kReady + 8 * b, (sums / 2) & 1))) settle(now);
                if (!__all_sync(kFull, bar_wait(base + Shared::kReady + 8 * b, (sums / 2) & 1, kTries))) {
                    failed = true;
                    break;
                }
                fence_after();
                ++sums;
            }
            if (t.kind != kGrad) settle(now);
            if (t.kind == kScores) {
                float z = 0.f;
                const int target = token.target - column;
                const float2 r = reduce_scores(from, a.V - column, target, &z);
                if (token.row >= 0 && (unsigned)target < 128u) a.z_target[row] = z;
                // both halves of the row
                float2 *merge = reinterpret_cast<float2 *>(mem + Shared::kMerge) + 128 * b + 32 * quarter + lane;
                const uint32_t upper = base + Shared::kUpper + 8 * (4 * b + quarter);
                __syncwarp();
                if (half) {
                    *merge = r;
                    __syncwarp();
                    if (lane == 0) bar_arrive(upper);
                } else {
                    if (!__all_sync(kFull, bar_wait(upper, ((sums - 1) / 2) & 1, kTries))) {
                        failed = true;
                        break;
                    }
                    if (row < count) a.part[(int64_t)(t.n0 / kTile) * a.T_pad + row] = join(r, *merge);
                }
            } else if (t.kind == kGrad) {
                const int words = list.words_of(a, t.piece);
                float aim = 0.f;
                const int at = t.piece % a.held * a.piece + column;
#pragma unroll 1
                for (int part = 0; part <= (int)a.fine; ++part)
#pragma unroll 1
                    for (int c = 0; c < 128; c += 64) {
                        if (lane == 0) stores_read();
                        __syncwarp();
                        grad_columns(from + c, stage, lane, words - column - c, token, aimed - c, aim, part, [&] {
                            if (c && part == (int)a.fine) sums_read(b);  // the products need not wait for the rest
                        });
                        fence_async_shared();
                        __syncwarp();
                        if (lane == 0) store_box(&a.dz_out, stage, at + c, row0 + part * (int)a.T_pad);
                        if (c == 0 && part == 0) settle(later);
                    }
                if (!a.fine && token.row >= 0 && (unsigned)aimed < 128u) a.rest[row] = rest_of(aim);
                __syncwarp();  // before this unit is counted
            } else if (t.kind == kDWeight && a.parts == 1) {
#pragma unroll 1
                for (int c = 0; c < 128; c += 64) {
                    if (lane == 0) stores_read();
                    __syncwarp();
#pragma unroll
                    for (int h = 0; h < 64; h += 32) {
                        uint32_t v[32];
                        if (t.blocks > 0) {
                            tmem_load(from + c + h, v);
                            load_wait(v);
                        } else {
#pragma unroll
                            for (int i = 0; i < 32; ++i) v[i] = 0;
                        }
                        uint32_t x[16];
#pragma unroll
                        for (int i = 0; i < 16; ++i)
                            x[i] = pack_bf16(__uint_as_float(v[2 * i]) * g, __uint_as_float(v[2 * i + 1]) * g);
#pragma unroll
                        for (int i = 0; i < 4; ++i)
                            store_shared(swizzled(stage, lane, h / 8 + i), x[4 * i], x[4 * i + 1], x[4 * i + 2], x[4 * i + 3]);
                    }
                    fence_async_shared();
                    __syncwarp();
                    // the piece's last tile may reach past it, into words that are not its own
                    const int v0 = t.piece * a.piece + row0;
                    if (lane == 0 && column + c < a.d && v0 < a.V) store_box(&a.dw, stage, column + c, v0);
                }
            } else {
                // by way of shared memory: copies add the sums of a piece to those of the
                // pieces before; in the last one eight lanes have 128 bytes of a row. The sums
                // of dW over a part of the tokens are all stored apart.
                const bool of_w = t.kind == kDWeight;
                const bool first = t.piece == 0 || a.split || of_w;
                const int to = row0 + (of_w ? t.part * a.V_pad + t.piece * a.piece : a.split ? t.piece * (int)a.T_pad : 0);
                const CUtensorMap *out = of_w ? &a.w_sums : &a.sums;
                const int r = lane / 8, piece = lane % 8;
#pragma unroll 1
                for (int c = 0; c < 128; c += 32) {
                    uint32_t v[32];
                    __syncwarp();
                    if (t.blocks > 0) {
                        tmem_load(from + c, v);
                        load_wait(v);
                    } else {
#pragma unroll
                        for (int i = 0; i < 32; ++i) v[i] = 0;
                    }
                    if (lane == 0) stores_read();
                    __syncwarp();
#pragma unroll
                    for (int i = 0; i < 8; ++i)
                        store_shared(swizzled(stage, lane, i), v[4 * i], v[4 * i + 1], v[4 * i + 2], v[4 * i + 3]);
                    if (!ends) {
                        fence_async_shared();
                        __syncwarp();
                        if (lane == 0 && first) store_box(out, stage, column + c, to);
                        if (lane == 0 && !first) add_box(out, stage, column + c, to);
                        continue;
                    }
                    const int col = column + c + 4 * piece;
                    float4 sums[8];
#pragma unroll
                    for (int i = 0; i < 8; ++i) {
                        sums[i] = before.sums[i];
                        add_rest(sums[i], __shfl_sync(kFull, rest, r + 4 * i), before.w[i]);
                    }
                    if (c < 96) before.load(a, first, row0 + r, count, col + 32, token.target);
                    __syncwarp();
#pragma unroll
                    for (int i = 0; i < 8; ++i) {
                        const int at = r + 4 * i;
                        const int64_t place = __shfl_sync(kFull, token.row, at);
                        float4 x = load_shared(swizzled(stage, at, piece));
                        if (row0 + at >= count || col >= a.d) continue;
                        x.x += sums[i].x, x.y += sums[i].y, x.z += sums[i].z, x.w += sums[i].w;
                        *reinterpret_cast<uint2 *>(a.dh + place * a.dh_stride + col) =
                            make_uint2(pack_bf16(x.x * g, x.y * g), pack_bf16(x.z * g, x.w * g));
                    }
                }
            }
            if (t.blocks > 0 && t.kind != kGrad) sums_read(b);
            // what others wait for: dz and the sums of dH in memory; of dW, that dz has been read
            if (t.kind == kGrad || t.kind == kDHidden) {
                pending = list.counter(a, t);
            } else if (t.kind == kDWeight) {
                __syncwarp();
                if (lane == 0) count_done(&a.head->done[t.piece][kDWeight]);
                __syncwarp();
            }
        }
        settle(now);
        if (lane == 0) stores_done<0>();
    }
    if (failed) set_status(a.status, DPB_DEV_TIMEOUT);
    __syncwarp();
    fence_before();
    __syncthreads();
    cluster_sync();
    if (warp == 1) tmem_free_pair(tmem, 512);
}

// ---- tokens ---------------------------------------------------------------------------

// Where tokens are left out: the others' rows closed up, and zeros behind them
// to the end of a tile (a product sums over these); zeros in the gradient of
// those left out. By `warps` warps, of which this is one.
__device__ __forceinline__ void close_up(const Args &a, int count, int64_t warp, int64_t warps) {
    const int lane = threadIdx.x & 31, pieces = a.d / 8;
    const int64_t end = min(a.T, (int64_t)(count + kTile - 1) / kTile * kTile);
    const uint4 none = make_uint4(0, 0, 0, 0);
    for (int64_t t = warp; t < a.T; t += warps) {
        const int place = a.place[t];
        const uint4 *from = reinterpret_cast<const uint4 *>(a.h + t * a.h_stride);
        uint4 *to = reinterpret_cast<uint4 *>(a.closed_rows + (int64_t)place * a.d);
        uint4 *dh = reinterpret_cast<uint4 *>(a.dh + t * a.dh_stride);
        uint4 *rest = reinterpret_cast<uint4 *>(a.closed_rows + t * a.d);
        for (int i = lane; i < pieces; i += 32) {
            if (place >= 0) to[i] = from[i];
            else if (a.dh) dh[i] = none;
            if (t >= count && t < end) rest[i] = none;
        }
    }
}

__global__ void __launch_bounds__(256) gather_kernel(const __grid_constant__ Args a) {
    start_next();
    wait_previous();
    if (!a.head->all) close_up(a, a.head->count, blockIdx.x * 8ll + threadIdx.x / 32, gridDim.x * 8ll);
}

// The tokens that take part, closed up in their order, by one cluster: each
// block takes a stretch of them, counts those before each (of a warp's by
// votes, of the warps' and blocks' by sums) and writes them. Also the largest
// |grad_loss|, the counters, and what ignored tokens give.
constexpr int kPrepareBlocks = 8;
struct Tally {
    int count;
    float top;
};
template <typename I>
__global__ void __cluster_dims__(kPrepareBlocks, 1, 1) __launch_bounds__(1024)
    prepare_kernel(const __grid_constant__ Args a, const I *targets, int64_t ignore, const float *grad, int grad_stride,
                   const float *lse) {
    __shared__ Tally warps[32], block;
    start_next();
    const int tid = threadIdx.x, lane = tid & 31, warp = tid / 32;
    const uint32_t rank = cluster_rank();
    // of each warp: a multiple of 32 tokens
    const int64_t each = ((a.T + 32 * kPrepareBlocks - 1) / (32 * kPrepareBlocks) + 31) / 32 * 32;
    const int64_t t0 = min(a.T, (int64_t)(rank * 32 + warp) * each), t1 = min(a.T, t0 + each);
    auto counts = [&](int64_t y) { return y >= 0 && y < a.V && y != ignore; };
    Tally mine{0, 0.f};
#pragma unroll 4
    for (int64_t t = t0 + lane; t < t0 + each; t += 32) {
        const int64_t y = t < t1 ? (int64_t)targets[t] : ignore;
        const bool in = t < t1 && counts(y);
        if (!in && y != ignore) set_status(a.status, DPB_DEV_BAD_INDEX);
        mine.count += __popc(__ballot_sync(kFull, in));
        if (grad && in) {
            const float g = fabsf(grad[t * grad_stride]);
            if (g <= 3.402823466e38f) mine.top = fmaxf(mine.top, g);
        }
    }
#pragma unroll
    for (int i = 16; i > 0; i /= 2) mine.top = fmaxf(mine.top, __shfl_xor_sync(kFull, mine.top, i));
    if (lane == 0) warps[warp] = mine;
    __syncthreads();
    int place = 0;
    Tally all{0, 0.f};
    for (int w = 0; w < 32; ++w) {
        if (w < warp) place += warps[w].count;
        all.count += warps[w].count;
        all.top = fmaxf(all.top, warps[w].top);
    }
    if (tid == 0) block = all;
    cluster_sync();
    all = Tally{0, 0.f};
    for (uint32_t r = 0; r < kPrepareBlocks; ++r) {
        const uint32_t at = peer_addr(smem_addr(&block), r);
        Tally o;
        asm volatile("ld.shared::cluster.b32 %0, [%1];" : "=r"(o.count) : "r"(at) : "memory");
        asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(o.top) : "r"(at + 4) : "memory");
        if (r < rank) place += o.count;
        all.count += o.count;
        all.top = fmaxf(all.top, o.top);
    }
    if (all.top == 0.f) all.top = 1.f;
    if (rank == 0) {
        if (tid == 0) {
            a.head->count = all.count;
            a.head->all = all.count == a.T;
            if (a.counted) *a.counted = all.count;
            a.head->g_max = all.top;
        }
        if (tid == 0) a.head->next = 0;
        if (tid < 4 * kMostPieces) (&a.head->done[0][0])[tid] = 0;
    }
#pragma unroll 4
    for (int64_t t = t0 + lane; t < t0 + each; t += 32) {
        const int64_t y = t < t1 ? (int64_t)targets[t] : ignore;
        const bool in = t < t1 && counts(y);
        const unsigned votes = __ballot_sync(kFull, in);
        const int here = place + __popc(votes & ((1u << lane) - 1));
        place += __popc(votes);
        if (t >= t1) continue;
        a.place[t] = in ? here : -1;
        if (in)
            a.tokens[here] = Token{(int)y, lse ? lse[t] : 0.f, grad ? grad[t * grad_stride] / all.top : 0.f, (int)t};
        else if (a.loss)
            a.loss[t] = a.lse[t] = 0.f;
    }
    cluster_sync();  // the others have read this block's tally, and all places are written
    if (a.few && all.count != a.T) close_up(a, all.count, rank * 32 + warp, 32 * kPrepareBlocks);
}

// lse and loss of the others' maximum and sum and a target's score. An infinite score
// has no loss.
struct LogSum {
    float lse, loss;
};
__device__ __forceinline__ LogSum log_sum(float2 others, float z) {
    if (z >= others.x) {
        const float l = log1pf(others.y * expf(others.x - z));
        return LogSum{z + l, z < CUDART_INF_F ? l : CUDART_NAN_F};
    }
    const float l = logf(others.y + expf(z - others.x));
    return LogSum{others.x + l, others.x - z + l};
}

// The tiles' maxima and sums of 32 rows, joined in the tiles' order of each of
// 32 threads and then of the threads; and the target's score.
__global__ void __launch_bounds__(1024, 2) join_kernel(const __grid_constant__ Args a) {
    __shared__ float2 parts[32][33], joined[32];
    __shared__ float scores[32];
    wait_previous();
    const int lane = threadIdx.x & 31, slice = threadIdx.x / 32, count = a.head->count;
    const int tiles = (a.V + kTile - 1) / kTile;
    const int64_t first = blockIdx.x * 32ll, row = first + lane;
    if (first >= count) return;
    if (a.exact == kInJoin && first + slice < count) {
        const float z = target_score(a, a.tokens[first + slice]);
        if (lane == 0) scores[slice] = z;
    }
    float2 r = make_float2(kLowest, 0.f);
    if (row < count)
        for (int i = slice; i < tiles; i += 32) r = join(r, a.part[i * a.T_pad + row]);
    parts[slice][lane] = r;
    __syncthreads();
    r = parts[lane][slice];  // lane: the slice, slice: the row
#pragma unroll
    for (int i = 16; i > 0; i /= 2) {
        const float2 o = make_float2(__shfl_down_sync(kFull, r.x, i), __shfl_down_sync(kFull, r.y, i));
        r = join(r, o);
    }
    if (lane == 0) joined[slice] = r;
    __syncthreads();
    if (slice > 0 || row >= count) return;
    // The loss is not formed from the rounded lse, and the target is apart, so that
    // it keeps its digits however small it is. lse is that of the tensor cores' score,
    // which the gradient will form again: exp(z - lse) is 1 if all others are 0.
    const int to = a.tokens[row].row;
    const LogSum x = log_sum(joined[lane], a.z_target[row]);
    a.lse[to] = x.lse;
    a.loss[to] = a.exact == kAsMultiplied ? x.loss : log_sum(joined[lane], a.exact == kBeside ? a.z_exact[row] : scores[lane]).loss;
}

// dH from the pieces' sums, where they are apart, and dW from the parts': four
// columns a lane. Where there are few, `slices` warps share an output's sums, each
// its own in order, and then the warps' are added up (33 tokens of 50257 words, 51
// pieces: 5 us in place of 19; 1000 tokens, 13 pieces: 18 with one warp, 24 with eight).
constexpr int kJoinWarps = 8;
__global__ void __launch_bounds__(32 * kJoinWarps) join_sums_kernel(const __grid_constant__ Args a, int slices) {
    __shared__ float4 sums[kJoinWarps][32];
    wait_previous();
    const int each = a.d / 4, lane = threadIdx.x & 31, warp = threadIdx.x / 32, slice = warp % slices;
    const float g = a.head->g_max;
    const int64_t rows_h = a.split && a.want_h ? a.head->count : 0, rows_w = a.parts > 1 && a.want_w ? a.V : 0;
    const int64_t all = (rows_h + rows_w) * each;
    const int outputs = 32 * kJoinWarps / slices;
    for (int64_t i0 = blockIdx.x * (int64_t)outputs; i0 < all; i0 += gridDim.x * (int64_t)outputs) {
        const int64_t at = i0 + warp / slices * 32 + lane, i = min(at, all - 1), row = i / each;
        const int column = (int)(i - row * each) * 4;
        const bool h = row < rows_h;
        const int n = h ? a.pieces : a.parts, p1 = n * (slice + 1) / slices;
        const int64_t step = (h ? a.T_pad : a.V_pad) * a.d;
        const float *from = h ? a.acc + row * a.d + column : a.w_acc + (row - rows_h) * a.d + column;
        float4 sum = make_float4(0.f, 0.f, 0.f, 0.f);
        for (int p = n * slice / slices; p < p1; p += 8) {
            float4 x[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) x[j] = __ldcg(reinterpret_cast<const float4 *>(from + min(p + j, p1 - 1) * step));
#pragma unroll
            for (int j = 0; j < 8; ++j)
                if (p + j < p1) sum.x += x[j].x, sum.y += x[j].y, sum.z += x[j].z, sum.w += x[j].w;
        }
        if (slices > 1) {
            sums[warp][lane] = sum;
            __syncthreads();
            if (slice == 0)
                for (int k = 1; k < slices; ++k) {
                    const float4 x = sums[warp + k][lane];
                    sum.x += x.x, sum.y += x.y, sum.z += x.z, sum.w += x.w;
                }
            __syncthreads();
        }
        if (slice == 0 && h && !a.fine)
            add_rest(sum, a.rest[row], *reinterpret_cast<const uint2 *>(a.w + a.tokens[row].target * a.w_stride + column));
        if (slice == 0 && at < all)
            *reinterpret_cast<uint2 *>((h ? a.dh + a.tokens[row].row * a.dh_stride : a.dw_rows + (row - rows_h) * a.dw_stride) + column) =
                make_uint2(pack_bf16(sum.x * g, sum.y * g), pack_bf16(sum.z * g, sum.w * g));
    }
}

// ---- host side ------------------------------------------------------------------

// Map of rows in boxes of 128 bytes x `box_rows` rows; what lies outside reads as zero.
dpb_status make_map(CUtensorMap *map, const void *data, int64_t stride, int64_t rows, int64_t columns, int box_rows,
                    bool wide = false) {
    const auto fn = tensor_map_encoder();
    if (!fn) return fail(DPB_ERR_CUDA, "the driver has no cuTensorMapEncodeTiled");
    const int elem = wide ? 4 : 2;
    const cuuint64_t dims[2] = {(cuuint64_t)columns, (cuuint64_t)rows};
    const cuuint64_t strides[1] = {(cuuint64_t)(rows > 1 ? stride : (columns + 7) / 8 * 8) * elem};
    const cuuint32_t box[2] = {(cuuint32_t)(128 / elem), (cuuint32_t)box_rows}, one[2] = {1, 1};
    const CUresult r = fn(map, wide ? CU_TENSOR_MAP_DATA_TYPE_FLOAT32 : CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 2,
                          const_cast<void *>(data), dims, strides, box, one, CU_TENSOR_MAP_INTERLEAVE_NONE,
                          CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
    if (r != CUDA_SUCCESS) return fail(DPB_ERR_CUDA, "cuTensorMapEncodeTiled failed (%d)", (int)r);
    return DPB_OK;
}

int64_t round_up(int64_t x, int64_t to) { return (x + to - 1) / to * to; }

// Pieces of the gradient. With many tokens: kPieceBytes of dz each, kBuffers of
// them held, dH added up over them one after the other. Where all of dz takes no
// more than that, all of it is held, and the pieces are as many as give every pair
// of blocks two units of dH, whose sums are kept apart: one after the other few
// units would follow each other through the whole vocabulary (1000 tokens, 50257
// words, 768 columns: 300 us, 210 apart; 2000: 342 and 360; 4096, too many for it,
// 560). With the fewest tokens, whose rounding errors of dz do not average out, dz
// is held to 16 bits, in two bf16: 33 tokens take 119 us, 512 199 (268 and 282 in
// one bf16 and one after the other).
constexpr int64_t kPieceBytes = 64ll << 20;
constexpr int kLeastPiece = 4096, kFineRows = 512;
// Where dW, of few words and columns, has fewer units than there are pairs of
// blocks, they are of parts of the tokens, this many at least, whose sums are added
// up in the end: 65536 tokens, 1000 words, 256 columns took 174 us for the gradient
// (191 with the targets' remainders in dH), 390 with one unit for all tokens; 16384,
// 100, 64 40 and 93; 4096, 1000, 768 63 and 75 (parts of 4096: 174, 46, 77; of 1024
// and two units a pair: 194, 42, 64).
constexpr int kLeastPart = 2048;

struct Space {
    int64_t T_pad, V_pad, piece, pieces, held, columns, parts = 1, part_rows = 0;  // columns: of dz
    bool split = false, fine = false;
    size_t head, tokens, place, closed, part, z_target, z_exact, rest, dz, acc, w_acc, bytes;
    Space(const dpb_linear_loss_config *c, bool backward) {
        const size_t T = (size_t)c->tokens, d = (size_t)c->dim, V = (size_t)c->vocab;
        const int64_t words = round_up(c->vocab, kTile);
        T_pad = round_up(c->tokens, kTile), V_pad = words;
        fine = T_pad <= kFineRows && 4 * T_pad * words <= kBuffers * kPieceBytes;
        if (2 * T_pad * words <= kBuffers * kPieceBytes) {
            const int64_t tiles = std::max<int64_t>(1, T_pad / kTile) * ((c->dim + kTile - 1) / kTile);
            pieces = std::min<int64_t>((2 * (sms_of_device() / 2) + tiles - 1) / tiles, std::min<int64_t>(words / kTile, kMostPieces));
            piece = round_up((c->vocab + pieces - 1) / pieces, kTile);
            held = pieces = (c->vocab + piece - 1) / piece;
            split = pieces > 1;
        } else {
            piece = std::max<int64_t>(kPieceBytes / (2 * std::max<int64_t>(T_pad, 1)) / kTile * kTile, kLeastPiece);
            piece = std::max(piece, round_up((c->vocab + kMostPieces - 1) / kMostPieces, kTile));
            piece = std::min(piece, words);
            pieces = (c->vocab + piece - 1) / piece;
            held = std::min<int64_t>(pieces, kBuffers);
        }
        columns = std::min(held * piece, words);  // the last of all pieces may be shorter
        const int64_t w_units = words / kTile * ((c->dim + kTile - 1) / kTile), pairs = sms_of_device() / 2;
        if (held == pieces && w_units < pairs && T_pad >= 2 * kLeastPart) {
            parts = std::min((pairs + w_units - 1) / w_units, T_pad / kLeastPart);
            part_rows = round_up((c->tokens + parts - 1) / parts, kTile);
            parts = (c->tokens + part_rows - 1) / part_rows;
        }
        size_t at = 1024;  // the status word's
        auto take = [&](size_t n) {
            const size_t r = at;
            at += (n + 1023) / 1024 * 1024;
            return r;
        };
        head = take(sizeof(Head));
        tokens = take(T * sizeof(Token));
        place = take(T * 4);
        closed = take(T * d * 2);
        if (backward) {
            dz = take((size_t)T_pad * (fine ? 2 : 1) * columns * 2);
            acc = take(split ? (size_t)pieces * T_pad * d * 4 : pieces > 1 ? T * d * 4 : 0);
            w_acc = take(parts > 1 ? (size_t)parts * V_pad * d * 4 : 0);
            rest = take(T * 4);
            part = z_target = z_exact = at;
        } else {
            part = take((V + kTile - 1) / kTile * (size_t)T_pad * sizeof(float2));
            z_target = take((size_t)T_pad * 4);
            z_exact = take((size_t)T_pad * 4);
            dz = acc = w_acc = rest = at;
        }
        bytes = at;
    }
};

constexpr int64_t kMostTokens = 1ll << 24, kMostWords = 1ll << 28, kMostUnits = 1ll << 26;
constexpr int kMostDim = 1 << 20;

// Units of the gradient, which has the forward's and more.
int64_t units_of(const dpb_linear_loss_config *c) {
    const int64_t m = (c->tokens + kTile - 1) / kTile, v = ((int64_t)c->vocab + kTile - 1) / kTile;
    const int64_t d = ((int64_t)c->dim + kTile - 1) / kTile;
    const Space w(c, true);
    return m * v + v * d * w.parts + m * d * w.pieces;
}

dpb_status check_config(const dpb_linear_loss_config *c) {
    if (!c) return fail(DPB_ERR_INVALID_ARG, "cfg is NULL");
    if (c->dtype != DPB_BF16) return fail(DPB_ERR_UNSUPPORTED, "the linear cross entropy takes bf16 rows");
    if (c->tokens < 0 || c->vocab < 1 || c->dim < 1) return fail(DPB_ERR_INVALID_ARG, "a size is too small");
    // A unit's products, of all tokens, of a piece of the words or of all columns, take far less than the bound of a
    // wait for them: 2^24 tokens some 0.1 s and 2^20 columns 4 ms, where 2^20 polls of 1.5 us take 1.6 s.
    if (c->tokens > kMostTokens || c->vocab > kMostWords || c->dim > kMostDim)
        return fail(DPB_ERR_UNSUPPORTED, "at most 2^24 tokens, 2^28 words and 2^20 columns");
    if (units_of(c) > kMostUnits) return fail(DPB_ERR_UNSUPPORTED, "too many tokens for a vocabulary and rows this large");
    if (c->dim % 8) return fail(DPB_ERR_UNSUPPORTED, "dim must be a multiple of 8");
    if (c->index_bytes != 4 && c->index_bytes != 8) return fail(DPB_ERR_INVALID_ARG, "index_bytes must be 4 or 8");
    if (c->grad_stride != 0 && c->grad_stride != 1) return fail(DPB_ERR_INVALID_ARG, "grad_stride must be 0 or 1");
    return check_slot(c->status_slot);
}

dpb_status check_rows(const dpb_rows *r, const char *name, int64_t n, int dim) {
    if (n == 0) return DPB_OK;
    if (!r) return fail(DPB_ERR_INVALID_ARG, "%s is NULL", name);
    DPB_CHECK(need(r->data, name, 16));
    if (n > 1 && (r->stride < dim || r->stride % 8))
        return fail(DPB_ERR_INVALID_ARG, "the stride of %s must be a multiple of 8, at least dim", name);
    if (r->stride >= (1ll << 38)) return fail(DPB_ERR_UNSUPPORTED, "the stride of %s is too large", name);
    return DPB_OK;
}

dpb_status launch_products(const Args &a, int64_t units, cudaStream_t s) {
    const cudaError_t e = allow_smem(reinterpret_cast<const void *>(product_kernel), kSmem);
    if (e != cudaSuccess) return launch_status(e, "linear_cross_entropy");
    const unsigned pairs = (unsigned)std::max<int64_t>(1, std::min<int64_t>(units, sms_of_device() / 2));
    return launch_status(launch_early(product_kernel, dim3(2 * pairs), kThreads, kSmem, s, a), "linear_cross_entropy");
}

// What both directions begin with.
dpb_status begin(Args &a, const Space &w, const dpb_linear_loss_config *c, const dpb_rows *hidden, const dpb_rows *weight,
                 const void *targets, const float *grad, const float *lse, uint8_t *ws, cudaStream_t s) {
    a.h = static_cast<const bf16 *>(hidden->data);
    a.h_stride = hidden->stride;
    a.w = static_cast<const bf16 *>(weight->data);
    a.w_stride = weight->stride;
    a.head = reinterpret_cast<Head *>(ws + w.head);
    a.tokens = reinterpret_cast<Token *>(ws + w.tokens);
    a.place = reinterpret_cast<int *>(ws + w.place);
    a.closed_rows = reinterpret_cast<bf16 *>(ws + w.closed);
    a.T = c->tokens;
    a.T_pad = w.T_pad;
    a.V = c->vocab;
    a.d = c->dim;
    a.piece = (int)w.piece;
    a.pieces = (int)w.pieces;
    a.held = (int)w.held;
    a.parts = (int)w.parts;
    a.part_rows = (int)w.part_rows;
    a.V_pad = (int)w.V_pad;
    a.split = w.split;
    a.fine = w.fine;
    // A launch less where eight blocks close the rows up as fast: half of 340 x 768 ignored 16.8 us (17.3 with the
    // launch), of 1000 x 256 15.8 (14.9), of 1000 x 768 19.4 (17.7); none ignored 15.6, 13.9, 16.2 (16.5, 14.5,
    // 17.0). The launch also takes 2.5 us of the host's time.
    a.few = (int64_t)a.T * a.d <= (1 << 18);
    a.tries = wait_limit(kTries);
    DPB_CHECK(make_map(&a.hidden, hidden->data, hidden->stride, c->tokens, c->dim, 64));
    DPB_CHECK(make_map(&a.closed, a.closed_rows, c->dim, c->tokens, c->dim, 64));
    DPB_CHECK(make_map(&a.weight, weight->data, weight->stride, c->vocab, c->dim, 64));
    if (c->index_bytes == 4)
        prepare_kernel<<<kPrepareBlocks, 1024, 0, s>>>(a, static_cast<const int32_t *>(targets), c->ignore_index, grad, c->grad_stride, lse);
    else
        prepare_kernel<<<kPrepareBlocks, 1024, 0, s>>>(a, static_cast<const int64_t *>(targets), c->ignore_index, grad, c->grad_stride, lse);
    DPB_CHECK(launch_status(cudaGetLastError(), "linear_cross_entropy (tokens)"));
    if (a.few) return DPB_OK;
    const unsigned blocks = (unsigned)std::min<int64_t>((c->tokens + 7) / 8, 1216);
    return launch_status(launch_early(gather_kernel, dim3(blocks), 256, 0, s, a), "linear_cross_entropy (rows)");
}

}  // namespace
}  // namespace dpb

using namespace dpb;

extern "C" {

dpb_status dpb_linear_cross_entropy_workspace_size(const dpb_linear_loss_config *cfg, int32_t backward, size_t *bytes) {
    DPB_CHECK(check_config(cfg));
    if (!bytes) return fail(DPB_ERR_INVALID_ARG, "bytes is NULL");
    *bytes = Space(cfg, backward != 0).bytes;
    return DPB_OK;
}

dpb_status dpb_linear_cross_entropy_forward(const dpb_linear_loss_config *cfg, const dpb_rows *hidden,
                                            const dpb_rows *weight, const void *targets, float *loss, float *lse,
                                            int32_t *counted, void *workspace, size_t workspace_bytes, void *stream) {
    DPB_CHECK(check_config(cfg));
    if (counted) DPB_CHECK(need(counted, "counted", 4));
    if (cfg->tokens == 0) {
        if (!counted) return DPB_OK;
        return launch_status(cudaMemsetAsync(counted, 0, 4, static_cast<cudaStream_t>(stream)), "linear_cross_entropy");
    }
    DPB_CHECK(check_rows(hidden, "hidden", cfg->tokens, cfg->dim));
    DPB_CHECK(check_rows(weight, "weight", cfg->vocab, cfg->dim));
    DPB_CHECK(need(targets, "targets", cfg->index_bytes));
    DPB_CHECK(need(loss, "loss", 4));
    DPB_CHECK(need(lse, "lse", 4));
    const Space w(cfg, false);
    Args a{};
    DPB_CHECK(place_status(cfg->status_slot, workspace, workspace_bytes, w.bytes, &a.status));
    uint8_t *ws = static_cast<uint8_t *>(workspace);
    const cudaStream_t s = static_cast<cudaStream_t>(stream);
    a.loss = loss;
    a.lse = lse;
    a.counted = counted;
    a.part = reinterpret_cast<float2 *>(ws + w.part);
    a.z_target = reinterpret_cast<float *>(ws + w.z_target);
    a.z_exact = reinterpret_cast<float *>(ws + w.z_exact);
    // Of rows of up to 256 columns the tensor cores' sums have 16 steps at most: the loss is off by 1e-7 with either
    // (200 columns: 9.8e-8 and 8.3e-8 of the batch's norm; 792: 1.8e-6 and 8e-7 of a small loss). Beside the products it
    // costs nothing where a block's rows take them longer (8192 words and 2^24 values of the weight at least: 33 tokens
    // of 50257 words 36.5 us; 39 in join_kernel); the others' rows are short work for join_kernel (4096 tokens, 1000
    // words, 768 columns: 1 us).
    a.exact = cfg->dim <= 256 ? kAsMultiplied : cfg->vocab >= (1 << 13) && (int64_t)cfg->vocab * cfg->dim >= (1 << 24) ? kBeside : kInJoin;
    DPB_CHECK(begin(a, w, cfg, hidden, weight, targets, nullptr, nullptr, ws, s));
    DPB_CHECK(launch_products(a, w.T_pad / kTile * ((cfg->vocab + kTile - 1) / kTile), s));
    return launch_status(launch_early(join_kernel, dim3((unsigned)((cfg->tokens + 31) / 32)), 1024, 0, s, a),
                         "linear_cross_entropy (rows' sums)");
}

dpb_status dpb_linear_cross_entropy_backward(const dpb_linear_loss_config *cfg, const dpb_rows *hidden,
                                             const dpb_rows *weight, const void *targets, const float *lse,
                                             const float *grad_loss, const dpb_rows *grad_hidden,
                                             const dpb_rows *grad_weight, void *workspace, size_t workspace_bytes,
                                             void *stream) {
    DPB_CHECK(check_config(cfg));
    const cudaStream_t s = static_cast<cudaStream_t>(stream);
    if (grad_weight) DPB_CHECK(check_rows(grad_weight, "grad_weight", cfg->vocab, cfg->dim));
    if (cfg->tokens == 0) {
        if (!grad_weight) return DPB_OK;
        return launch_status(cudaMemset2DAsync(grad_weight->data, (cfg->vocab > 1 ? grad_weight->stride : cfg->dim) * 2ll, 0,
                                               cfg->dim * 2ll, cfg->vocab, s),
                             "linear_cross_entropy_backward");
    }
    DPB_CHECK(check_rows(hidden, "hidden", cfg->tokens, cfg->dim));
    DPB_CHECK(check_rows(weight, "weight", cfg->vocab, cfg->dim));
    if (grad_hidden) DPB_CHECK(check_rows(grad_hidden, "grad_hidden", cfg->tokens, cfg->dim));
    DPB_CHECK(need(targets, "targets", cfg->index_bytes));
    DPB_CHECK(need(lse, "lse", 4));
    DPB_CHECK(need(grad_loss, "grad_loss", 4));
    const Space w(cfg, true);
    Args a{};
    DPB_CHECK(place_status(cfg->status_slot, workspace, workspace_bytes, w.bytes, &a.status));
    if (!grad_hidden && !grad_weight) return DPB_OK;
    uint8_t *ws = static_cast<uint8_t *>(workspace);
    a.want_h = grad_hidden != nullptr;
    a.want_w = grad_weight != nullptr;
    if (grad_hidden) a.dh = static_cast<bf16 *>(grad_hidden->data), a.dh_stride = grad_hidden->stride;
    if (grad_weight) a.dw_rows = static_cast<bf16 *>(grad_weight->data), a.dw_stride = grad_weight->stride;
    if (grad_weight) DPB_CHECK(make_map(&a.dw, grad_weight->data, grad_weight->stride, cfg->vocab, cfg->dim, 32));
    a.rest = reinterpret_cast<float *>(ws + w.rest);
    a.acc = reinterpret_cast<float *>(ws + w.acc);
    if (w.pieces > 1)
        DPB_CHECK(make_map(&a.sums, a.acc, cfg->dim, w.split ? w.pieces * w.T_pad : cfg->tokens, cfg->dim, 32, true));
    a.w_acc = reinterpret_cast<float *>(ws + w.w_acc);
    if (w.parts > 1) DPB_CHECK(make_map(&a.w_sums, a.w_acc, cfg->dim, w.parts * w.V_pad, cfg->dim, 32, true));
    const int64_t rows = w.T_pad * (w.fine ? 2 : 1);
    DPB_CHECK(make_map(&a.dz, ws + w.dz, w.columns, rows, w.columns, 64));
    DPB_CHECK(make_map(&a.dz_out, ws + w.dz, w.columns, rows, w.columns, 32));
    DPB_CHECK(begin(a, w, cfg, hidden, weight, targets, grad_loss, lse, ws, s));
    const int64_t tiles_m = w.T_pad / kTile, tiles_v = (cfg->vocab + kTile - 1) / kTile, tiles_d = (cfg->dim + kTile - 1) / kTile;
    DPB_CHECK(launch_products(a, tiles_m * tiles_v + tiles_v * tiles_d * w.parts, s));
    const int64_t apart = (w.split && grad_hidden ? cfg->tokens : 0) + (w.parts > 1 && grad_weight ? cfg->vocab : 0);
    if (apart == 0) return DPB_OK;
    // as for both gradients, so that one alone has the same bits
    const int64_t outputs = apart * (cfg->dim / 4), both = ((w.split ? cfg->tokens : 0) + (w.parts > 1 ? cfg->vocab : 0)) * (cfg->dim / 4);
    int slices = 1;
    while (slices < kJoinWarps && both * 2 * slices <= (1 << 18)) slices *= 2;
    const unsigned blocks = (unsigned)std::min<int64_t>((outputs * slices + 32 * kJoinWarps - 1) / (32 * kJoinWarps), 8 * sms_of_device());
    return launch_status(launch_early(join_sums_kernel, dim3(blocks), 32 * kJoinWarps, 0, s, a, slices), "linear_cross_entropy_backward (sums)");
}

}  // extern "C"
