// dpb_attention.cu -- softmax attention over packed sequences and its
// gradient, on the tcgen05 tensor cores.
//
// Both kernels have one shape. A block holds 128-row tiles of one side (queries
// in the forward and in the query gradient, keys in the key and value gradient)
// and streams blocks of 128 rows of the other side past them; nothing of size
// queries x keys is ever in memory. Warps have roles: one copies tiles by
// tensor maps into a ring of slots, one or two threads issue the matrix
// products, and warpgroups do the arithmetic, a row of a tile to a thread (or
// to one thread of each warpgroup, which then share its columns). A product's
// result comes from TMEM by rows; the probabilities (and their gradients) go
// back to TMEM in bf16, where the next product takes them as its A operand
// without a pass through shared memory:
//   forward         S = Q K^T;  O += P V
//   query gradient  S = Q K^T, dP = dO V^T;  dQ += dS K
//   key gradient    S^T = K Q^T, dP^T = V dO^T;  dV += P^T dO, dK += dS^T Q
// The gradient takes seven products where five would do with one pass that
// added its dQ shares in memory: each result then has one owner, so sums are
// in a fixed order and no fp32 copy of dQ is kept.
//
// Scores, sums and the statistics of a row are fp32. P and dS are rounded to
// bf16, because that is what the tensor cores take; what they are summed into
// is fp32 again, and each result is rounded once when it is written.
//
// Rows of a neighbouring sequence that a tile's box reaches into are set to
// zero in shared memory where a product would sum over them (0 x NaN), and
// masked by comparison elsewhere.
#include <cuda_bf16.h>
#include <cudaTypedefs.h>

#include <algorithm>
#include <cmath>
#include <cstring>

#include "dpb_checks.h"
#include "dpb_device.cuh"
#include "dpb_tensor_core.cuh"

namespace dpb {
namespace {

using namespace tc;
using bf16 = __nv_bfloat16;

constexpr uint32_t kTries = 1u << 20;  // polls of a wait before it gives up
constexpr int kRows = 128;             // rows of a tile (M of the products)
constexpr int kMostWarps = 16;         // row warps of a gradient block, at most
constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;

struct Out {
    bf16 *p;
    int64_t ts, hs;
};
struct In {
    const bf16 *p;
    int64_t ts, hs;
};

struct AttnArgs {
    CUtensorMap q, k, v, g;  // g: grad_o
    const int32_t *cu_q, *cu_k;
    int64_t total_q, total_k;
    int seqs, max_q, max_k, hq, hkv, group, D, causal, tiles, close;
    int items;            // blocks of the forward's grid for the sequences
    float scale, scale2;  // scale, and scale x log2 e
    In o, go;
    Out out, dq, dk, dv;
    float *lse;
    float *delta;
    struct Plan *plan;  // of the gradient
    struct Task *tasks_k, *tasks_q;
    int64_t cap_k, cap_q;
    int *arrived;  // [slots][row warps]
    float *parts;  // [slots][128][2 DP]
    int slots, sms;
    int32_t *status;
};

// One sequence: its tokens [q0, q0 + n) and [k0, k0 + m). Loading its offsets
// and looking at them are apart, so that a block's set-up runs meanwhile.
struct Offsets {
    int64_t q0, q1, k0, k1;
};
struct Seq {
    int q0, n, k0, m;
    bool ok;
};

__device__ __forceinline__ Offsets load_offsets(const AttnArgs &a, int s) {
    Offsets r{0, a.total_q, 0, a.total_k};
    if (a.cu_q) {
        r.q0 = __ldg(a.cu_q + s), r.q1 = __ldg(a.cu_q + s + 1);
        r.k0 = __ldg(a.cu_k + s), r.k1 = __ldg(a.cu_k + s + 1);
    }
    return r;
}
__device__ __forceinline__ Seq sequence(const AttnArgs &a, const Offsets &o) {
    Seq r;
    r.ok = o.q0 >= 0 && o.q1 >= o.q0 && o.q1 <= a.total_q && o.k0 >= 0 && o.k1 >= o.k0 && o.k1 <= a.total_k &&
           o.q1 - o.q0 <= a.max_q && o.k1 - o.k0 <= a.max_k;
    r.q0 = (int)o.q0, r.n = (int)(o.q1 - o.q0), r.k0 = (int)o.k0, r.m = (int)(o.k1 - o.k0);
    return r;
}
// Sequence s, -1 <= s <= seqs, where -1 and seqs stand for the rows before the
// first and after the last. What is no sound sequence (not ok) has the rows that
// its offsets pass on the way up, which see nothing and are seen by none: from
// the first token to the last such a way passes every row, so each is a sound
// sequence's or one of these.
__device__ __forceinline__ Seq rows_of(const AttnArgs &a, int s) {
    Offsets o{0, a.total_q, 0, a.total_k};
    if (a.cu_q) {  // four loads at once, whatever s is
        const int i = max(s, 0), j = min(s + 1, a.seqs);
        o.q0 = __ldg(a.cu_q + i), o.q1 = __ldg(a.cu_q + j);
        o.k0 = __ldg(a.cu_k + i), o.k1 = __ldg(a.cu_k + j);
    } else if (s < 0) {
        o.q1 = o.k1 = 0;
    } else if (s > 0) {
        o.q0 = a.total_q, o.k0 = a.total_k;
    }
    if (s < 0) o.q0 = o.k0 = 0;
    if (s >= a.seqs) o.q1 = a.total_q, o.k1 = a.total_k;
    Seq r = sequence(a, o);
    const bool is = s >= 0 && s < a.seqs;
    if (is && !r.ok) set_status(a.status, DPB_DEV_BAD_LENGTH);
    r.ok = r.ok && is;
    if (!r.ok) {
        r.q0 = (int)max((int64_t)0, o.q0), r.n = (int)max((int64_t)0, min(o.q1, a.total_q) - r.q0);
        r.k0 = (int)max((int64_t)0, o.k0), r.m = (int)max((int64_t)0, min(o.k1, a.total_k) - r.k0);
    }
    return r;
}

// A tile of `rows` rows of one head: DP / 64 boxes of 64 columns.
template <int DP>
__device__ __forceinline__ void copy_tile(uint32_t dst, const CUtensorMap *map, int head, int token, int rows,
                                          uint32_t bar) {
#pragma unroll
    for (int h = 0; h < DP / 64; ++h) copy_box(dst + h * rows * 128, map, 64 * h, head, token, bar);
}

// Zeroes rows [from, rows) of a tile. One warp.
template <int DP>
__device__ __forceinline__ void zero_rows(uint8_t *tile, int from, int rows) {
    const int lane = threadIdx.x & 31;
    for (int h = 0; h < DP / 64; ++h)
        for (int i = from * 8 + lane; i < rows * 8; i += 32)
            *reinterpret_cast<uint4 *>(tile + h * rows * 128 + i * 16) = make_uint4(0u, 0u, 0u, 0u);
}

// The ring of slots that the copying warp fills and the products empty. Tile i
// uses one of N slots for the (i / N)-th time: slot i % N, or with SWAP (four
// slots, tiles in pairs) pairs take turns on two slots each and exchange them
// within the pair from one turn to the next: of a pair, the second tile is
// done with first, so the first tile of the pair two further on, which is
// wanted first, gets its slot.
template <int N, int BYTES, bool SWAP = false>
struct Ring {
    static_assert(!SWAP || N == 4, "pairs of tiles in four slots");
    uint8_t *data;
    uint32_t full, empty, tail;  // full[N], empty[N], tail
    __device__ __forceinline__ int index(int i) const {
        if (SWAP) return (i & 2) | ((i ^ (i >> 2)) & 1);
        return i % N;
    }
    __device__ __forceinline__ uint32_t full_bar(int i) const { return full + 8 * index(i); }
    __device__ __forceinline__ uint32_t empty_bar(int i) const { return empty + 8 * index(i); }
    __device__ __forceinline__ uint32_t parity(int i) const { return (i / N) & 1; }
    __device__ __forceinline__ bool wait_full(int i) const { return bar_wait(full_bar(i), parity(i), kTries); }
    __device__ __forceinline__ uint8_t *slot(int i) const { return data + index(i) * BYTES; }
    __device__ __forceinline__ uint32_t addr(int i) const { return smem_addr(slot(i)); }
    // All lanes: slot i is free (its previous products are done).
    __device__ __forceinline__ bool wait_free(int i) const {
        return i < N || __all_sync(kFull, bar_wait(empty_bar(i), parity(i) ^ 1, kTries));
    }
    // All lanes: copies rows [token, token + rows) of a head into slot i; where
    // only `live` of them belong to the sequence (and `sums`: a product sums
    // over them), the others are zeroed before the slot counts as full.
    template <int DP>
    __device__ __forceinline__ bool fill(int i, const CUtensorMap *map, int head, int token, int rows, int live,
                                         bool sums, int &tails) const {
        if (!sums || live >= rows) {
            if (elect_one()) {
                bar_arrive_expect(full_bar(i), BYTES);
                copy_tile<DP>(addr(i), map, head, token, rows, full_bar(i));
            }
            __syncwarp();
            return true;
        }
        if (elect_one()) {
            bar_arrive_expect(tail, BYTES);
            copy_tile<DP>(addr(i), map, head, token, rows, tail);
        }
        __syncwarp();
        const bool ok = __all_sync(kFull, bar_wait(tail, tails & 1, kTries));
        ++tails;
        if (!ok) return false;
        zero_rows<DP>(slot(i), live, rows);
        fence_async_shared();
        __syncwarp();
        if (elect_one()) bar_arrive(full_bar(i));
        __syncwarp();
        return true;
    }
    // After a wait that gave up: every copy issued so far has landed (tiles
    // [0, issued); bounded).
    __device__ __forceinline__ void drain(int issued) const {
        for (int i = max(0, issued - N); i < issued; ++i) bar_wait(full_bar(i), parity(i), kTries);
    }
};

__device__ __forceinline__ void write_zero_row(bf16 *row, int D) {
    for (int i = 0; i < D; i += 8) *reinterpret_cast<uint4 *>(row + i) = make_uint4(0u, 0u, 0u, 0u);
}

// Writes 32 columns [at, at + 32) of this warp's 32 rows of a result from
// `stage` (32 rows of 64 bytes, the 16-byte pieces of each exchanged so that
// neither side meets bank conflicts), so that a store covers whole stretches
// of rows. Rows from `rows` on, and columns from D on, are left out.
__device__ __forceinline__ uint8_t *stage_piece(uint8_t *stage, int row, int i) {
    return stage + row * 64 + ((i ^ ((row >> 1) & 3)) * 16);
}
__device__ __forceinline__ void write_stage(uint8_t *stage, const Out &out, int64_t token, int head, int rows, int at,
                                            int D) {
    const int lane = threadIdx.x & 31, piece = lane & 3, r0 = lane >> 2;
    __syncwarp();
    uint4 x[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) x[i] = *reinterpret_cast<const uint4 *>(stage_piece(stage, r0 + 8 * i, piece));
    if (at + 8 * piece < D)
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (r0 + 8 * i < rows)
                *reinterpret_cast<uint4 *>(out.p + (token + r0 + 8 * i) * out.ts + head * out.hs + at + 8 * piece) = x[i];
    __syncwarp();
}
// The same of CH x 32 columns from TMEM (fp32, times f) to columns from `col`
// on, as bf16. read() is called once TMEM has been read.
template <int CH, typename F>
__device__ __forceinline__ void write_rows(uint32_t tmem, uint8_t *stage, const Out &out, int64_t token, int head,
                                           int rows, int col, int D, float f, F read) {
    const int lane = threadIdx.x & 31;
    uint32_t u[CH][16];
#pragma unroll
    for (int c = 0; c < CH; ++c) {
        uint32_t v[32];
        tmem_load(tmem + 32 * c, v);
        load_wait(v);
#pragma unroll
        for (int e = 0; e < 16; ++e)
            u[c][e] = pack_bf16(__uint_as_float(v[2 * e]) * f, __uint_as_float(v[2 * e + 1]) * f);
    }
    read();
#pragma unroll
    for (int c = 0; c < CH; ++c) {
#pragma unroll
        for (int i = 0; i < 4; ++i)
            *reinterpret_cast<uint4 *>(stage_piece(stage, lane, i)) =
                make_uint4(u[c][4 * i], u[c][4 * i + 1], u[c][4 * i + 2], u[c][4 * i + 3]);
        write_stage(stage, out, token, head, rows, col + 32 * c, D);
    }
}

// The block's set-up: the copying warp makes the barriers and goes on at once
// (its first copies are under way while TMEM is allocated); the others wait.
template <int THREADS>
__device__ __forceinline__ void setup_arrive() {
    asm volatile("barrier.cta.arrive 1, %0;" ::"n"(THREADS) : "memory");
}
template <int THREADS>
__device__ __forceinline__ void setup_wait() {
    asm volatile("barrier.cta.sync 1, %0;" ::"n"(THREADS) : "memory");
}

// What a block takes on: a tile of keys, one (or in the forward a pair) of
// queries, or the end.
enum { kKeys, kQueries, kEnd };
struct Item {
    int kind, head, tile, first, count, pieces, slot, piece;
    Seq q;
};

// The items that the copying warp of a block hands on to the others.
template <int N>
struct ItemList {
    int4 *data;
    uint32_t full, free;  // barriers [N]: item is there, has been read by all
    __device__ __forceinline__ void read(Item &it, int c) const {
        const int4 *at = data + 3 * (c % N), x = at[0], y = at[1], z = at[2];
        it.q.q0 = x.x, it.q.n = x.y, it.q.k0 = x.z, it.q.m = x.w;
        it.tile = y.x, it.first = y.y, it.count = y.z, it.pieces = y.w;
        it.slot = z.x, it.piece = z.y, it.kind = z.z, it.head = z.w;
    }
    // All lanes of the copying warp: hands on item c.
    __device__ __forceinline__ bool put(const Item &it, int c) const {
        const int at = c % N;
        if (c >= N && !__all_sync(kFull, bar_wait(free + 8 * at, ((c / N) & 1) ^ 1, kTries))) return false;
        if (elect_one()) {
            data[3 * at] = make_int4(it.q.q0, it.q.n, it.q.k0, it.q.m);
            data[3 * at + 1] = make_int4(it.tile, it.first, it.count, it.pieces);
            data[3 * at + 2] = make_int4(it.slot, it.piece, it.kind, it.head);
            bar_arrive(full + 8 * at);
        }
        __syncwarp();
        return true;
    }
    // One thread: takes item c.
    __device__ __forceinline__ bool get_one(Item &it, int &c) const {
        if (!bar_wait(full + 8 * (c % N), (c / N) & 1, kTries)) return false;
        read(it, c);
        bar_arrive(free + 8 * (c % N));
        ++c;
        return true;
    }
    // All lanes of a warp: takes item c, which stays in the list until the warp
    // has finished it.
    __device__ __forceinline__ bool get_warp(Item &it, int &c) const {
        if (!__all_sync(kFull, bar_wait(full + 8 * (c % N), (c / N) & 1, kTries))) return false;
        read(it, c);
        ++c;
        return true;
    }
    __device__ __forceinline__ void finished(int c) const {
        __syncwarp();
        if ((threadIdx.x & 31) == 0) bar_arrive(free + 8 * (c % N));
    }
};

// ---- forward ------------------------------------------------------------------

template <int DP_, int BN_, int NS_>
struct FwdShape {
    static constexpr int DP = DP_, BN = BN_, NS = NS_;
    // P has columns of its own where there is room beside S and O: the next S
    // is then computed as soon as this one has been read. Otherwise P takes
    // the place of S, and the next S comes after its product.
    static constexpr bool kOwnP = 2 * (BN + DP + BN / 2) <= 512;
    static constexpr int kTile = kRows * DP * 2, kSlot = BN * DP * 2;
    static constexpr int kColumns = 512;
    static constexpr int kColO = 2 * BN, kColP = kOwnP ? 2 * (BN + DP) : 0, kStepP = kOwnP ? BN / 2 : BN;
    static constexpr int kItems = 4, kReaders = kOwnP ? 10 : 9;  // of the list of items
    static constexpr int kBars = 4 + 2 * NS + 1 + 7 + 8 + 2 * kItems + 1;
    static constexpr int kStage = 32 * 32 * 2;  // a warp's rows of 32 result columns
    static constexpr int kSmem = 1024 + 2 * kTile + NS * kSlot + 8 * kStage + 48 * kItems + 16 + 8 * kBars + 16;
    static constexpr int kThreads = 384;  // two softmax warpgroups, one of the copying and the issuing warp
    // registers of a softmax thread and of the others: 256 x 208 + 128 x 88 = 384 x 168
    static constexpr int kRegsRow = 208, kRegsOther = 88;
};

// Visible keys of query row i (of n, against m keys).
__device__ __forceinline__ int visible(const AttnArgs &a, const Seq &q, int i) {
    return a.causal ? max(0, min(q.m, i + (q.m - q.n) + 1)) : q.m;
}

// Blocks of BN keys that query tile `tile` has to see (0 where it has no rows).
template <int BN>
__device__ __forceinline__ int tile_blocks(const AttnArgs &a, const Seq &q, int tile) {
    const int r0 = tile * kRows;
    return r0 < q.n ? (visible(a, q, min(r0 + kRows, q.n) - 1) + BN - 1) / BN : 0;
}

__device__ __forceinline__ int pairs_of(const Seq &q) { return (q.n + 2 * kRows - 1) / (2 * kRows); }

// The place-th pair of tiles of queries of all sequences in turn, the last of
// each first, or false after all of them. All lanes of a warp, which look at 32
// sequences at a time from where they left off (places mostly grow).
struct Finder {
    int first, before;  // sequence that lane 0 looks at, pairs before it
    __device__ __forceinline__ bool find(const AttnArgs &a, int place, int &seq, int &tile) {
        const int lane = threadIdx.x & 31;
        if (place < before) first = before = 0;
        for (; first < a.seqs; first += 32) {
            const int s = first + lane;
            Seq q{0, 0, 0, 0, false};
            if (s < a.seqs) q = rows_of(a, s);
            const int pairs = pairs_of(q);
            int upto = pairs;
#pragma unroll
            for (int o = 1; o < 32; o *= 2) {
                const int x = __shfl_up_sync(kFull, upto, o);
                if (lane >= o) upto += x;
            }
            const uint32_t past = __ballot_sync(kFull, before + upto > place);
            if (past) {
                const int at = __ffs(past) - 1;
                seq = first + at;
                tile = before + __shfl_sync(kFull, upto, at) - 1 - place;
                return true;
            }
            before += __shfl_sync(kFull, upto, 31);
        }
        return false;
    }
};

// Blocks stay: one that has copied all of an item asks the hardware for a block of
// the grid that has not started, and takes its item (of those that have rows)
// over, so that copies and first products of the next item run while this one
// is being finished.
//
// Measured (causal; 4 x visible pairs x head_dim operations a head), against a
// block for each item: 1 x 12289, 12 heads of 64: 213 us (222), 1087 TFLOP/s;
// 8 x 1024, 12 heads of 64: 26.7 us (29.9); 1 x 8192, 16 heads of 128: 191 us
// (191), 1440 TFLOP/s; 8 x 1024, 16 heads of 128: 45 us (50.7). At 128 bound by
// the tensor cores. At 64 a block of scores takes 1170 cycles, of them 512 of
// exponentials (32 a cycle) and some 590 of products: the row warps' chain from
// one to the other (2.0 instructions a cycle, of 4) is what is left. Short
// sequences are bound by the way of an item's first block from memory to its
// result.
template <class C>
__global__ void __launch_bounds__(C::kThreads, 1) attention_forward_kernel(const __grid_constant__ AttnArgs a) {
    constexpr int DP = C::DP, BN = C::BN;
    constexpr int kCopier = 8, kScores = 9, kValues = C::kOwnP ? 10 : 9;  // warps
    extern __shared__ uint8_t smem_raw[];
    uint8_t *smem = smem_raw + ((1024 - (smem_addr(smem_raw) & 1023)) & 1023);
    const int warp = threadIdx.x / 32, lane = threadIdx.x & 31;

    uint8_t *stages = smem + 2 * C::kTile + C::NS * C::kSlot;
    int4 *items = reinterpret_cast<int4 *>(stages + 8 * C::kStage);
    const uint32_t answer = smem_addr(items + 3 * C::kItems);
    uint64_t *bars = reinterpret_cast<uint64_t *>(items + 3 * C::kItems + 1);
    const uint32_t bar0 = smem_addr(bars);
    // of each tile of queries: it is there, has been used for the last time
    const uint32_t q_full = bar0, q_free = q_full + 16;
    Ring<C::NS, C::kSlot> ring{smem + 2 * C::kTile, bar0 + 32, bar0 + 32 + 8 * C::NS, bar0 + 32 + 16 * C::NS};
    // per tile: S is there, O is done, P's product is done; all is done; by the
    // row warps: each half of P is there, S has been read, O has been read; an
    // item is there, has been read; the hardware has answered
    const uint32_t s_full = bar0 + 8 * (5 + 2 * C::NS), o_full = s_full + 16, p_done = o_full + 16, done = p_done + 16,
                   p_full = done + 8, s_read = p_full + 32, o_free = s_read + 16, item_full = o_free + 16,
                   answered = item_full + 16 * C::kItems;
    const ItemList<C::kItems> list{items, item_full, item_full + 8 * C::kItems};
    uint32_t *slot = reinterpret_cast<uint32_t *>(bars + C::kBars);
    Item it;
    bool failed = false;
    int c = 0;  // items taken

    if (warp >= 8) {
        give_registers<C::kRegsOther>();
        if (warp == kCopier) {
            for (int i = lane; i < C::kBars; i += 32) {
                const uint32_t b = bar0 + 8 * i;
                bar_init(b, b == answered                       ? 1
                            : b >= list.free                    ? C::kReaders
                            : b >= item_full                    ? 1
                            : b >= p_full                       ? 4
                            : b == done && kValues != kScores ? 2
                                                                : 1);
            }
            bar_init_fence();
            __syncwarp();
            setup_arrive<C::kThreads>();
            // ring's tiles copied, answers had, copies of each of the two tiles
            int i = 0, tails = 0, asked = 0, sent0 = 0, sent1 = 0;
            uint32_t at = blockIdx.x;
            bool have = true;
            Finder finder{0, 0};
            // The last blocks of the grid, and those of skipped sequences, have rows of no
            // sound sequence: which (a sequence, or -1 and seqs as for rows_of) and their
            // next pair of tiles (and, of those before and after the sequences, head).
            // `at` goes on beyond the grid's sequences (over) where ones that overlap have
            // more pairs of tiles than it counts.
            constexpr int kNone = -2;
            int rests = kNone, piece = 0;
            bool over = false;
            // takes over a block that has not started, if there is one
            auto next = [&]() {
                if (elect_one()) {
                    bar_arrive_expect(answered, 16);
                    ask_block(answer, answered);
                }
                __syncwarp();
                failed = !__all_sync(kFull, bar_wait(answered, asked & 1, kTries));
                ++asked;
                have = !failed && block_answer(answer, at);
                over = false;
                fence_async_shared();
                __syncwarp();
            };
            for (;;) {
                it = Item{};
                it.kind = kEnd;
                while (have) {
                    it.head = (int)(at % a.hq);
                    // the usual way stays together (cold code costs the training step 3 us)
                    if (__builtin_expect(rests == kNone && (at < (uint32_t)a.items || over), 1)) {
                        // the heads of a group side by side; the longest rows first, or
                        // sequence by sequence
                        const int rest = (int)(at / a.hq);
                        int seq = rest % a.seqs;
                        it.tile = a.tiles - 1 - rest / a.seqs;
                        if (a.close && !finder.find(a, rest, seq, it.tile)) {
                            next();
                            continue;
                        }
                        it.q = sequence(a, load_offsets(a, seq));
                        if (__builtin_expect(it.q.ok, 1)) {
                            if (it.tile * 2 * kRows < it.q.n) {
                                it.kind = kQueries;
                                break;
                            }
                            next();
                            continue;
                        }
                        rests = seq, piece = it.tile;
                    } else if (rests == kNone) {
                        rests = -1, piece = (int)at - a.items;
                    }
                    const bool outside = rests < 0 || rests >= a.seqs;
                    it.tile = piece;
                    if (outside) it.head = piece % a.hq, it.tile = piece / a.hq;
                    it.q = rows_of(a, rests);
                    const int pairs = pairs_of(it.q);
                    if (it.tile < pairs) {
                        // a skipped sequence's further pairs: as far on as any sound one has
                        // them, or as the finder says
                        piece = outside ? piece + (int)gridDim.x - a.items : a.close ? 0x7fffffff : piece + a.tiles;
                        it.q.m = 0;
                        it.kind = kQueries;
                        break;
                    }
                    if (rests < 0) {
                        rests = a.seqs, piece -= pairs * a.hq;
                    } else {
                        rests = kNone;
                        if (outside && a.close) over = true;
                        else if (over) at += gridDim.x - a.items;
                        else next();
                    }
                }
                failed = failed || !list.put(it, c);
                if (failed || it.kind == kEnd) break;
                ++c;
                const Seq &q = it.q;
                it.count = max(tile_blocks<BN>(a, q, 2 * it.tile), tile_blocks<BN>(a, q, 2 * it.tile + 1));
                const int kv_head = it.head / a.group;
                auto queries = [&](int t, int &sent) {
                    if (failed || (2 * it.tile + t) * kRows >= q.n) return;
                    failed = sent > 0 && !__all_sync(kFull, bar_wait(q_free + 8 * t, (sent - 1) & 1, kTries));
                    if (failed) return;
                    ++sent;
                    if (elect_one()) {
                        bar_arrive_expect(q_full + 8 * t, C::kTile);
                        copy_tile<DP>(smem_addr(smem) + t * C::kTile, &a.q, it.head, q.q0 + (2 * it.tile + t) * kRows,
                                      kRows, q_full + 8 * t);
                    }
                    __syncwarp();
                };
                auto block = [&](int j, bool values) {
                    failed = failed || !ring.wait_free(i) ||
                             !ring.template fill<DP>(i, values ? &a.v : &a.k, kv_head, q.k0 + j * BN, BN, q.m - j * BN,
                                                     values, tails);
                    if (!failed) ++i;
                };
                if (it.count > 0) {
                    // what the first products need first
                    queries(0, sent0);
                    block(0, false);
                    queries(1, sent1);
                    block(0, true);
                    for (int j = 1; j < it.count && !failed; ++j) {
                        block(j, false);
                        block(j, true);
                    }
                }
                if (failed) break;
                if (over && rests == kNone) at += gridDim.x - a.items;
                else if (rests == kNone) next();
            }
            // no copy is in flight when the block ends, whatever gave up
            ring.drain(i);
            if (sent0 > 0) bar_wait(q_full, (sent0 - 1) & 1, kTries);
            if (sent1 > 0) bar_wait(q_full + 8, (sent1 - 1) & 1, kTries);
        } else {
            if (warp == kScores) tmem_alloc(smem_addr(slot), C::kColumns);
            fence_before();
            setup_wait<C::kThreads>();
            fence_after();
            const uint32_t tmem = *slot;
            const uint32_t q_addr = smem_addr(smem);
            // bit t of each: whether the blocks, items with blocks and copies of
            // tile t so far are odd in number (a barrier that has not been used
            // counts as past the odd phase before)
            uint32_t b = 0, o = 0, sent = 0;
            int base = 0;  // ring's tiles
            auto odd = [](uint32_t bits, int t) { return (bits >> t) & 1; };
            auto scores = [&](int t, int i) {
                fence_after();
                const uint64_t kd = desc_k_inside(ring.addr(i)), qd = desc_k_inside(q_addr + t * C::kTile);
#pragma unroll
                for (int k = 0; k < DP / 16; ++k)
                    mma_ss(tmem + t * BN, desc_at(qd, (k / 4) * kRows * 128 + (k % 4) * 32),
                           desc_at(kd, (k / 4) * BN * 128 + (k % 4) * 32), mma_shape(BN, false), k > 0);
                mma_commit(s_full + 8 * t);
            };
            // O += P V of tile t, each half of the keys as soon as its P is
            // there; O's place is free once the sums of the item before are read
            auto values = [&](int t, int i, bool first) {
                if (first && !bar_wait(o_free + 8 * t, odd(o, t) ^ 1, kTries)) return false;
                const uint64_t vd = desc_k_rows(ring.addr(i), BN * 128);
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    if (!bar_wait(p_full + 16 * t + 8 * h, odd(b, t), kTries)) return false;
                    fence_after();
#pragma unroll
                    for (int k = h * BN / 32; k < (h + 1) * BN / 32; ++k)
                        mma_ts(tmem + C::kColO + t * DP, tmem + C::kColP + t * C::kStepP + 8 * k,
                               desc_at(vd, k * 2048), mma_shape(DP, true), !first || k > 0);
                }
                b ^= 1u << t;
                return true;
            };
            if (warp == kScores && elect_one()) {
                // ---- scores; where P takes S's place, the values' products too
                for (failed = !list.get_one(it, c); !failed && it.kind != kEnd;
                     failed = failed || !list.get_one(it, c)) {
                    const int nb0 = tile_blocks<BN>(a, it.q, 2 * it.tile), nb1 = tile_blocks<BN>(a, it.q, 2 * it.tile + 1);
                    const int blocks = max(nb0, nb1);
                    if (blocks == 0) continue;
                    const bool rows1 = (2 * it.tile + 1) * kRows < it.q.n;
                    // the first block's, once the tile is there; one with rows is
                    // waited for, even where it has no block
                    failed = !ring.wait_full(base);
                    for (int t = 0; t < 2 && !failed; ++t) {
                        const int nb = t ? nb1 : nb0;
                        if (t && !rows1) break;
                        failed = !bar_wait(q_full + 8 * t, odd(sent, t), kTries);
                        sent ^= 1u << t;
                        if (!failed && nb > 0) {
                            if (C::kOwnP) {
                                failed = !bar_wait(s_read + 8 * t, odd(b, t) ^ 1, kTries);
                                b ^= 1u << t;
                            }
                            if (!failed) scores(t, base);
                        }
                        if (!failed && nb <= 1) mma_commit(q_free + 8 * t);
                    }
                    if (failed) break;
                    mma_commit(ring.empty_bar(base));
                    for (int j = 0; j < blocks && !failed; ++j) {
                        const bool more = j + 1 < blocks;
                        const int k_next = base + 2 * j + 2, v = base + 2 * j + 1;
                        failed = (more && !ring.wait_full(k_next)) || (!C::kOwnP && !ring.wait_full(v));
#pragma unroll 1
                        for (int t = 0; t < 2 && !failed; ++t) {
                            const int left = (t ? nb1 : nb0) - j;  // blocks of the tile, this one included
                            if (left <= 0) continue;
                            if (C::kOwnP) {
                                if (left == 1) continue;
                                failed = !bar_wait(s_read + 8 * t, odd(b, t) ^ 1, kTries);
                                if (failed) break;
                                b ^= 1u << t;
                            } else {
                                failed = !values(t, v, j == 0);
                                if (failed) break;
                                if (left == 1) {
                                    mma_commit(o_full + 8 * t);
                                    o ^= 1u << t;
                                    continue;
                                }
                            }
                            scores(t, k_next);  // with P in S's place: products run in the order of their issue
                            if (left == 2) mma_commit(q_free + 8 * t);
                        }
                        if (failed) break;
                        if (!C::kOwnP) mma_commit(ring.empty_bar(v));
                        if (more) mma_commit(ring.empty_bar(k_next));
                    }
                    base += 2 * blocks;
                }
                // every product, and every arrival that it makes, is done
                // before the block's memory is given back
                mma_commit(done);
                failed |= !bar_wait(done, 0, kTries);
            } else if (C::kOwnP && warp == kValues && elect_one()) {
                // ---- values
                for (failed = !list.get_one(it, c); !failed && it.kind != kEnd;
                     failed = failed || !list.get_one(it, c)) {
                    const int nb0 = tile_blocks<BN>(a, it.q, 2 * it.tile), nb1 = tile_blocks<BN>(a, it.q, 2 * it.tile + 1);
                    const int blocks = max(nb0, nb1);
                    for (int j = 0; j < blocks && !failed; ++j) {
                        const int v = base + 2 * j + 1;
                        failed = !ring.wait_full(v);
#pragma unroll 1
                        for (int t = 0; t < 2 && !failed; ++t) {
                            const int left = (t ? nb1 : nb0) - j;
                            if (left <= 0) continue;
                            failed = !values(t, v, j == 0);
                            if (failed) break;
                            mma_commit(p_done + 8 * t);
                            if (left == 1) {
                                mma_commit(o_full + 8 * t);
                                o ^= 1u << t;
                            }
                        }
                        if (!failed) mma_commit(ring.empty_bar(v));
                    }
                    base += 2 * blocks;
                }
                mma_commit(done);
                failed |= !bar_wait(done, 0, kTries);
            }
            __syncwarp();
        }
    } else {
        take_registers<C::kRegsRow>();
        fence_before();
        setup_wait<C::kThreads>();
        fence_after();
        const uint32_t tmem = *slot;
        // ---- softmax: a row a thread
        const int t = warp / 4;
        const uint32_t lanes = (uint32_t)(warp & 3) << 21;  // this warp's 32 TMEM lanes
        const uint32_t s_addr = tmem + lanes + t * BN, o_addr = tmem + lanes + C::kColO + t * DP;
        const uint32_t p_addr = tmem + lanes + C::kColP + t * C::kStepP;
        const uint64_t scale2 = pair(a.scale2, a.scale2);
        int b = 0, o = 0;  // blocks and items with blocks so far
        for (;;) {
            failed = !list.get_warp(it, c);
            if (failed || it.kind == kEnd) break;
            const int lim = visible(a, it.q, (2 * it.tile + t) * kRows + (threadIdx.x & 127));
            const int nb = tile_blocks<BN>(a, it.q, 2 * it.tile + t);
            float top = 0.f;  // reference maximum, of scale2 S
            uint64_t sum2[2] = {0, 0};  // four shares of the sum of 2^(scale2 S - top)
            for (int j = 0; j < nb; ++j, ++b) {
                if (!__all_sync(kFull, bar_wait(s_full + 8 * t, b & 1, kTries))) {
                    failed = true;
                    break;
                }
                fence_after();
                uint32_t s[BN / 32][32];
#pragma unroll
                for (int c = 0; c < BN / 32; ++c) tmem_load(s_addr + 32 * c, s[c]);
#pragma unroll
                for (int c = 0; c < BN / 32; ++c) load_wait(s[c]);
                if (C::kOwnP) {
                    fence_before();
                    __syncwarp();
                    if (lane == 0) bar_arrive(s_read + 8 * t);
                }
                const int seen = lim - j * BN;  // visible columns of this block
                if (!__all_sync(kFull, seen >= BN)) {
#pragma unroll
                    for (int c = 0; c < BN; ++c)
                        if (c >= seen) s[c / 32][c % 32] = 0xff800000u;  // -inf
                }
                float m[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
#pragma unroll
                for (int c = 0; c < BN; c += 8)
#pragma unroll
                    for (int e = 0; e < 4; ++e)
                        m[e] = max3(m[e], __uint_as_float(s[c / 32][c % 32 + 2 * e]),
                                    __uint_as_float(s[c / 32][c % 32 + 2 * e + 1]));
                const float mx = fmaxf(max3(m[0], m[1], m[2]), m[3]) * a.scale2;
                // this tile's product of the block before has to be done before P
                // is written or O is scaled (with P in place of S, S came after it)
                bool waited = !C::kOwnP || b == 0;
                if (j == 0) {
                    top = mx == -INFINITY ? 0.f : mx;
                } else if (__any_sync(kFull, mx > top + 8.f)) {
                    // The running maximum is only followed when it has grown by a
                    // factor of 2^8: until then the sums stay far from overflow,
                    // and O is not touched.
                    if (!waited) {
                        if (!__all_sync(kFull, bar_wait(p_done + 8 * t, (b - 1) & 1, kTries))) {
                            failed = true;
                            break;
                        }
                        fence_after();
                        waited = true;
                    }
                    const float next = mx > top + 8.f ? mx : top, f = exp2_approx(top - next);
                    top = next;
                    const uint64_t f2 = pair(f, f);
                    sum2[0] = mul2(sum2[0], f2);
                    sum2[1] = mul2(sum2[1], f2);
#pragma unroll 1
                    for (int c = 0; c < DP; c += 32) {
                        uint32_t v[32];
                        tmem_load(o_addr + c, v);
                        load_wait(v);
#pragma unroll
                        for (int e = 0; e < 32; ++e) v[e] = __float_as_uint(__uint_as_float(v[e]) * f);
                        tmem_store(o_addr + c, v);
                    }
                }
                const uint64_t top2 = pair(-top, -top);
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    static_assert(BN == 128, "a half of P is one store of 32 columns");
                    uint32_t p[32];
#pragma unroll
                    for (int e = 0; e < 64; e += 2) {
                        const int x = 64 * h + e;
                        const float2 y = unpair(fma2(pair_bits(s[x / 32][x % 32], s[x / 32][x % 32 + 1]), scale2, top2));
                        const float p0 = exp2_approx(y.x), p1 = exp2_approx(y.y);
                        sum2[(e / 2) & 1] = add2(sum2[(e / 2) & 1], pair(p0, p1));
                        p[e / 2] = pack_bf16(p0, p1);
                    }
                    if (!waited) {
                        if (!__all_sync(kFull, bar_wait(p_done + 8 * t, (b - 1) & 1, kTries))) {
                            failed = true;
                            break;
                        }
                        fence_after();
                        waited = true;
                    }
                    tmem_store(p_addr + 32 * h, p);
                    store_wait();
                    fence_before();
                    __syncwarp();
                    if (lane == 0) bar_arrive(p_full + 16 * t + 8 * h);
                }
                if (failed) break;
            }
            if (failed) break;
            const float2 sums = unpair(add2(sum2[0], sum2[1]));
            const float sum = sums.x + sums.y;
            Item was;  // read anew, so that the loop above need not hold it
            list.read(was, c - 1);
            const int first = (2 * was.tile + t) * kRows + (warp & 3) * 32;  // the warp's first row
            const int64_t token = was.q.q0 + (int64_t)first;
            if (nb > 0) {
                if (!__all_sync(kFull, bar_wait(o_full + 8 * t, o & 1, kTries))) {
                    failed = true;
                    break;
                }
                ++o;
                fence_after();
                write_rows<DP / 32>(o_addr, stages + warp * C::kStage, a.out, token, was.head, was.q.n - first, 0, a.D,
                                    sum > 0.f || sum != sum ? 1.f / sum : 0.f, [&]() {
                                        fence_before();
                                        __syncwarp();
                                        if (lane == 0) bar_arrive(o_free + 8 * t);
                                    });
            } else if (first + lane < was.q.n) {
                write_zero_row(a.out.p + (token + lane) * a.out.ts + was.head * a.out.hs, a.D);
            }
            if (first + lane < was.q.n)
                a.lse[(int64_t)was.head * a.total_q + token + lane] =
                    lim > 0 ? (top + __log2f(sum)) * kLn2 : -INFINITY;
            list.finished(c - 1);
        }
    }
    if (failed) set_status(a.status, DPB_DEV_TIMEOUT);
    fence_before();
    __syncthreads();
    if (warp == kScores) tmem_free(*slot, C::kColumns);
}

// ---- gradients ------------------------------------------------------------------

// One tile of 128 rows against blocks of 128: S and the gradient of P take 256
// TMEM columns, the sums the rest. Warpgroups share a tile's columns. With heads
// of 64 the rows' arithmetic is what bounds a block: four warpgroups of 32
// columns each (a thread's chain from S to dS is short, and four warps on each
// scheduler fill each other's waits): 1 x 12289 causal, 12 heads: 661 us, 708
// with two. With heads of 128 the products are, and two are as good (1 x 8192
// causal, 16 heads: 587 us, 595 with four). These four are of a kernel with a
// block for each tile.
template <int DP_>
struct GradShape {
    static constexpr int DP = DP_, BN = 128, NS = DP == 64 ? 8 : 4;
    static constexpr int kParts = DP == 64 ? 4 : 2, kWidth = BN / kParts, kRowWarps = 4 * kParts;
    static constexpr int kTile = kRows * DP * 2;
    // after the row warps: the copying warp, and two that issue products, one
    // those of two tiles in shared memory, one those that sum what the row warps made
    static constexpr int kCopier = kRowWarps, kIssuer = kRowWarps + 1, kSummer = kRowWarps + 2;
    static constexpr int kThreads = 32 * kRowWarps + 128;
    // registers: 512 x 104 + 128 x 64 = 640 x 96, or 256 x 208 + 128 x 88 = 384 x 168
    static constexpr int kRegsRow = kParts == 4 ? 104 : 208, kRegsOther = kParts == 4 ? 64 : 88;
    static constexpr int kColS = 0, kColG = 128, kColSum = 256;  // S, the gradient of P, the sums
    static constexpr int kColumns = 512;
    static constexpr int kItems = 4;  // of the list of items that the copying warp hands on
    static constexpr int kBars = 4 + 2 * NS + 1 + 11 + 2 * kItems;
    // the keys' gradient: P and dS have columns of their own where there is room
    static constexpr bool kOwn = 256 + 2 * DP + 128 <= 512;
    static constexpr int kColP = kOwn ? 256 + 2 * DP : kColS, kColD = kOwn ? kColP + 64 : kColG;
    static constexpr int kColW = 256 + DP;  // dS of the queries' gradient
    static constexpr int kStep = kOwn ? kWidth / 2 : kWidth;  // columns from one part's P to the next's
    static constexpr int kVec = kRowWarps * 2 * kWidth * 4;   // a warp's lse and delta of its columns
    static constexpr int kStage = 32 * 32 * 2;                // a warp's rows of 32 result columns
    static constexpr int64_t kSlot = kRows * 2 * DP;          // floats of a part's sums
    static constexpr int kSmem = 1024 + 2 * kTile + NS * kTile + kVec + kRowWarps * kStage + 48 * kItems + 8 * kBars + 16;
    using Slots = Ring<NS, kTile, NS == 4>;
};

// d = a b^T of two tiles in shared memory (K = DP).
template <int DP>
__device__ __forceinline__ void tile_product(uint32_t d, uint32_t a, uint32_t b) {
    const uint64_t da = desc_k_inside(a), db = desc_k_inside(b);
#pragma unroll
    for (int k = 0; k < DP / 16; ++k)
        mma_ss(d, desc_at(da, (k / 4) * kRows * 128 + (k % 4) * 32), desc_at(db, (k / 4) * kRows * 128 + (k % 4) * 32),
               mma_shape(128, false), k > 0);
}

// d += a (TMEM: 128 bf16 a lane, each part's `step` columns from the one before)
// x a tile in shared memory (K = its 128 rows).
template <class C>
__device__ __forceinline__ void sum_product(uint32_t d, uint32_t a, uint32_t step, uint32_t b, bool add) {
    const uint64_t db = desc_k_rows(b, kRows * 128);
    constexpr int kPer = C::kWidth / 16;  // products a part
#pragma unroll
    for (int k = 0; k < 8; ++k)
        mma_ts(d, a + (k / kPer) * step + (k % kPer) * 8, desc_at(db, k * 2048), mma_shape(C::DP, true), add || k > 0);
}

// A part of the gradient's work: blocks [first, first + count) of those that a
// tile of keys or queries of one sequence meets. Where they are not all of them,
// each of the `pieces` parts leaves its sums in memory (head h in place slot +
// h pieces + piece), and who comes last adds them up.
struct Task {
    int q0, n, k0, m, tile, first, count, pieces, slot, piece, pad[2];
};
constexpr int kLeast = 8;    // blocks of a part: its sums cost as much as one or two
constexpr int kSlots = 304;  // parts with sums in memory, at most: two for each of 152 SMs
// How many there are, and the next item (a tile of a head) that no block has.
struct Plan {
    unsigned long long next;
    int keys, queries;
};

// Barriers and memory of the gradient kernel.
template <class C>
struct GradBars {
    // each of the two tiles is there, has been used for the last time; S and the
    // gradient of P are there, have been read; dS (and P, for the keys' gradient)
    // is there; its product is done; the sums are there, have been read; all is
    // done; an item of the list is there, has been read by all
    uint32_t tile_full, tile_free, s_full, g_full, w_done, v_done, acc_full, done, s_read, g_read, w_full, v_full, acc_free,
        item_full;
    typename C::Slots ring;
    ItemList<C::kItems> items;
    uint32_t *slot;
    __device__ __forceinline__ GradBars(uint8_t *smem) {
        items.data = reinterpret_cast<int4 *>(smem + (2 + C::NS) * C::kTile + C::kVec + C::kRowWarps * C::kStage);
        uint64_t *bars = reinterpret_cast<uint64_t *>(items.data + 3 * C::kItems);
        tile_full = smem_addr(bars);
        tile_free = tile_full + 16;
        ring = {smem + 2 * C::kTile, tile_full + 32, tile_full + 32 + 8 * C::NS, tile_full + 32 + 16 * C::NS};
        s_full = tile_full + 8 * (5 + 2 * C::NS);
        g_full = s_full + 8;
        w_done = s_full + 16;
        v_done = s_full + 24;
        acc_full = s_full + 32;
        done = s_full + 40;
        s_read = s_full + 48;  // from here on arrived on by the row warps
        g_read = s_full + 56;
        w_full = s_full + 64;
        v_full = s_full + 72;
        acc_free = s_full + 80;
        item_full = s_full + 88;
        items.full = item_full;
        items.free = item_full + 8 * C::kItems;
        slot = reinterpret_cast<uint32_t *>(bars + C::kBars);
    }
    __device__ __forceinline__ void make() const {
        for (int i = threadIdx.x & 31; i < C::kBars; i += 32) {
            const uint32_t b = tile_full + 8 * i;
            bar_init(b, b >= items.free ? C::kRowWarps + 2
                        : b >= item_full ? 1
                        : b >= s_read    ? C::kRowWarps
                        : b == done      ? 2
                                         : 1);
        }
        bar_init_fence();
        __syncwarp();
    }
};

// Zeroes one side's gradients: thread `mine` of `all` does its share.
__device__ __forceinline__ void zero_gradients(const AttnArgs &a, bool keys, int tokens, int mine, int all) {
    const int heads = keys ? a.hkv : a.hq, pieces = a.D / 8;
#pragma unroll 1
    for (int64_t i = mine; i < (int64_t)tokens * heads * pieces; i += all) {
        const int64_t token = i / pieces / heads;
        const int head = (int)(i / pieces % heads), col = (int)(i % pieces) * 8;
#pragma unroll 1
        for (int o = keys ? 1 : 0; o < (keys ? 3 : 1); ++o) {
            const Out &out = o == 0 ? a.dq : o == 1 ? a.dk : a.dv;
            *reinterpret_cast<uint4 *>(out.p + token * out.ts + head * out.hs + col) = make_uint4(0u, 0u, 0u, 0u);
        }
    }
}

// The queries' blocks that a tile of keys meets: from the first that sees one of
// its keys, of every query head of the group in turn.
struct KeyBlocks {
    int b0, per_head, count;
    template <int BN>
    __device__ __forceinline__ static KeyBlocks of(const AttnArgs &a, const Seq &q, int tile) {
        KeyBlocks k;
        k.b0 = a.causal ? max(0, tile * kRows - (q.m - q.n)) / BN : 0;
        k.per_head = max(0, (q.n + BN - 1) / BN - k.b0);
        k.count = k.per_head * a.group;
        return k;
    }
};

// Lists the tiles of keys and of queries of all sequences, those with the most
// blocks first (to 1/256 of the longest; their order within that does not
// matter to any result). A tile of more than half an SM's share of all blocks
// is listed in parts, as far as there is room for their sums; which, follows
// from the numbers of blocks alone. Rows that no sound sequence holds are listed
// as tiles without a block. One block of THREADS; no loop is unrolled, since
// fetching code that runs once is most of the time.
template <int THREADS>
__device__ void make_plan(const AttnArgs &a) {
    constexpr int kBuckets = 256;
    __shared__ int place[2][kBuckets];
    __shared__ unsigned long long total;
    __shared__ int longest, slot, split, seen, lost;
    const int warp = threadIdx.x / 32, lane = threadIdx.x & 31;
    const int64_t most = (int64_t)((max(a.max_q, a.max_k) - 1) / kRows + 1) * a.group;
    int shift = 0;
    while ((most >> shift) >= kBuckets) ++shift;
    auto bucket = [&](int blocks) { return kBuckets - 1 - (blocks >> shift); };
    auto clear = [&]() {
        __syncthreads();
#pragma unroll 1
        for (int i = threadIdx.x; i < 2 * kBuckets; i += THREADS) place[i / kBuckets][i % kBuckets] = 0;
        __syncthreads();
    };
    // f(side, sequence, tile, blocks): a warp takes every 16th sequence, whose
    // offsets its lanes load 32 at a time; a lane lists one of a single tile by
    // itself, then all lanes each longer one
    constexpr int kWarps = THREADS / 32;
    auto each = [&](auto f) {
#pragma unroll 1
        for (int s0 = warp - 1; s0 <= a.seqs; s0 += 32 * kWarps) {
            const int s = s0 + kWarps * lane;
            Seq mine{0, 0, 0, 0, true};
            if (s <= a.seqs) mine = rows_of(a, s);
            const bool more = max(mine.n, mine.m) > kRows;
            uint32_t left = __ballot_sync(kFull, more);
            Seq q = mine;
            if (more) q.n = q.m = 0;
            int first = 0, step = 1;
#pragma unroll 1
            for (;;) {
#pragma unroll 1
                for (int t = first; t < (q.m + kRows - 1) / kRows; t += step)
                    f(0, q, t, q.ok ? KeyBlocks::of<kRows>(a, q, t).count : 0);
#pragma unroll 1
                for (int t = first; t < (q.n + kRows - 1) / kRows; t += step)
                    f(1, q, t, q.ok ? tile_blocks<kRows>(a, q, t) : 0);
                __syncwarp();
                if (left == 0) break;
                const int i = __ffs(left) - 1;
                left &= left - 1;
                q.ok = __shfl_sync(kFull, mine.ok, i);
                q.q0 = __shfl_sync(kFull, mine.q0, i), q.n = __shfl_sync(kFull, mine.n, i);
                q.k0 = __shfl_sync(kFull, mine.k0, i), q.m = __shfl_sync(kFull, mine.m, i);
                first = lane, step = 32;
            }
        }
    };
    if (threadIdx.x == 0) total = 0, longest = 0x7fffffff, slot = 0, split = 0, seen = 0, lost = 0;
    unsigned long long mine = 0;
    int most_mine = 0;
    clear();
    each([&](int side, const Seq &, int, int blocks) {
        atomicAdd(&place[side][bucket(blocks)], 1);
        mine += (unsigned long long)blocks * (side ? a.hq : a.hkv);
        most_mine = max(most_mine, blocks);
    });
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) mine += __shfl_xor_sync(kFull, mine, o);
    most_mine = __reduce_max_sync(kFull, most_mine);
    if (lane == 0 && mine > 0) {
        atomicAdd(&total, mine);
        atomicMax(&seen, most_mine);
    }
    __syncthreads();
    // the parts of a tile of (about) as many blocks, none longer than l
    auto parts = [&](int blocks, int l) {
        return blocks > l ? min((blocks | ((1 << shift) - 1)) / l + 1, blocks) : 1;
    };
    if (a.slots > 0) {
        if (warp == 0) {
            int l = (int)min(max((unsigned long long)kLeast, total / (2 * a.sms)), 0x40000000ull);
#pragma unroll 1
            while (seen > l) {
                int64_t need = 0;
#pragma unroll 1
                for (int i = lane; i < 2 * kBuckets; i += 32) {
                    // the most blocks of the bucket: no tile of it has more parts
                    const int n = place[i / kBuckets][i % kBuckets];
                    const int blocks = ((kBuckets - i % kBuckets) << shift) - 1;
                    if (n > 0 && blocks > l) need += n * (int64_t)(i < kBuckets ? a.hkv : a.hq) * (blocks / l + 1);
                }
#pragma unroll
                for (int o = 16; o > 0; o >>= 1) need += __shfl_xor_sync(kFull, need, o);
                if (lane == 0) split = need > 0;
                if (need <= a.slots) break;
                l += l / 4;
            }
            if (lane == 0) longest = l;
        }
        __syncthreads();
    }
    if (split) {
#pragma unroll 1
        for (int i = threadIdx.x; i < a.slots * kMostWarps; i += THREADS) a.arrived[i] = 0;
        clear();
        each([&](int side, const Seq &, int, int blocks) {
            const int n = parts(blocks, longest), each_has = n > 1 ? blocks / n : blocks, more = blocks - n * each_has;
#pragma unroll 1
            for (int i = 0; i < n; ++i) atomicAdd(&place[side][bucket(each_has + (i < more))], 1);
        });
        __syncthreads();
    }
    if (warp < 2) {
        // each lane's eight buckets, then the lanes' sums
        constexpr int kEach = kBuckets / 32;
        int v[kEach], sum = 0;
#pragma unroll
        for (int i = 0; i < kEach; ++i) sum += v[i] = place[warp][lane * kEach + i];
        int before = sum;
#pragma unroll
        for (int o = 1; o < 32; o *= 2) {
            const int x = __shfl_up_sync(kFull, before, o);
            if (lane >= o) before += x;
        }
        const int all = __shfl_sync(kFull, before, 31);
        before -= sum;
#pragma unroll
        for (int i = 0; i < kEach; ++i) {
            place[warp][lane * kEach + i] = before;
            before += v[i];
        }
        if (lane == 0) {
            // more than sound offsets can have (or than an int counts)
            if (all < 0 || all > (warp == 0 ? a.cap_k : a.cap_q)) lost = 1;
            if (warp == 0) {
                a.plan->next = 0;
                a.plan->keys = (int)min((int64_t)all, a.cap_k);
            } else {
                a.plan->queries = (int)min((int64_t)all, a.cap_q);
            }
        }
    }
    __syncthreads();
    if (lost) {  // the tiles left out keep zeros (sequences that overlap, which is flagged)
        zero_gradients(a, false, (int)a.total_q, threadIdx.x, THREADS);
        zero_gradients(a, true, (int)a.total_k, threadIdx.x, THREADS);
    }
    each([&](int side, const Seq &q, int t, int blocks) {
        const int n = parts(blocks, longest), each_has = n > 1 ? blocks / n : blocks, more = blocks - n * each_has;
        const int base = n > 1 ? atomicAdd(&slot, n * (side ? a.hq : a.hkv)) : 0;
#pragma unroll 1
        for (int i = 0; i < n; ++i) {
            const int first = i * each_has + min(i, more), count = each_has + (i < more);
            const int at = atomicAdd(&place[side][bucket(count)], 1);
            if (at < 0 || at >= (side ? a.cap_q : a.cap_k)) return;
            (side ? a.tasks_q : a.tasks_k)[at] = Task{q.q0, q.n, q.k0, q.m, t, first, count, n, base, i, {0, 0}};
        }
    });
}

// write_rows() of an item. Of one in parts the sums go to memory, and the warp
// that is the last of its like there adds them up, always in the parts' order.
template <int CH, typename F>
__device__ __forceinline__ void write_sums(const AttnArgs &a, uint32_t tmem, uint8_t *stage, const Out &out,
                                           int64_t token, const Item &it, int rows, int col, float f,
                                           int64_t slot_floats, F read) {
    if (it.pieces == 1) return write_rows<CH>(tmem, stage, out, token, it.head, rows, col, a.D, f, read);
    const int lane = threadIdx.x & 31, warp = threadIdx.x / 32, slot = it.slot + it.head * it.pieces;
    float4 *sums = reinterpret_cast<float4 *>(a.parts + slot * slot_floats + warp * (CH * 1024)) + lane;
    const int64_t step = slot_floats / 4;  // from one part's to the next's
#pragma unroll 1
    for (int c = 0; c < CH; ++c) {
        uint32_t v[32];
        tmem_load(tmem + 32 * c, v);
        load_wait(v);
#pragma unroll
        for (int e = 0; e < 8; ++e)
            __stcg(sums + it.piece * step + (8 * c + e) * 32,
                   make_float4(__uint_as_float(v[4 * e]), __uint_as_float(v[4 * e + 1]), __uint_as_float(v[4 * e + 2]),
                               __uint_as_float(v[4 * e + 3])));
    }
    read();
    __threadfence();
    __syncwarp();
    int before = 0;
    if (lane == 0) before = atomicAdd(a.arrived + slot * kMostWarps + warp, 1);
    if (__shfl_sync(kFull, before, 0) != it.pieces - 1) return;
    __threadfence();
#pragma unroll 1
    for (int c = 0; c < CH; ++c) {
        float4 x[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) x[e] = __ldcg(sums + (8 * c + e) * 32);
#pragma unroll 1
        for (int k = 1; k < it.pieces; ++k) {
            float4 y[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) y[e] = __ldcg(sums + k * step + (8 * c + e) * 32);
#pragma unroll
            for (int e = 0; e < 8; ++e) x[e].x += y[e].x, x[e].y += y[e].y, x[e].z += y[e].z, x[e].w += y[e].w;
        }
#pragma unroll
        for (int i = 0; i < 4; ++i)
            *reinterpret_cast<uint4 *>(stage_piece(stage, lane, i)) =
                make_uint4(pack_bf16(x[2 * i].x * f, x[2 * i].y * f), pack_bf16(x[2 * i].z * f, x[2 * i].w * f),
                           pack_bf16(x[2 * i + 1].x * f, x[2 * i + 1].y * f),
                           pack_bf16(x[2 * i + 1].z * f, x[2 * i + 1].w * f));
        write_stage(stage, out, token, it.head, rows, col + 32 * c, a.D);
    }
}

// What the gradient kernel needs first: the list of tiles (block 0), and (the
// others) delta = sum over the head of o grad_o, for every query row: LANES lanes
// a row, 8 values each.
template <int LANES>
__global__ void __launch_bounds__(512) attention_delta_kernel(const __grid_constant__ AttnArgs a) {
    start_next();
    if (blockIdx.x == 0) return make_plan<512>(a);
    constexpr int kRowsAtOnce = 512 / LANES;
    const int64_t rows = a.total_q * a.hq, stride = (int64_t)(gridDim.x - 1) * kRowsAtOnce;
    const int piece = threadIdx.x % LANES, mine = threadIdx.x / LANES;
    for (int64_t first = (int64_t)(blockIdx.x - 1) * kRowsAtOnce; first < rows; first += stride) {
        const int64_t r = first + mine, t = r / a.hq;
        const int h = (int)(r % a.hq);
        float d = 0.f;
        if (r < rows && piece * 8 < a.D) {
            const uint4 x = *reinterpret_cast<const uint4 *>(a.o.p + t * a.o.ts + h * a.o.hs + piece * 8);
            const uint4 y = *reinterpret_cast<const uint4 *>(a.go.p + t * a.go.ts + h * a.go.hs + piece * 8);
            const uint32_t xs[4] = {x.x, x.y, x.z, x.w}, ys[4] = {y.x, y.y, y.z, y.w};
#pragma unroll
            for (int c = 0; c < 4; ++c) {
                d = fmaf(__uint_as_float(xs[c] << 16), __uint_as_float(ys[c] << 16), d);
                d = fmaf(__uint_as_float(xs[c] & 0xffff0000u), __uint_as_float(ys[c] & 0xffff0000u), d);
            }
        }
#pragma unroll
        for (int o = LANES / 2; o > 0; o >>= 1) d += __shfl_xor_sync(kFull, d, o);
        if (r < rows && piece == 0) a.delta[(int64_t)h * a.total_q + t] = d;
    }
}

// ---- the gradient kernel ----------------------------------------------------------

// Blocks stay, and take items (a tile of a head) from the list one after the
// other: the tiles of keys first, then those of queries, either with the longest
// first, so that what comes last is short. The copying warp takes an item and
// hands it on; a block's barriers count on from one item to the next, so that an
// item's copies and first products run while the one before is being finished.
//
// Measured, with the delta kernel (causal; rate of the five products that are
// the least: 2.5 x the forward's), against a kernel for each side with a block
// for each tile: 1 x 12289, 12 heads of 64: 645 us (666), 899 TFLOP/s; 8 x 1024,
// 12 heads of 64: 71 us (98); 1 x 8192, 16 heads of 128: 570 us (590), 1206
// TFLOP/s, of the seven products done 1688; sequences of 3001, 638, 429, 95 and
// less, 16 heads of 128 on 4: 124 us (215; 140 with no tile in parts, when one SM
// has the longest tile of keys for 128 us). Bound by the tensor cores at 128; at
// 64 (1800 cycles a block, 1030 of products, 512 of exponentials) by the row
// warps' arithmetic, 2.5 instructions a cycle of 4. Writing an item's sums
// only after the next one's first block gained nothing (73 and 686 us).
template <class C>
__global__ void __launch_bounds__(C::kThreads, 1) attention_grad_kernel(const __grid_constant__ AttnArgs a) {
    constexpr int DP = C::DP, BN = C::BN, W = C::kWidth;
    constexpr int kColV = C::kColSum, kColK = C::kColSum + DP;
    extern __shared__ uint8_t smem_raw[];
    uint8_t *smem = smem_raw + ((1024 - (smem_addr(smem_raw) & 1023)) & 1023);
    const int warp = threadIdx.x / 32, lane = threadIdx.x & 31;
    const GradBars<C> bars(smem);
    const auto &ring = bars.ring;
    Item it;
    bool failed = false;
    int c = 0;  // items taken

    if (warp >= C::kRowWarps) give_registers<C::kRegsOther>();
    if (warp == C::kCopier) {
        bars.make();
        setup_arrive<C::kThreads>();
        wait_previous();
        const int64_t keys = (int64_t)a.plan->keys * a.hkv, all = keys + (int64_t)a.plan->queries * a.hq;
        int64_t at = blockIdx.x;
        // ring's tiles copied, items with blocks, copies of each of the two tiles
        int i = 0, tails = 0, n = 0, sent0 = 0, sent1 = 0;
        for (;;) {
            it = Item{};
            it.kind = at < keys ? kKeys : at < all ? kQueries : kEnd;
            const bool queries = it.kind == kQueries;
            if (it.kind != kEnd) {
                const int64_t rest = queries ? at - keys : at;
                const int heads = queries ? a.hq : a.hkv;
                const int4 *t = reinterpret_cast<const int4 *>((queries ? a.tasks_q : a.tasks_k) + rest / heads);
                const int4 x = t[0], y = t[1], z = t[2];
                it.q.q0 = x.x, it.q.n = x.y, it.q.k0 = x.z, it.q.m = x.w;
                it.tile = y.x, it.first = y.y, it.count = y.z, it.pieces = y.w;
                it.slot = z.x, it.piece = z.y;
                it.head = (int)(rest % heads);
            }
            failed = !bars.items.put(it, c);
            if (failed || it.kind == kEnd) break;
            ++c;
            const Seq &q = it.q;
            const KeyBlocks kb = KeyBlocks::of<BN>(a, q, it.tile);
            if (it.count > 0) {
                auto rows = [&](const CUtensorMap *map, int t) {
                    failed = failed ||
                             (n > 0 && !__all_sync(kFull, bar_wait(bars.tile_free + 8 * t, (n - 1) & 1, kTries)));
                    if (failed) return;
                    ++(t ? sent1 : sent0);
                    if (elect_one()) {
                        bar_arrive_expect(bars.tile_full + 8 * t, C::kTile);
                        copy_tile<DP>(smem_addr(smem) + t * C::kTile, map, it.head,
                                      (queries ? q.q0 : q.k0) + it.tile * kRows, kRows, bars.tile_full + 8 * t);
                    }
                    __syncwarp();
                };
                const int before = queries || it.first == 0 ? 0 : it.first / kb.per_head;  // heads of the group
                int h = queries ? it.head / a.group : it.head * a.group + before;
                int b = queries ? it.first : kb.b0 + it.first - before * kb.per_head;
                const int first = queries ? q.k0 : q.q0, length = queries ? q.m : q.n;
                // V's product sums over columns of the head alone
                auto block = [&](const CUtensorMap *map, bool sums) {
                    failed = failed || !ring.wait_free(i) ||
                             !ring.template fill<DP>(i, map, h, first + b * BN, BN, length - b * BN, sums, tails);
                    if (!failed) ++i;
                };
                const CUtensorMap *const x = queries ? &a.k : &a.q, *const y = queries ? &a.v : &a.g;
                // what the first products need first
                rows(queries ? &a.q : &a.k, 0);
                block(x, true);
                rows(queries ? &a.g : &a.v, 1);
                block(y, !queries);
                for (int e = 1; e < it.count && !failed; ++e) {
                    ++b;
                    if (!queries && b == kb.b0 + kb.per_head) b = kb.b0, ++h;
                    block(x, true);
                    block(y, !queries);
                }
                ++n;
            }
            if (failed) break;
            if (lane == 0) at = (int64_t)(gridDim.x + atomicAdd(&a.plan->next, 1ull));
            at = __shfl_sync(kFull, at, 0);
        }
        // no copy is in flight when the block ends, whatever gave up
        ring.drain(i);
        if (sent0 > 0) bar_wait(bars.tile_full, (sent0 - 1) & 1, kTries);
        if (sent1 > 0) bar_wait(bars.tile_full + 8, (sent1 - 1) & 1, kTries);
    } else if (warp >= C::kRowWarps) {
        if (warp == C::kIssuer) tmem_alloc(smem_addr(bars.slot), C::kColumns);
        fence_before();
        setup_wait<C::kThreads>();
        fence_after();
        const uint32_t tmem = *bars.slot;
        const uint32_t tile0 = smem_addr(smem), tile1 = tile0 + C::kTile;
        int i = 0, b = 0, n = 0;  // tiles, blocks and items with blocks so far
        auto scores = [&](int ri, bool last) {
            fence_after();
            tile_product<DP>(tmem + C::kColS, tile0, ring.addr(ri));
            mma_commit(bars.s_full);
            if (last) mma_commit(bars.tile_free);
        };
        auto grads = [&](int ri, bool last) {
            fence_after();
            tile_product<DP>(tmem + C::kColG, tile1, ring.addr(ri + 1));
            mma_commit(bars.g_full);
            if (last) mma_commit(bars.tile_free + 8);
        };
        auto sum_v = [&](int ri, bool add) {
            fence_after();
            sum_product<C>(tmem + kColV, tmem + C::kColP, C::kStep, ring.addr(ri + 1), add);
        };
        auto sum_k = [&](int ri, bool add) {
            fence_after();
            sum_product<C>(tmem + kColK, tmem + C::kColD, C::kStep, ring.addr(ri), add);
        };
        if (warp == C::kIssuer && elect_one()) {
            failed = !bars.items.get_one(it, c);
            // ---- tiles of keys
            if (C::kOwn) {
                // P^T and dS^T have columns of their own: the next S^T and gradient
                // of P^T are computed as soon as these have been read
                for (; !failed && it.kind == kKeys; failed = failed || !bars.items.get_one(it, c)) {
                    const int blocks = it.count;
                    for (int j = 0; j < blocks; ++j, ++b, i += 2) {
                        failed = (j == 0 && !bar_wait(bars.tile_full, n & 1, kTries)) || !ring.wait_full(i) ||
                                 (b > 0 && !bar_wait(bars.s_read, (b - 1) & 1, kTries));
                        if (failed) break;
                        scores(i, j + 1 == blocks);
                        failed = (j == 0 && !bar_wait(bars.tile_full + 8, n & 1, kTries)) || !ring.wait_full(i + 1) ||
                                 (b > 0 && !bar_wait(bars.g_read, (b - 1) & 1, kTries));
                        if (failed) break;
                        grads(i, j + 1 == blocks);
                    }
                    n += blocks > 0;
                }
            } else {
                // P^T takes the place of S^T, dS^T that of the gradient of P^T,
                // and the next product into either comes after the one that reads
                // it (products run in the order of their issue): while the rows'
                // arithmetic makes P^T, dK and the next gradient are computed, while
                // it makes dS^T, dV and the next S^T, which may be the next item's.
                auto blocks_of = [&]() { return it.kind == kKeys ? it.count : 0; };
                // the next tile of keys that meets queries (or what comes after the last)
                auto next_item = [&]() {
                    do failed = failed || !bars.items.get_one(it, c);
                    while (!failed && it.kind == kKeys && blocks_of() == 0);
                };
                if (it.kind == kKeys && blocks_of() == 0) next_item();
                int blocks = failed ? 0 : blocks_of();
                if (blocks > 0) {
                    failed = !bar_wait(bars.tile_full, 0, kTries) || !ring.wait_full(0);
                    if (!failed) scores(0, blocks == 1);
                    failed = failed || !bar_wait(bars.tile_full + 8, 0, kTries) || !ring.wait_full(1);
                    if (!failed) grads(0, blocks == 1);
                }
                while (blocks > 0 && !failed) {
                    int after = 0;
                    for (int j = 0; j < blocks; ++j, ++b, i += 2) {
                        const bool turn = j + 1 == blocks;
                        failed = !bar_wait(bars.v_full, b & 1, kTries) ||
                                 (j == 0 && n > 0 && !bar_wait(bars.acc_free, (n - 1) & 1, kTries));
                        if (failed) break;
                        sum_v(i, j > 0);
                        mma_commit(ring.empty_bar(i + 1));
                        if (turn) {
                            next_item();
                            if (failed) break;
                            after = blocks_of();
                        }
                        const bool more = !turn || after > 0, last = turn ? after == 1 : j + 2 == blocks;
                        if (more) {
                            failed = (turn && !bar_wait(bars.tile_full, (n + 1) & 1, kTries)) || !ring.wait_full(i + 2);
                            if (failed) break;
                            scores(i + 2, last);
                        }
                        failed = !bar_wait(bars.w_full, b & 1, kTries);
                        if (failed) break;
                        sum_k(i, j > 0);
                        mma_commit(ring.empty_bar(i));
                        if (turn) mma_commit(bars.acc_full);
                        if (more) {
                            failed = (turn && !bar_wait(bars.tile_full + 8, (n + 1) & 1, kTries)) || !ring.wait_full(i + 3);
                            if (failed) break;
                            grads(i + 2, last);
                        }
                    }
                    ++n;
                    blocks = after;
                }
            }
            // ---- tiles of queries: S and the gradient of P of each block, once
            // those of the block before have been read
            int r = C::kOwn ? b : 0;  // blocks of these two barriers
            for (; !failed && it.kind == kQueries; failed = failed || !bars.items.get_one(it, c)) {
                const int blocks = it.count;
                for (int j = 0; j < blocks; ++j, ++r, i += 2) {
                    failed = (j == 0 && !bar_wait(bars.tile_full, n & 1, kTries)) || !ring.wait_full(i) ||
                             (r > 0 && !bar_wait(bars.s_read, (r - 1) & 1, kTries));
                    if (failed) break;
                    fence_after();
                    tile_product<DP>(tmem + C::kColS, tile0, ring.addr(i));
                    mma_commit(bars.s_full);
                    if (j + 1 == blocks) mma_commit(bars.tile_free);
                    failed = (j == 0 && !bar_wait(bars.tile_full + 8, n & 1, kTries)) || !ring.wait_full(i + 1) ||
                             (r > 0 && !bar_wait(bars.g_read, (r - 1) & 1, kTries));
                    if (failed) break;
                    fence_after();
                    tile_product<DP>(tmem + C::kColG, tile1, ring.addr(i + 1));
                    mma_commit(bars.g_full);
                    mma_commit(ring.empty_bar(i + 1));
                    if (j + 1 == blocks) mma_commit(bars.tile_free + 8);
                }
                n += blocks > 0;
            }
            // every product, and every arrival that it makes, is done before
            // the block's memory is given back
            mma_commit(bars.done);
            failed |= !bar_wait(bars.done, 0, kTries);
        } else if (warp == C::kSummer && elect_one()) {
            failed = !bars.items.get_one(it, c);
            if (C::kOwn) {
                for (; !failed && it.kind == kKeys; failed = failed || !bars.items.get_one(it, c)) {
                    const int blocks = it.count;
                    for (int j = 0; j < blocks; ++j, ++b, i += 2) {
                        failed = !bar_wait(bars.v_full, b & 1, kTries) ||
                                 (j == 0 && n > 0 && !bar_wait(bars.acc_free, (n - 1) & 1, kTries));
                        if (failed) break;
                        sum_v(i, j > 0);
                        mma_commit(bars.v_done);
                        failed = !bar_wait(bars.w_full, b & 1, kTries);
                        if (failed) break;
                        sum_k(i, j > 0);
                        mma_commit(bars.w_done);
                        // the other products of this block are done: the row warps had them
                        mma_commit(ring.empty_bar(i));
                        mma_commit(ring.empty_bar(i + 1));
                        if (j + 1 == blocks) mma_commit(bars.acc_full);
                    }
                    n += blocks > 0;
                }
            } else {
                for (; !failed && it.kind == kKeys; failed = failed || !bars.items.get_one(it, c)) {
                    // the issuer's; each is seen to its end, so that the barriers'
                    // parities below are those of this item's blocks
                    const int blocks = it.count;
                    if (blocks == 0) continue;
                    failed = !bar_wait(bars.acc_full, n & 1, kTries);
                    b += blocks, i += 2 * blocks, ++n;
                }
            }
            // dQ += dS K (K's scores are done: the row warps had them)
            for (; !failed && it.kind == kQueries; failed = failed || !bars.items.get_one(it, c)) {
                const int blocks = it.count;
                for (int j = 0; j < blocks; ++j, ++b, i += 2) {
                    failed = !bar_wait(bars.w_full, b & 1, kTries) ||
                             (j == 0 && n > 0 && !bar_wait(bars.acc_free, (n - 1) & 1, kTries));
                    if (failed) break;
                    fence_after();
                    sum_product<C>(tmem + C::kColSum, tmem + C::kColW, W / 2, ring.addr(i), j > 0);
                    mma_commit(bars.w_done);
                    mma_commit(ring.empty_bar(i));
                    if (j + 1 == blocks) mma_commit(bars.acc_full);
                }
                n += blocks > 0;
            }
            mma_commit(bars.done);
            failed |= !bar_wait(bars.done, 0, kTries);
        }
        __syncwarp();
    } else {
        take_registers<C::kRegsRow>();
        fence_before();
        setup_wait<C::kThreads>();
        fence_after();
        const uint32_t tmem = *bars.slot;
        const int part = warp / 4;  // of the columns
        const uint32_t lanes = tmem + ((uint32_t)(warp & 3) << 21);
        uint8_t *stage = smem + (2 + C::NS) * C::kTile + C::kVec + warp * C::kStage;
        const uint64_t scale2 = pair(a.scale2, a.scale2);
        int b = 0, n = 0;  // blocks and items with blocks so far
        wait_previous();
        failed = !bars.items.get_warp(it, c);

        // ---- tiles of keys
        const uint32_t s_addr = lanes + C::kColS + W * part, g_addr = lanes + C::kColG + W * part;
        const uint32_t p_addr = lanes + C::kColP + C::kStep * part, d_addr = lanes + C::kColD + C::kStep * part;
        float *vec = reinterpret_cast<float *>(smem + (2 + C::NS) * C::kTile) + warp * 2 * W;
        // this lane's share of its columns' lse and delta, loaded a block ahead
        // (an item's first before the item before is written out) and not looked
        // at before the block is there
        float nl[W / 32], nd[W / 32];
        KeyBlocks k{};
        int h = 0, fb = 0;  // of the next block fetched
        auto fetch = [&]() {
#pragma unroll
            for (int e = 0; e < W / 32; ++e) {
                const int r = fb * BN + W * part + lane + 32 * e;
                nl[e] = -INFINITY, nd[e] = 0.f;
                if (r < it.q.n) {
                    const int64_t at = (int64_t)h * a.total_q + it.q.q0 + r;
                    nl[e] = a.lse[at];
                    nd[e] = a.delta[at];
                }
            }
            if (++fb == k.b0 + k.per_head) fb = k.b0, ++h;
        };
        auto start = [&]() {
            k = KeyBlocks::of<BN>(a, it.q, it.tile);
            if (it.count > 0) {
                const int before = it.first == 0 ? 0 : it.first / k.per_head;
                h = it.head * a.group + before, fb = k.b0 + it.first - before * k.per_head;
                fetch();
            }
        };
        if (!failed && it.kind == kKeys) start();
        while (!failed && it.kind == kKeys) {
            const int r = it.tile * kRows + (threadIdx.x & 127), count = it.count;
            const int below = a.causal ? r - (it.q.m - it.q.n) - W * part : 0;  // queries before it do not see key r
            int bi = (fb == k.b0 ? k.b0 + k.per_head : fb) - 1;  // the block at hand: the one fetched
            for (int e = 0; e < count; ++e, ++b) {
                __syncwarp();
#pragma unroll
                for (int x = 0; x < W / 32; ++x) {
                    // -lse x log2 e; minus infinity for rows that are not there or see
                    // nothing: probability 0
                    vec[lane + 32 * x] = nl[x] == -INFINITY ? -INFINITY : -nl[x] * kLog2e;
                    vec[W + lane + 32 * x] = -nd[x];
                }
                __syncwarp();
                if (e + 1 < count) fetch();
                // masked: query i sees key r when i >= r - off
                const int low = below - bi * BN;
                if (++bi == k.b0 + k.per_head) bi = k.b0;
                const bool whole = __all_sync(kFull, low <= 0);
                if (!__all_sync(kFull, bar_wait(bars.s_full, b & 1, kTries))) {
                    failed = true;
                    break;
                }
                fence_after();
                uint32_t s[W], w[W / 2];
                {
                    uint32_t x[W / 32][32];
#pragma unroll
                    for (int c = 0; c < W / 32; ++c) tmem_load(s_addr + 32 * c, x[c]);
#pragma unroll
                    for (int c = 0; c < W / 32; ++c) load_wait(x[c]);
                    if (C::kOwn) {
                        fence_before();
                        __syncwarp();
                        if (lane == 0) bar_arrive(bars.s_read);
                    }
#pragma unroll
                    for (int c = 0; c < W; c += 4) {
                        const ulonglong2 l = *reinterpret_cast<const ulonglong2 *>(vec + c);
#pragma unroll
                        for (int x4 = c; x4 < c + 4; x4 += 2) {
                            const float2 y = unpair(fma2(pair_bits(x[x4 / 32][x4 % 32], x[x4 / 32][x4 % 32 + 1]), scale2,
                                                         x4 > c ? l.y : l.x));
                            s[x4] = __float_as_uint(exp2_approx(y.x));
                            s[x4 + 1] = __float_as_uint(exp2_approx(y.y));
                        }
                    }
                }
                if (!whole) {
#pragma unroll
                    for (int c = 0; c < W; ++c)
                        if (c < low) s[c] = 0u;
                }
#pragma unroll
                for (int c = 0; c < W; c += 2) w[c / 2] = pack_bf16(__uint_as_float(s[c]), __uint_as_float(s[c + 1]));
                if (C::kOwn && b > 0 && !__all_sync(kFull, bar_wait(bars.v_done, (b - 1) & 1, kTries))) {
                    failed = true;
                    break;
                }
                fence_after();
                tmem_store(p_addr, w);
                store_wait();
                fence_before();
                __syncwarp();
                if (lane == 0) bar_arrive(bars.v_full);
                if (!__all_sync(kFull, bar_wait(bars.g_full, b & 1, kTries))) {
                    failed = true;
                    break;
                }
                fence_after();
                uint32_t g[W / 32][32];
#pragma unroll
                for (int c = 0; c < W / 32; ++c) tmem_load(g_addr + 32 * c, g[c]);
#pragma unroll
                for (int c = 0; c < W / 32; ++c) load_wait(g[c]);
                if (C::kOwn) {
                    fence_before();
                    __syncwarp();
                    if (lane == 0) bar_arrive(bars.g_read);
                }
                if (!whole) {
#pragma unroll
                    for (int c = 0; c < W; ++c)
                        if (c < low) g[c / 32][c % 32] = 0u;
                }
#pragma unroll
                for (int c = 0; c < W; c += 4) {
                    const ulonglong2 d = *reinterpret_cast<const ulonglong2 *>(vec + W + c);
#pragma unroll
                    for (int x4 = c; x4 < c + 4; x4 += 2) {
                        const float2 y = unpair(mul2(pair_bits(s[x4], s[x4 + 1]),
                                                     add2(pair_bits(g[x4 / 32][x4 % 32], g[x4 / 32][x4 % 32 + 1]),
                                                          x4 > c ? d.y : d.x)));
                        w[x4 / 2] = pack_bf16(y.x, y.y);
                    }
                }
                if (C::kOwn && b > 0 && !__all_sync(kFull, bar_wait(bars.w_done, (b - 1) & 1, kTries))) {
                    failed = true;
                    break;
                }
                fence_after();
                tmem_store(d_addr, w);
                store_wait();
                fence_before();
                __syncwarp();
                if (lane == 0) bar_arrive(bars.w_full);
            }
            if (failed) break;
            failed = !bars.items.get_warp(it, c);
            if (failed) break;
            if (it.kind == kKeys) start();
            Item was;  // the item that ends here
            bars.items.read(was, c - 2);
            const int first = was.tile * kRows + (warp & 3) * 32;  // the warp's first row
            const int64_t token = was.q.k0 + (int64_t)first;
            if (was.count > 0) {
                if (!__all_sync(kFull, bar_wait(bars.acc_full, n & 1, kTries))) {
                    failed = true;
                    break;
                }
                fence_after();
                // dV's columns, then dK's, shared out over the parts
                constexpr int CH = 2 * DP / 32 / C::kParts;
                const int c0 = part * CH, col = 32 * c0 % DP;
                const bool keys = 32 * c0 >= DP;
                write_sums<CH>(a, lanes + C::kColSum + 32 * c0, stage, keys ? a.dk : a.dv, token, was, was.q.m - first,
                                  col, keys ? a.scale : 1.f, C::kSlot, [&]() {
                                      fence_before();
                                      __syncwarp();
                                      if (lane == 0) bar_arrive(bars.acc_free);
                                  });
                ++n;
            } else if (first + lane < was.q.m && part < 2) {
                const Out &out = part ? a.dk : a.dv;
                write_zero_row(out.p + (token + lane) * out.ts + was.head * out.hs, a.D);
            }
            bars.items.finished(c - 2);
        }

        // ---- tiles of queries
        // an item's row: its lse and delta are loaded before the item before is
        // written out
        float lse = 0.f, delta = 0.f;
        auto load_row = [&]() {
            const int r = it.tile * kRows + (threadIdx.x & 127);
            lse = -INFINITY, delta = 0.f;
            if (r < it.q.n) {
                const int64_t at = (int64_t)it.head * a.total_q + it.q.q0 + r;
                lse = a.lse[at];
                delta = a.delta[at];
            }
        };
        // of these barriers: with heads of 128 the keys' gradient does without them
        int r1 = C::kOwn ? b : 0;
        if (!failed && it.kind == kQueries) load_row();
        while (!failed && it.kind == kQueries) {
            const int blocks = it.count;
            // keys that the row sees, from this part's first on
            const int lim = visible(a, it.q, it.tile * kRows + (threadIdx.x & 127)) - it.first * BN - W * part;
            // a row that sees nothing: every probability 0
            const float l2 = lse == -INFINITY ? -INFINITY : -lse * kLog2e;
            const uint64_t lse22 = pair(l2, l2), delta2 = pair(-delta, -delta);
            for (int j = 0; j < blocks; ++j, ++b, ++r1) {
                if (!__all_sync(kFull, bar_wait(bars.s_full, b & 1, kTries))) {
                    failed = true;
                    break;
                }
                fence_after();
                uint32_t s[W], g[W / 32][32], w[W / 2];
                {
                    uint32_t x[W / 32][32];
#pragma unroll
                    for (int c = 0; c < W / 32; ++c) tmem_load(lanes + C::kColS + W * part + 32 * c, x[c]);
#pragma unroll
                    for (int c = 0; c < W / 32; ++c) load_wait(x[c]);
                    fence_before();
                    __syncwarp();
                    if (lane == 0) bar_arrive(bars.s_read);
#pragma unroll
                    for (int c = 0; c < W; c += 2) {
                        const float2 y = unpair(fma2(pair_bits(x[c / 32][c % 32], x[c / 32][c % 32 + 1]), scale2, lse22));
                        s[c] = __float_as_uint(exp2_approx(y.x));
                        s[c + 1] = __float_as_uint(exp2_approx(y.y));
                    }
                }
                if (!__all_sync(kFull, bar_wait(bars.g_full, b & 1, kTries))) {
                    failed = true;
                    break;
                }
                fence_after();
#pragma unroll
                for (int c = 0; c < W / 32; ++c) tmem_load(lanes + C::kColG + W * part + 32 * c, g[c]);
#pragma unroll
                for (int c = 0; c < W / 32; ++c) load_wait(g[c]);
                fence_before();
                __syncwarp();
                if (lane == 0) bar_arrive(bars.g_read);
                const int seen = lim - j * BN;
                if (!__all_sync(kFull, seen >= W)) {
#pragma unroll
                    for (int c = 0; c < W; ++c)
                        if (c >= seen) s[c] = g[c / 32][c % 32] = 0u;
                }
#pragma unroll
                for (int c = 0; c < W; c += 2) {
                    const float2 d = unpair(mul2(pair_bits(s[c], s[c + 1]),
                                                 add2(pair_bits(g[c / 32][c % 32], g[c / 32][c % 32 + 1]), delta2)));
                    w[c / 2] = pack_bf16(d.x, d.y);
                }
                // dS's place: the block before is done with it, and at an item's
                // start every warp with the sums of the one before
                if ((r1 > 0 && !__all_sync(kFull, bar_wait(bars.w_done, (r1 - 1) & 1, kTries))) ||
                    (j == 0 && n > 0 && !__all_sync(kFull, bar_wait(bars.acc_free, (n - 1) & 1, kTries)))) {
                    failed = true;
                    break;
                }
                fence_after();
                tmem_store(lanes + C::kColW + W / 2 * part, w);
                store_wait();
                fence_before();
                __syncwarp();
                if (lane == 0) bar_arrive(bars.w_full);
            }
            if (failed) break;
            failed = !bars.items.get_warp(it, c);
            if (failed) break;
            if (it.kind == kQueries) load_row();
            Item was;
            bars.items.read(was, c - 2);
            const int first = was.tile * kRows + (warp & 3) * 32;
            const int64_t token = was.q.q0 + (int64_t)first;
            if (was.count > 0) {
                if (!__all_sync(kFull, bar_wait(bars.acc_full, n & 1, kTries))) {
                    failed = true;
                    break;
                }
                fence_after();
                auto read = [&]() {
                    fence_before();
                    __syncwarp();
                    if (lane == 0) bar_arrive(bars.acc_free);
                };
                constexpr int CH = DP / 32 / C::kParts > 0 ? DP / 32 / C::kParts : 1;
                if (part < DP / 32 / CH)
                    write_sums<CH>(a, lanes + C::kColSum + 32 * CH * part, stage, a.dq, token, was, was.q.n - first,
                                      32 * CH * part, a.scale, C::kSlot, read);
                else
                    read();
                ++n;
            } else if (first + lane < was.q.n && part == 0) {
                write_zero_row(a.dq.p + (token + lane) * a.dq.ts + was.head * a.dq.hs, a.D);
            }
            bars.items.finished(c - 2);
        }
    }
    if (failed) set_status(a.status, DPB_DEV_TIMEOUT);
    fence_before();
    __syncthreads();
    if (warp == C::kIssuer) tmem_free(*bars.slot, C::kColumns);
}

// ---- host side ------------------------------------------------------------------

PFN_cuTensorMapEncodeTiled_v12000 encoder() {
    static PFN_cuTensorMapEncodeTiled_v12000 fn = [] {
        void *p = nullptr;
        cudaDriverEntryPointQueryResult r;
        if (cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &p, 12000, cudaEnableDefault, &r) !=
                cudaSuccess ||
            r != cudaDriverEntryPointSuccess) {
            cudaGetLastError();
            p = nullptr;
        }
        return reinterpret_cast<PFN_cuTensorMapEncodeTiled_v12000>(p);
    }();
    return fn;
}

// Map of a [tokens][heads][D] tensor in boxes of 64 columns x `rows` tokens of
// one head; columns past D read as zero.
dpb_status make_map(CUtensorMap *map, const dpb_heads *h, int64_t tokens, int heads, int D, int rows) {
    std::memset(map, 0, sizeof(*map));
    if (tokens == 0) return DPB_OK;
    const auto fn = encoder();
    if (!fn) return fail(DPB_ERR_CUDA, "the driver has no cuTensorMapEncodeTiled");
    const int64_t hs = heads > 1 ? h->head_stride : 64, ts = tokens > 1 ? h->token_stride : 64;
    const cuuint64_t dims[3] = {(cuuint64_t)D, (cuuint64_t)heads, (cuuint64_t)tokens};
    const cuuint64_t strides[2] = {(cuuint64_t)hs * 2, (cuuint64_t)ts * 2};
    const cuuint32_t box[3] = {64, 1, (cuuint32_t)rows}, one[3] = {1, 1, 1};
    const CUresult r = fn(map, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 3, h->data, dims, strides, box, one,
                          CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B,
                          CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
    if (r != CUDA_SUCCESS) return fail(DPB_ERR_CUDA, "cuTensorMapEncodeTiled failed (%d)", (int)r);
    return DPB_OK;
}

dpb_status check_rows(const dpb_heads *h, const char *name, int64_t tokens, int heads) {
    if (tokens == 0) return DPB_OK;
    if (!h) return fail(DPB_ERR_INVALID_ARG, "%s is NULL", name);
    DPB_CHECK(need(h->data, name, 16));
    if ((tokens > 1 && (h->token_stride <= 0 || h->token_stride % 8)) ||
        (heads > 1 && (h->head_stride <= 0 || h->head_stride % 8)))
        return fail(DPB_ERR_INVALID_ARG, "the strides of %s must be positive multiples of 8", name);
    if (h->token_stride >= (1ll << 38) || h->head_stride >= (1ll << 38))
        return fail(DPB_ERR_UNSUPPORTED, "the strides of %s are too large", name);
    return DPB_OK;
}

dpb_status check_attention(const dpb_attention_config *c) {
    if (!c) return fail(DPB_ERR_INVALID_ARG, "cfg is NULL");
    if (c->dtype != DPB_BF16) return fail(DPB_ERR_UNSUPPORTED, "attention takes bf16 rows");
    if (c->seqs > 0x7fffff00) return fail(DPB_ERR_UNSUPPORTED, "at most 2^31 - 256 sequences");
    if (c->seqs < 0 || c->total_q < 0 || c->total_k < 0 || c->max_q < 0 || c->max_k < 0)
        return fail(DPB_ERR_INVALID_ARG, "a size is negative");
    if (c->total_q > 0x7fffff00ll || c->total_k > 0x7fffff00ll)
        return fail(DPB_ERR_UNSUPPORTED, "at most 2^31 - 256 tokens");
    if (c->heads_q < 1 || c->heads_kv < 1 || c->heads_q % c->heads_kv)
        return fail(DPB_ERR_INVALID_ARG, "heads_q must be a positive multiple of heads_kv");
    if (c->head_dim < 8 || c->head_dim > 128 || c->head_dim % 8)
        return fail(DPB_ERR_UNSUPPORTED, "head_dim must be a multiple of 8 in [8, 128]");
    DPB_CHECK(check_slot(c->status_slot));
    if (!(c->scale > 0.f) || !std::isfinite(c->scale))
        return fail(DPB_ERR_INVALID_ARG, "scale must be positive and finite");
    return DPB_OK;
}

dpb_status check_offsets(const dpb_attention_config *c, const int32_t *cu_q, const int32_t *cu_k) {
    if ((cu_q == nullptr) != (cu_k == nullptr))
        return fail(DPB_ERR_INVALID_ARG, "cu_q and cu_k must both be given or both be NULL");
    if (!cu_q && c->seqs > 1) return fail(DPB_ERR_INVALID_ARG, "without offsets there is one sequence");
    if (cu_q) {
        DPB_CHECK(need(cu_q, "cu_q", 4));
        DPB_CHECK(need(cu_k, "cu_k", 4));
    }
    return DPB_OK;
}

// The gradient's workspace after the status word: a Plan and its lists, the
// counts and sums of tiles in parts, delta. Sound offsets give no more than a
// tile for every 128 tokens and one a sequence, and one before and after them.
struct GradSpace {
    int64_t cap_k, cap_q;
    int slots;
    size_t plan, tasks_k, tasks_q, arrived, parts, delta, bytes;
    explicit GradSpace(const dpb_attention_config *c) {
        const int64_t blocks = ((int64_t)std::max(c->max_q, c->max_k) + kRows - 1) / kRows * (c->heads_q / c->heads_kv);
        slots = blocks > kLeast ? kSlots : 0;
        cap_k = c->total_k / kRows + c->seqs + 2 + slots;
        cap_q = c->total_q / kRows + c->seqs + 2 + slots;
        plan = kStatusBytes;
        tasks_k = plan + sizeof(Task);
        tasks_q = tasks_k + sizeof(Task) * (size_t)cap_k;
        arrived = tasks_q + sizeof(Task) * (size_t)cap_q;
        parts = arrived + sizeof(int) * kMostWarps * (size_t)slots;
        delta = parts + sizeof(float) * kRows * 2 * (c->head_dim <= 64 ? 64 : 128) * (size_t)slots;
        bytes = delta + sizeof(float) * (size_t)c->heads_q * (size_t)c->total_q;
    }
};
size_t attention_workspace(const dpb_attention_config *c) { return GradSpace(c).bytes; }

void fill_args(AttnArgs &a, const dpb_attention_config *c, const int32_t *cu_q, const int32_t *cu_k) {
    a.cu_q = cu_q;
    a.cu_k = cu_k;
    a.total_q = c->total_q;
    a.total_k = c->total_k;
    a.seqs = c->seqs;
    a.max_q = (int)std::min<int64_t>(c->max_q, c->total_q);  // no sequence is longer
    a.max_k = (int)std::min<int64_t>(c->max_k, c->total_k);
    a.hq = c->heads_q;
    a.hkv = c->heads_kv;
    a.group = c->heads_q / c->heads_kv;
    a.D = c->head_dim;
    a.causal = c->causal != 0;
    a.scale = c->scale;
    a.scale2 = c->scale * kLog2e;
}

In in_rows(const dpb_heads *h) { return h ? In{static_cast<const bf16 *>(h->data), h->token_stride, h->head_stride} : In{}; }
Out out_rows(const dpb_heads *h) { return h ? Out{static_cast<bf16 *>(h->data), h->token_stride, h->head_stride} : Out{}; }

// A register split draws on what the block is launched with: a build whose
// kernel got fewer registers must not run it (its threads would wait for ever).
template <class C>
cudaError_t registers_cover(const void *kernel) {
    cudaFuncAttributes f;
    const cudaError_t e = cudaFuncGetAttributes(&f, kernel);
    if (e != cudaSuccess) return e;
    return f.numRegs * C::kThreads >= (C::kThreads - 128) * C::kRegsRow + 128 * C::kRegsOther
               ? cudaSuccess
               : cudaErrorLaunchOutOfResources;
}

int multiprocessors() {
    int dev = 0, sms = 1;
    if (cudaGetDevice(&dev) != cudaSuccess || cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess)
        cudaGetLastError();
    return sms;
}

// EARLY: the kernel may start, and set itself up, while the one before it in
// the stream runs; it waits for that one's results itself.
template <class C, void (*KERNEL)(AttnArgs), bool EARLY>
cudaError_t launch_blocks(const AttnArgs &a, int64_t blocks, cudaStream_t s) {
    if (blocks == 0) return cudaSuccess;
    if (blocks > 0x7fffffffll) return cudaErrorInvalidConfiguration;
    const void *kernel = reinterpret_cast<const void *>(KERNEL);
    static const cudaError_t covered = registers_cover<C>(kernel);
    if (covered != cudaSuccess) return covered;
    const cudaError_t e = allow_smem(kernel, C::kSmem);
    if (e != cudaSuccess) return e;
    cudaLaunchConfig_t how{};
    how.gridDim = dim3((unsigned)blocks);
    how.blockDim = dim3(C::kThreads);
    how.dynamicSmemBytes = C::kSmem;
    how.stream = s;
    cudaLaunchAttribute early{};
    early.id = cudaLaunchAttributeProgrammaticStreamSerialization;
    early.val.programmaticStreamSerializationAllowed = 1;
    how.attrs = &early;
    how.numAttrs = EARLY ? 1 : 0;
    const cudaError_t launched = cudaLaunchKernelEx(&how, KERNEL, a);
    return launched == cudaSuccess ? cudaGetLastError() : launched;
}

using Fwd64 = FwdShape<64, 128, 8>;
using Fwd128 = FwdShape<128, 128, 4>;
using Grad64 = GradShape<64>;
using Grad128 = GradShape<128>;

template <class C>
cudaError_t launch_attention_forward(AttnArgs &a, cudaStream_t s) {
    a.tiles = (int)std::max<int64_t>(((int64_t)a.max_q + 2 * kRows - 1) / (2 * kRows), 1);
    // With lengths far from the longest most blocks of a grid for it would be
    // empty: where there can be no more than half of it, the blocks count the
    // sequences' own pairs of tiles (64 x 1024, 12 heads of 64, with the longest
    // given as 65536: 164 us, 772 without; sequences of 3001, 638, 429 and less,
    // 16 heads of 64: 35.5, 39.3). With equal lengths, known, the longest rows of
    // all go first: 145 us.
    const int64_t most = a.total_q / (2 * kRows) + a.seqs;
    a.close = (int64_t)a.tiles * a.seqs > 2 * most;
    const int64_t items = (a.close ? most : (int64_t)a.tiles * a.seqs) * a.hq;
    // The last blocks, one for every two SMs at most, write the rows before the first
    // sequence and after the last (32 x 1024 of 65536 rows, 12 heads of 64: 124 us, 353
    // with two blocks a head; without such rows 8 x 1024 takes 24.7 us as before).
    const int64_t blocks = items + std::min<int64_t>((multiprocessors() + 1) / 2, (a.total_q / (2 * kRows) + 2) * a.hq);
    if (blocks > 0x7fffffffll) return cudaErrorInvalidConfiguration;
    a.items = (int)items;
    return launch_blocks<C, attention_forward_kernel<C>, false>(a, blocks, s);
}

template <class C>
dpb_status launch_attention_backward(AttnArgs &a, cudaStream_t s) {
    const int sms = multiprocessors();
    a.sms = sms;
    constexpr int kLanes = C::DP / 8, kRowsAtOnce = 512 / kLanes;
    const int64_t rows = a.total_q * a.hq;
    const int64_t blocks = 1 + std::min<int64_t>((rows + kRowsAtOnce - 1) / kRowsAtOnce, 16 * sms);
    attention_delta_kernel<kLanes><<<(unsigned)blocks, 512, 0, s>>>(a);
    DPB_CHECK(launch_status(cudaGetLastError(), "attention_backward (delta)"));
    const int64_t items = a.cap_k * a.hkv + a.cap_q * a.hq;
    return launch_status(launch_blocks<C, attention_grad_kernel<C>, true>(a, std::min<int64_t>(items, sms), s),
                         "attention_backward");
}

}  // namespace
}  // namespace dpb

using namespace dpb;

extern "C" {

dpb_status dpb_attention_workspace_size(const dpb_attention_config *cfg, size_t *bytes) {
    DPB_CHECK(check_attention(cfg));
    if (!bytes) return fail(DPB_ERR_INVALID_ARG, "bytes is NULL");
    *bytes = attention_workspace(cfg);
    return DPB_OK;
}

dpb_status dpb_attention_forward(const dpb_attention_config *cfg, const dpb_heads *q, const dpb_heads *k,
                                 const dpb_heads *v, const int32_t *cu_q, const int32_t *cu_k, const dpb_heads *o,
                                 float *lse, void *workspace, size_t workspace_bytes, void *stream) {
    DPB_CHECK(check_attention(cfg));
    if (cfg->total_q == 0) return DPB_OK;
    DPB_CHECK(check_rows(q, "q", cfg->total_q, cfg->heads_q));
    DPB_CHECK(check_rows(k, "k", cfg->total_k, cfg->heads_kv));
    DPB_CHECK(check_rows(v, "v", cfg->total_k, cfg->heads_kv));
    DPB_CHECK(check_rows(o, "o", cfg->total_q, cfg->heads_q));
    DPB_CHECK(check_offsets(cfg, cu_q, cu_k));
    DPB_CHECK(need(lse, "lse", 4));
    AttnArgs a{};
    DPB_CHECK(place_status(cfg->status_slot, workspace, workspace_bytes, kStatusBytes, &a.status));
    fill_args(a, cfg, cu_q, cu_k);
    const bool small = cfg->head_dim <= 64;
    DPB_CHECK(make_map(&a.q, q, cfg->total_q, cfg->heads_q, cfg->head_dim, kRows));
    DPB_CHECK(make_map(&a.k, k, cfg->total_k, cfg->heads_kv, cfg->head_dim, small ? Fwd64::BN : Fwd128::BN));
    DPB_CHECK(make_map(&a.v, v, cfg->total_k, cfg->heads_kv, cfg->head_dim, small ? Fwd64::BN : Fwd128::BN));
    a.out = out_rows(o);
    a.lse = lse;
    const cudaStream_t s = static_cast<cudaStream_t>(stream);
    return launch_status(small ? launch_attention_forward<Fwd64>(a, s) : launch_attention_forward<Fwd128>(a, s),
                         "attention_forward");
}

dpb_status dpb_attention_backward(const dpb_attention_config *cfg, const dpb_heads *q, const dpb_heads *k,
                                  const dpb_heads *v, const dpb_heads *o, const float *lse, const dpb_heads *grad_o,
                                  const int32_t *cu_q, const int32_t *cu_k, const dpb_heads *grad_q,
                                  const dpb_heads *grad_k, const dpb_heads *grad_v, void *workspace,
                                  size_t workspace_bytes, void *stream) {
    DPB_CHECK(check_attention(cfg));
    if (cfg->total_q == 0 && cfg->total_k == 0) return DPB_OK;
    DPB_CHECK(check_rows(q, "q", cfg->total_q, cfg->heads_q));
    DPB_CHECK(check_rows(k, "k", cfg->total_k, cfg->heads_kv));
    DPB_CHECK(check_rows(v, "v", cfg->total_k, cfg->heads_kv));
    DPB_CHECK(check_rows(o, "o", cfg->total_q, cfg->heads_q));
    DPB_CHECK(check_rows(grad_o, "grad_o", cfg->total_q, cfg->heads_q));
    DPB_CHECK(check_rows(grad_q, "grad_q", cfg->total_q, cfg->heads_q));
    DPB_CHECK(check_rows(grad_k, "grad_k", cfg->total_k, cfg->heads_kv));
    DPB_CHECK(check_rows(grad_v, "grad_v", cfg->total_k, cfg->heads_kv));
    DPB_CHECK(check_offsets(cfg, cu_q, cu_k));
    if (cfg->total_q > 0) DPB_CHECK(need(lse, "lse", 4));
    AttnArgs a{};
    DPB_CHECK(place_status(cfg->status_slot, workspace, workspace_bytes, attention_workspace(cfg), &a.status));
    fill_args(a, cfg, cu_q, cu_k);
    const GradSpace space(cfg);
    char *ws = static_cast<char *>(workspace);
    a.cap_k = space.cap_k, a.cap_q = space.cap_q, a.slots = space.slots;
    a.plan = reinterpret_cast<Plan *>(ws + space.plan);
    a.tasks_k = reinterpret_cast<Task *>(ws + space.tasks_k);
    a.tasks_q = reinterpret_cast<Task *>(ws + space.tasks_q);
    a.arrived = reinterpret_cast<int *>(ws + space.arrived);
    a.parts = reinterpret_cast<float *>(ws + space.parts);
    a.delta = reinterpret_cast<float *>(ws + space.delta);
    a.lse = const_cast<float *>(lse);
    a.o = in_rows(o);
    a.go = in_rows(grad_o);
    a.dq = out_rows(grad_q);
    a.dk = out_rows(grad_k);
    a.dv = out_rows(grad_v);
    const bool small = cfg->head_dim <= 64;
    const cudaStream_t s = static_cast<cudaStream_t>(stream);
    const int D = cfg->head_dim;
    DPB_CHECK(make_map(&a.q, q, cfg->total_q, cfg->heads_q, D, kRows));
    DPB_CHECK(make_map(&a.g, grad_o, cfg->total_q, cfg->heads_q, D, kRows));
    DPB_CHECK(make_map(&a.k, k, cfg->total_k, cfg->heads_kv, D, kRows));
    DPB_CHECK(make_map(&a.v, v, cfg->total_k, cfg->heads_kv, D, kRows));
    return small ? launch_attention_backward<Grad64>(a, s) : launch_attention_backward<Grad128>(a, s);
}

}  // extern "C"
