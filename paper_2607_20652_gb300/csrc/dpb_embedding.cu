// dpb_embedding.cu -- embedding lookup with a scale, and its gradient by sorted
// tokens.
//
//   y_t = scale W[id_t],   dW[v] = scale sum over id_t = v of dy_t
//
// Memory bounds the lookup (65536 tokens, 768 columns bf16: 31 us, 5.7 TB/s). The
// gradient sorts the tokens by their ids first (stable, so that a row's sum has
// the tokens' own order), in one cluster of blocks while the others write the
// zeros of dW, and then sums stretches of the sorted tokens: a warp each, whatever
// rows they belong to, so that a token met thousands of times costs no more than
// as many different ones. A row whose tokens lie in several stretches is joined
// from their partial sums in the stretches' order. No atomics on values: equal
// inputs give equal bits. 65536 tokens of 50257 words, frequent ones among them,
// take 53 us: the order 17, the sums some 21 to 30, as many different rows there are,
// the joins 4. Tokens that are written to memory where their digit puts them, without
// being brought together first, take 55 in all, as two words of 32 bits 59. 1000
// tokens still take 9 us to sort, waiting blocks for one another.
#include <algorithm>

#include "dpb_checks.h"
#include "dpb_device.cuh"
#include "dpb_rows.cuh"
#include "dpb_tensor_core.cuh"

namespace dpb {
namespace {

constexpr int kSortBlocks = 16;   // of the sorting cluster
constexpr int kSortWarps = 32;    // of a block
constexpr int kDigits = 256;      // 8 bits a pass
constexpr int kSumWarps = 4;      // of a summing block: few, so that an SM holds twelve of their 160 registers a lane
constexpr int kSumResident = 12;

// A token on its way: its id (vocab: none that counts) and its place.
struct alignas(8) Sorted {
    int id, token;
};

struct LookupArgs {
    const void *w, *dy;
    void *y, *dw;
    int64_t ws, ys, dys, dws;  // strides
    int64_t T;
    int V, d, passes, stretch;
    int64_t blocks;  // that have the stretches of tokens, a warp each
    float scale;
    Sorted *sorted[2];
    float *head, *tail;  // [blocks][d]: sums of the first row, begun before, and of the last, begun here and going on
    int *open;           // how many blocks' last rows go on, and which
    int32_t *status;
};

// ---- lookup -------------------------------------------------------------------------

// `lanes` lanes (a power of 2) copy a row.
template <typename E, int N, typename I>
__global__ void __launch_bounds__(256) embedding_kernel(const __grid_constant__ LookupArgs a, const I *ids, int lanes) {
    const int pieces = (a.d + N - 1) / N, in = threadIdx.x & (lanes - 1);
    const int64_t rows = (int64_t)gridDim.x * (256 / lanes);
    for (int64_t t = (int64_t)blockIdx.x * (256 / lanes) + threadIdx.x / lanes; t < a.T; t += rows) {
        const int64_t id = ids[t];
        const bool ok = id >= 0 && id < a.V;
        if (!ok && in == 0) set_status(a.status, DPB_DEV_BAD_INDEX);
        const E *w = static_cast<const E *>(a.w) + (ok ? id : 0) * a.ws;
        E *y = static_cast<E *>(a.y) + t * a.ys;
#pragma unroll 4
        for (int i = in; i < pieces; i += lanes) {
            Piece<E, N> v;
            load_piece(w + i * N, v);
#pragma unroll
            for (int j = 0; j < N; ++j) v.v[j] = ok ? v.v[j] * a.scale : 0.f;
            store_piece(y + i * N, v);
        }
    }
}

// ---- gradient: order, and zeros -------------------------------------------------------

__device__ __forceinline__ int read_peer(uint32_t addr) {
    int v;
    asm volatile("ld.shared::cluster.u32 %0, [%1];" : "=r"(v) : "r"(addr) : "memory");
    return v;
}

// The lanes with this lane's digit (-1: none; its answer then says nothing), by
// a vote for each bit (65536 tokens: 2 us less than by match.any).
__device__ __forceinline__ unsigned same_digit(int digit) {
    unsigned same = __ballot_sync(kFull, digit >= 0);
#pragma unroll
    for (int b = 0; b < 8; ++b) {
        const unsigned ones = __ballot_sync(kFull, (digit >> b) & 1);
        same &= (digit >> b) & 1 ? ones : ~ones;
    }
    return same;
}

// HELD: tokens of a lane under way; where that is all of them, they are read once a pass.
template <int HELD>
struct SortMemory {
    int count[kSortWarps][kDigits];
    Sorted stage[32 * HELD * kSortWarps];  // the block's tokens in their order, where they are still held
};
// of a warp: a multiple of 32
__host__ __device__ __forceinline__ int64_t tokens_of_warp(int64_t T) {
    const int64_t warps = kSortBlocks * kSortWarps;
    return ((T + warps - 1) / warps + 31) / 32 * 32;
}

// The first cluster sorts, a digit of 8 bits a pass: each warp counts the
// digits of its stretch of the tokens, the counts of all warps before it give
// each digit's first place, and it puts its tokens there in their order.
// The other clusters write zeros.
template <typename E, int N, typename I, int HELD>
__global__ void __launch_bounds__(32 * kSortWarps, 1) embedding_sort_kernel(const __grid_constant__ LookupArgs a, const I *ids) {
    const int tid = threadIdx.x, lane = tid & 31, warp = tid / 32;
    tc::start_next();
    if (blockIdx.x >= kSortBlocks) {
        const int pieces = (a.d + N - 1) / N;
        const int64_t warps = (int64_t)(gridDim.x - kSortBlocks) * kSortWarps;
        Piece<E, N> none;
#pragma unroll
        for (int j = 0; j < N; ++j) none.v[j] = 0.f;
        for (int64_t v = (int64_t)(blockIdx.x - kSortBlocks) * kSortWarps + warp; v < a.V; v += warps)
            for (int i = lane; i < pieces; i += 32) store_piece(static_cast<E *>(a.dw) + v * a.dws + i * N, none);
        return;
    }
    __shared__ int total[kDigits], shift[kDigits];
    __shared__ int2 sums[kDigits / 32];
    extern __shared__ __align__(8) uint8_t raw[];
    SortMemory<HELD> &memory = *reinterpret_cast<SortMemory<HELD> *>(raw);
    Sorted *const stage = memory.stage;
    int(*const count)[kDigits] = memory.count;
    const uint32_t rank = blockIdx.x;
    const int64_t each = tokens_of_warp(a.T);
    const int64_t t0 = min(a.T, (rank * kSortWarps + warp) * each), t1 = min(a.T, t0 + each);
    if (rank == 0 && tid == 0) *a.open = 0;
    for (int pass = 0; pass < a.passes; ++pass) {
        const Sorted *from = a.sorted[(pass & 1) ^ 1];
        Sorted *to = a.sorted[pass & 1];
        Sorted x[HELD];
        int place[HELD];  // among the warp's tokens of the same digit
        auto digit = [&](int id) { return id < 0 ? -1 : (id >> (8 * pass)) & 255; };
        // the tokens from t on, and their places behind those that `count` has
        auto load = [&](int64_t t) {
#pragma unroll
            for (int k = 0; k < HELD; ++k) {
                const int64_t at = t + 32 * k + lane;
                x[k] = Sorted{-1, 0};
                if (at >= t1) continue;
                if (pass > 0) {
                    x[k] = from[at];
                } else {
                    const int64_t id = ids[at];
                    const bool ok = id >= 0 && id < a.V;
                    if (!ok) set_status(a.status, DPB_DEV_BAD_INDEX);
                    x[k] = Sorted{ok ? (int)id : a.V, (int)at};
                }
            }
#pragma unroll
            for (int k = 0; k < HELD; ++k) {
                if (t + 32 * k >= t1) break;
                const int g = digit(x[k].id);
                const unsigned same = same_digit(g);
                place[k] = g >= 0 ? count[warp][g] + __popc(same & ((1u << lane) - 1)) : 0;
                __syncwarp();
                if (g >= 0 && lane == __ffs(same) - 1) count[warp][g] += __popc(same);
                __syncwarp();
            }
        };
        for (int i = tid; i < kSortWarps * kDigits; i += 32 * kSortWarps) count[0][i] = 0;
        __syncthreads();
        for (int64_t t = t0; t < t1; t += 32 * HELD) load(t);
        __syncthreads();
        if (tid < kDigits) {  // the block's warps before each
            int n = 0;
#pragma unroll 8
            for (int w = 0; w < kSortWarps; ++w) {
                const int c = count[w][tid];
                count[w][tid] = n;
                n += c;
            }
            total[tid] = n;
        }
        tc::cluster_sync();
        // A digit's first place in the block and in all. Tokens still held go by way of
        // shared memory, so that neighbours there, mostly of the same digit, are written
        // to memory side by side.
        const bool held = each <= 32 * HELD;
        int before = 0, all = 0, mine = 0;
        int2 upto;
        if (tid < kDigits) {
            const uint32_t at = tc::smem_addr(&total[tid]);
            mine = total[tid];
#pragma unroll
            for (uint32_t r = 0; r < kSortBlocks; ++r) {
                const int n = read_peer(tc::peer_addr(at, r));
                if (r < rank) before += n;
                all += n;
            }
            upto = make_int2(mine, all);
#pragma unroll
            for (int i = 1; i < 32; i *= 2) {
                const int2 n = make_int2(__shfl_up_sync(kFull, upto.x, i), __shfl_up_sync(kFull, upto.y, i));
                if (lane >= i) upto.x += n.x, upto.y += n.y;
            }
            if (lane == 31) sums[warp] = upto;
        }
        __syncthreads();
        if (tid < kDigits) {
            int here = upto.x - mine, first = upto.y - all + before;
            for (int w = 0; w < warp; ++w) here += sums[w].x, first += sums[w].y;
            shift[tid] = first - here;
#pragma unroll 8
            for (int w = 0; w < kSortWarps; ++w) count[w][tid] += held ? here : first;
        }
        __syncthreads();
        if (held) {  // their places in the warp from 0
#pragma unroll
            for (int k = 0; k < HELD; ++k)
                if (x[k].id >= 0 && t0 < t1) stage[count[warp][digit(x[k].id)] + place[k]] = x[k];
            __syncthreads();
            const int64_t first = min(a.T, rank * kSortWarps * each);
            const int n = (int)(min(a.T, first + kSortWarps * each) - first);
            for (int i = tid; i < n; i += 32 * kSortWarps) {
                const Sorted token = stage[i];
                to[i + shift[digit(token.id)]] = token;
            }
        } else {
            for (int64_t t = t0; t < t1; t += 32 * HELD) {
                load(t);
#pragma unroll
                for (int k = 0; k < HELD; ++k)
                    if (x[k].id >= 0) to[place[k]] = x[k];
            }
        }
        // the others have read this block's totals, and all tokens are in place
        tc::cluster_sync();
    }
}

// ---- gradient: sums ---------------------------------------------------------------------

// A warp sums one stretch of the sorted tokens over 32 P N columns, the next
// rows under way while it adds some. What it has of a row that does not begin
// and end in its stretch is added up over the block's stretches, in their order.
template <typename E, int N, int P>
__global__ void __launch_bounds__(32 * kSumWarps) embedding_sum_kernel(const __grid_constant__ LookupArgs a) {
    constexpr int kColumns = 32 * P * N;
    __shared__ float part[kSumWarps][2][kColumns];  // of the first row, begun before, and of the last, going on
    struct Ends {
        int head, tail;  // those rows' ids, or -1
        bool through;    // the first row goes on behind the stretch
    };
    __shared__ Ends ends[kSumWarps];
    tc::start_next();
    tc::wait_previous();
    const int lane = threadIdx.x & 31, warp = threadIdx.x / 32;
    const int64_t c = (int64_t)blockIdx.x * kSumWarps + warp;
    const Sorted *sorted = a.sorted[(a.passes - 1) & 1];
    const int64_t p0 = min(a.T, c * a.stretch), p1 = min(a.T, p0 + a.stretch);
    const int column = blockIdx.y * kColumns + lane * N;
    float acc[P][N];
    auto clear = [&] {
#pragma unroll
        for (int p = 0; p < P; ++p)
#pragma unroll
            for (int j = 0; j < N; ++j) acc[p][j] = 0.f;
    };
    clear();
    int id = -1;
    bool whole = true;  // the row's tokens begin in this stretch
    const int prev = p0 > 0 && p0 < p1 ? sorted[p0 - 1].id : -1, next = p0 < p1 && p1 < a.T ? sorted[p1].id : -1;
    auto flush = [&](bool complete) {
        if (id < 0 || id >= a.V) return;
#pragma unroll
        for (int p = 0; p < P; ++p) {
            const int i = column + p * 32 * N;
            if (i >= a.d) continue;
            if (whole && complete) {
                Piece<E, N> v;
#pragma unroll
                for (int j = 0; j < N; ++j) v.v[j] = acc[p][j] * a.scale;
                store_piece(static_cast<E *>(a.dw) + id * a.dws + i, v);
            } else {
#pragma unroll
                for (int j = 0; j < N; ++j) part[warp][whole][(lane + 32 * p) * N + j] = acc[p][j];
            }
        }
    };
    constexpr int kAtOnce = 4;
    for (int64_t b = p0; b < p1; b += 32) {
        const int n = (int)min((int64_t)32, p1 - b);
        const Sorted mine = lane < n ? sorted[b + lane] : Sorted{-1, 0};  // places past the end read row 0
        Bits<E, N> rows[2][kAtOnce][P];
        auto load = [&](int k0, Bits<E, N> (&to)[kAtOnce][P]) {
#pragma unroll
            for (int k = 0; k < kAtOnce; ++k) {
                const int64_t t = __shfl_sync(kFull, mine.token, (k0 + k) & 31);
                const E *dy = static_cast<const E *>(a.dy) + t * a.dys;
#pragma unroll
                for (int p = 0; p < P; ++p) load_bits(dy + (column + p * 32 * N < a.d ? column + p * 32 * N : 0), to[k][p]);
            }
        };
        auto add = [&](int k0, const Bits<E, N> (&from)[kAtOnce][P]) {
#pragma unroll
            for (int k = 0; k < kAtOnce; ++k) {
                const int now = __shfl_sync(kFull, mine.id, (k0 + k) & 31);
                if (k0 + k >= n) break;
                if (now != id) {
                    flush(true);
                    clear();
                    id = now;
                    whole = b + k0 + k > p0 || id != prev;
                }
#pragma unroll
                for (int p = 0; p < P; ++p) {
                    const Piece<E, N> v = values(from[k][p]);
#pragma unroll
                    for (int j = 0; j < N; ++j) acc[p][j] += v.v[j];
                }
            }
        };
        load(0, rows[0]);
        for (int k0 = 0; k0 < n; k0 += 2 * kAtOnce) {
            if (k0 + kAtOnce < n) load(k0 + kAtOnce, rows[1]);
            add(k0, rows[0]);
            if (k0 + 2 * kAtOnce < n) load(k0 + 2 * kAtOnce, rows[0]);
            if (k0 + kAtOnce < n) add(k0 + kAtOnce, rows[1]);
        }
    }
    flush(id != next);
    if (lane == 0) {
        const int first = p0 < p1 && sorted[p0].id == prev && prev < a.V ? prev : -1;
        ends[warp] = Ends{first, whole && id >= 0 && id < a.V && id == next ? id : -1, !whole && id == next};
    }
    __syncthreads();
    const int columns = min(kColumns, a.d - (int)blockIdx.y * kColumns);
    for (int i = threadIdx.x; i < columns; i += 32 * kSumWarps) {
        const int64_t at = (int64_t)blockIdx.y * kColumns + i;
        float sum = 0.f;
        bool before = true;  // the row began before the block
        bool open = false;   // and goes on
        for (int w = 0; w < kSumWarps; ++w) {
            const Ends e = ends[w];
            if (e.head >= 0) {
                sum += part[w][0][i];
                open = e.through;
                if (!open && before) a.head[blockIdx.x * (int64_t)a.d + at] = sum;
                if (!open && !before) st_elem(static_cast<E *>(a.dw), e.head * a.dws + at, sum * a.scale);
            }
            if (e.tail >= 0) sum = part[w][1][i], before = false, open = true;
        }
        if (open) (before ? a.head : a.tail)[blockIdx.x * (int64_t)a.d + at] = sum;
        if (open && !before && at == 0) a.open[1 + atomicAdd(a.open, 1)] = (int)blockIdx.x;
    }
}

// The rows whose tokens go on after the block where they begin: the sum of what
// each block has of them. A warp has 32 M columns of one at a time.
constexpr int kJoinWarps = 4;
template <typename E, int M>
__global__ void __launch_bounds__(32 * kJoinWarps) embedding_join_kernel(const __grid_constant__ LookupArgs a, int groups) {
    tc::wait_previous();
    const int lane = threadIdx.x & 31;
    const int64_t warps = (int64_t)gridDim.x * kJoinWarps, items = (int64_t)*a.open * groups;
    const Sorted *sorted = a.sorted[(a.passes - 1) & 1];
    const int64_t each = (int64_t)a.stretch * kSumWarps;  // tokens of a block
    for (int64_t w = (int64_t)blockIdx.x * kJoinWarps + threadIdx.x / 32; w < items; w += warps) {
        const int64_t c = a.open[1 + w / groups];
        const int id = sorted[(c + 1) * each].id, i = ((int)(w % groups) * 32 + lane) * M;
        const bool live = i < a.d;
        auto at = [&](const float *from, int64_t k) {
            Piece<float, M> x;
            load_piece(from + k * a.d + (live ? i : 0), x);
            return x;
        };
        Piece<float, M> sum = at(a.tail, c);
        constexpr int kAtOnce = 16;
        for (int64_t k = c + 1; k < a.blocks; k += kAtOnce) {
            // which of the next blocks begin with the row, and their sums at the same time
            const int64_t mine = min(k + lane, a.blocks - 1);
            Piece<float, M> x[kAtOnce];
            const bool has = lane < kAtOnce && k + lane < a.blocks && sorted[mine * each].id == id;
#pragma unroll
            for (int j = 0; j < kAtOnce; ++j) x[j] = at(a.head, min(k + j, a.blocks - 1));
            const int n = __popc(__ballot_sync(kFull, has));
#pragma unroll
            for (int j = 0; j < kAtOnce; ++j)
                if (j < n)
#pragma unroll
                    for (int m = 0; m < M; ++m) sum.v[m] += x[j].v[m];
            if (n < kAtOnce) break;
        }
        if (live)
#pragma unroll
            for (int m = 0; m < M; ++m) st_elem(static_cast<E *>(a.dw), id * a.dws + i + m, sum.v[m] * a.scale);
    }
}

// ---- host side ------------------------------------------------------------------

int passes_of(int V) {
    int n = 1;
    while (n < 4 && ((int64_t)1 << (8 * n)) <= V) ++n;  // ids up to V
    return n;
}

struct GradSpace {
    int stretch;
    int64_t blocks;
    size_t sorted[2], head, tail, open, bytes;
    explicit GradSpace(const dpb_embedding_config *c) {
        // As many stretches as warps are resident, of 8 tokens at least and 64 at most.
        const int64_t warps = (int64_t)kSumResident * sms_of_device();
        stretch = (int)std::max<int64_t>(8, std::min<int64_t>(64, (c->tokens + warps - 1) / warps));
        blocks = ((c->tokens + stretch - 1) / stretch + kSumWarps - 1) / kSumWarps;
        auto up = [](size_t n) { return (n + 255) / 256 * 256; };
        sorted[0] = kStatusBytes;
        sorted[1] = sorted[0] + up((size_t)c->tokens * sizeof(Sorted));
        head = sorted[1] + up((size_t)c->tokens * sizeof(Sorted));
        tail = head + up((size_t)blocks * c->dim * 4);
        open = tail + up((size_t)blocks * c->dim * 4);
        bytes = open + up(((size_t)blocks + 1) * 4);
    }
};

dpb_status check_config(const dpb_embedding_config *c) {
    if (!c) return fail(DPB_ERR_INVALID_ARG, "cfg is NULL");
    if (c->dtype != DPB_F32 && c->dtype != DPB_BF16) return fail(DPB_ERR_INVALID_ARG, "dtype must be DPB_F32 or DPB_BF16");
    if (c->tokens < 0 || c->vocab < 1 || c->dim < 1) return fail(DPB_ERR_INVALID_ARG, "a size is too small");
    if (c->tokens > 0x7fffff00ll || c->vocab > 0x7fffff00 || c->dim > (1 << 20))
        return fail(DPB_ERR_UNSUPPORTED, "at most 2^31 - 256 tokens and words, 2^20 columns");
    if (c->index_bytes != 4 && c->index_bytes != 8) return fail(DPB_ERR_INVALID_ARG, "index_bytes must be 4 or 8");
    if (!(c->scale - c->scale == 0.f)) return fail(DPB_ERR_INVALID_ARG, "scale must be finite");
    return check_slot(c->status_slot);
}

dpb_status check_rows(const dpb_embedding_config *c, const dpb_rows *r, int64_t n, const char *name) {
    if (n == 0) return DPB_OK;
    if (!r) return fail(DPB_ERR_INVALID_ARG, "%s is NULL", name);
    DPB_CHECK(need(r->data, name, c->dtype == DPB_F32 ? 4 : 2));
    if (n > 1 && r->stride < c->dim) return fail(DPB_ERR_INVALID_ARG, "the stride of %s must be at least dim", name);
    return DPB_OK;
}

template <typename E, int N>
dpb_status lookup(const LookupArgs &a, const void *ids, int index_bytes, cudaStream_t s) {
    const int pieces = (a.d + N - 1) / N;
    int lanes = 1;
    while (lanes < 32 && lanes < pieces) lanes *= 2;
    const unsigned blocks = (unsigned)std::min<int64_t>((a.T * lanes + 255) / 256, 1 << 20);
    if (index_bytes == 4)
        embedding_kernel<E, N><<<blocks, 256, 0, s>>>(a, static_cast<const int32_t *>(ids), lanes);
    else
        embedding_kernel<E, N><<<blocks, 256, 0, s>>>(a, static_cast<const int64_t *>(ids), lanes);
    return launch_status(cudaGetLastError(), "embedding");
}

template <typename E, int N, int P>
cudaError_t sums(const LookupArgs &a, cudaStream_t s) {
    const dim3 grid((unsigned)a.blocks, (unsigned)((a.d + 32 * P * N - 1) / (32 * P * N)));
    return launch_early(embedding_sum_kernel<E, N, P>, grid, 32 * kSumWarps, 0, s, a);
}

template <typename E, int N, int HELD, typename I>
cudaError_t sort_held(const LookupArgs &a, const I *ids, cudaStream_t s) {
    void (*const kernel)(const LookupArgs, const I *) = embedding_sort_kernel<E, N, I, HELD>;
    cudaLaunchConfig_t how{};
    how.gridDim = how.blockDim = dim3(32 * kSortWarps);
    how.dynamicSmemBytes = sizeof(SortMemory<HELD>);
    how.stream = s;
    cudaLaunchAttribute cluster{};
    cluster.id = cudaLaunchAttributeClusterDimension;
    cluster.val.clusterDim.x = kSortBlocks;
    cluster.val.clusterDim.y = cluster.val.clusterDim.z = 1;
    how.attrs = &cluster;
    how.numAttrs = 1;
    int resident;
    cudaError_t e = resident_clusters(reinterpret_cast<const void *>(kernel), how, &resident);
    if (e != cudaSuccess) return e;
    // Those that write zeros, all at the same time: with one cluster more than the device holds (152 SMs, 7 clusters)
    // the last starts when others end, and 50257 rows of 768 take 24 us where the order takes 17.
    const int others = std::max(1, std::min(resident - 1, (a.V + 32 * kSortBlocks - 1) / (32 * kSortBlocks)));
    how.gridDim = dim3(kSortBlocks * (1 + others));
    e = cudaLaunchKernelEx(&how, kernel, a, ids);
    return e == cudaSuccess ? cudaGetLastError() : e;
}

// Eight tokens a lane where four are not all of them and eight are: 131072 x 768
// 103 us, 113 with four, which read the tokens twice; 65536 x 768 54 and 53.5,
// 300000 x 768, where neither is enough, 195 and 189.
template <typename E, int N, typename I>
cudaError_t sort(const LookupArgs &a, const I *ids, cudaStream_t s) {
    const int64_t each = tokens_of_warp(a.T);
    return each > 32 * 4 && each <= 32 * 8 ? sort_held<E, N, 8>(a, ids, s) : sort_held<E, N, 4>(a, ids, s);
}

template <typename E, int N>
dpb_status gradient(const LookupArgs &a, const void *ids, int index_bytes, cudaStream_t s) {
    DPB_CHECK(launch_status(index_bytes == 4 ? sort<E, N>(a, static_cast<const int32_t *>(ids), s)
                                             : sort<E, N>(a, static_cast<const int64_t *>(ids), s),
                            "embedding_backward (order)"));
    const int pieces = (a.d + 32 * N - 1) / (32 * N);  // of a lane
    cudaError_t e;
    if (pieces == 1) e = sums<E, N, 1>(a, s);
    else if (pieces == 2 || pieces == 4) e = sums<E, N, 2>(a, s);
    else e = sums<E, N, 3>(a, s);
    DPB_CHECK(launch_status(e, "embedding_backward (sums)"));
    constexpr int M = N == 1 ? 1 : 4;
    const int groups = (a.d + 32 * M - 1) / (32 * M);
    const int64_t items = a.blocks * groups;
    const unsigned blocks = (unsigned)std::min<int64_t>((items + kJoinWarps - 1) / kJoinWarps, 4 * sms_of_device());
    return launch_status(launch_early(embedding_join_kernel<E, M>, dim3(blocks), 32 * kJoinWarps, 0, s, a, groups),
                         "embedding_backward (rows)");
}

}  // namespace
}  // namespace dpb

using namespace dpb;

extern "C" {

dpb_status dpb_embedding(const dpb_embedding_config *cfg, const dpb_rows *weight, const void *ids, const dpb_rows *y,
                         void *workspace, size_t workspace_bytes, void *stream) {
    DPB_CHECK(check_config(cfg));
    if (cfg->tokens == 0) return DPB_OK;
    DPB_CHECK(check_rows(cfg, weight, cfg->vocab, "weight"));
    DPB_CHECK(check_rows(cfg, y, cfg->tokens, "y"));
    DPB_CHECK(need(ids, "ids", cfg->index_bytes));
    LookupArgs a{};
    DPB_CHECK(place_status(cfg->status_slot, workspace, workspace_bytes, kStatusBytes, &a.status));
    a.w = weight->data, a.ws = weight->stride;
    a.y = y->data, a.ys = y->stride;
    a.T = cfg->tokens, a.V = cfg->vocab, a.d = cfg->dim, a.scale = cfg->scale;
    const int elem = cfg->dtype == DPB_F32 ? 4 : 2;
    const bool pieces = by_pieces(a.w, a.ws, a.V, elem) && by_pieces(a.y, a.ys, a.T, elem) && a.d * elem % 16 == 0;
    const cudaStream_t s = static_cast<cudaStream_t>(stream);
    using bf16 = __nv_bfloat16;
    if (cfg->dtype == DPB_F32)
        return pieces ? lookup<float, 4>(a, ids, cfg->index_bytes, s) : lookup<float, 1>(a, ids, cfg->index_bytes, s);
    return pieces ? lookup<bf16, 8>(a, ids, cfg->index_bytes, s) : lookup<bf16, 1>(a, ids, cfg->index_bytes, s);
}

dpb_status dpb_embedding_workspace_size(const dpb_embedding_config *cfg, size_t *bytes) {
    DPB_CHECK(check_config(cfg));
    if (!bytes) return fail(DPB_ERR_INVALID_ARG, "bytes is NULL");
    *bytes = GradSpace(cfg).bytes;
    return DPB_OK;
}

dpb_status dpb_embedding_backward(const dpb_embedding_config *cfg, const dpb_rows *grad_y, const void *ids,
                                  const dpb_rows *grad_weight, void *workspace, size_t workspace_bytes, void *stream) {
    DPB_CHECK(check_config(cfg));
    DPB_CHECK(check_rows(cfg, grad_weight, cfg->vocab, "grad_weight"));
    const int elem = cfg->dtype == DPB_F32 ? 4 : 2;
    const cudaStream_t s = static_cast<cudaStream_t>(stream);
    if (cfg->tokens == 0)
        return launch_status(cudaMemset2DAsync(grad_weight->data, (cfg->vocab > 1 ? grad_weight->stride : cfg->dim) * elem, 0,
                                               (size_t)cfg->dim * elem, cfg->vocab, s),
                             "embedding_backward");
    DPB_CHECK(check_rows(cfg, grad_y, cfg->tokens, "grad_y"));
    DPB_CHECK(need(ids, "ids", cfg->index_bytes));
    const GradSpace w(cfg);
    LookupArgs a{};
    DPB_CHECK(place_status(cfg->status_slot, workspace, workspace_bytes, w.bytes, &a.status));
    uint8_t *ws = static_cast<uint8_t *>(workspace);
    a.dy = grad_y->data, a.dys = grad_y->stride;
    a.dw = grad_weight->data, a.dws = grad_weight->stride;
    a.T = cfg->tokens, a.V = cfg->vocab, a.d = cfg->dim, a.scale = cfg->scale;
    a.passes = passes_of(a.V);
    a.stretch = w.stretch, a.blocks = w.blocks;
    for (int i = 0; i < 2; ++i) a.sorted[i] = reinterpret_cast<Sorted *>(ws + w.sorted[i]);
    a.head = reinterpret_cast<float *>(ws + w.head);
    a.tail = reinterpret_cast<float *>(ws + w.tail);
    a.open = reinterpret_cast<int *>(ws + w.open);
    const bool pieces = by_pieces(a.dy, a.dys, a.T, elem) && by_pieces(a.dw, a.dws, a.V, elem) && a.d * elem % 16 == 0;
    using bf16 = __nv_bfloat16;
    if (cfg->dtype == DPB_F32)
        return pieces ? gradient<float, 4>(a, ids, cfg->index_bytes, s) : gradient<float, 1>(a, ids, cfg->index_bytes, s);
    return pieces ? gradient<bf16, 8>(a, ids, cfg->index_bytes, s) : gradient<bf16, 1>(a, ids, cfg->index_bytes, s);
}

}  // extern "C"
