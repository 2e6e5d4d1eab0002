// dpb_norm.cu -- the residual's addition and the RMS norm behind it, and their
// gradient.
//
//   s = x + delta (rounded to the rows' type),  y = w s r,  r = (mean s^2 + eps)^(-1/2)
//   u = w dy,  h = s r,  dx = ds + r (u - h mean(u h)),  dw = sum_t dy h
//
// Memory bounds both: a row is read once and kept until its sum is known, and the
// next row is loaded meanwhile (65536 x 768 bf16: 64 us, 6.3 TB/s; 111 without). A
// warp has a row where its lanes can hold it, up to 1024 threads where not. The
// gradient's threads keep their columns' dw over all rows of their block, and the
// blocks' sums are added up in the blocks' order; its rows on their way are in
// shared memory (65536 x 768 bf16: 74 us, 5.4 TB/s; 49999 x 1000 76; 32768 x 768
// fp32 71; 16384 x 4096 bf16 87; 10000 x 16384 fp32 390; with them in registers 81,
// 79, 85, 114 and 745). Of each some 3 us are for dw; summed up a warp after the
// other, waiting for each, a block's took 4 us more at 49999 x 1000.
//
// Rows that do not lie in pieces of 16 bytes go value by value, in registers: 20000
// x 777 bf16 takes 56 us and 106 for the gradient, 3.1 and 5.8 times what its bytes
// need, 5000 x 5001 116 and 155 (3.9 and 5.3). From 8193 values on such a row's 1024
// threads have too few registers and spill (up to 870 bytes a thread, 592 in the
// gradient).
#include <algorithm>

#include "dpb_checks.h"
#include "dpb_device.cuh"
#include "dpb_rows.cuh"
#include "dpb_tensor_core.cuh"

namespace dpb {
namespace {

constexpr int kMostDim = 16384;
constexpr int kGradBlocks = 4;  // of an SM, at most, in the gradient

struct NormArgs {
    const void *x, *delta, *w, *dy, *ds;
    void *y, *s, *dx;
    int64_t xs, deltas, dys, dss, ys, ss, dxs;  // strides
    float *dw, *part;
    int64_t T;
    int d, blocks;
    float eps;
};

// The sums of two values over a row's threads (part of a warp, or whole warps); all of the block's threads call it.
__device__ __forceinline__ float2 row_sums(float2 v, int row_threads, float2 *sums) {
#pragma unroll
    for (int i = 16; i > 0; i /= 2) {
        if (i >= row_threads) continue;
        v.x += __shfl_xor_sync(kFull, v.x, i);
        v.y += __shfl_xor_sync(kFull, v.y, i);
    }
    if (row_threads <= 32) return v;
    const int row_warps = row_threads / 32, warp = threadIdx.x / 32, first = warp / row_warps * row_warps;
    if ((threadIdx.x & 31) == 0) sums[warp] = v;
    __syncthreads();
    v = make_float2(0.f, 0.f);
    for (int i = 0; i < row_warps; ++i) v.x += sums[first + i].x, v.y += sums[first + i].y;
    __syncthreads();
    return v;
}

// P pieces of a row, one of each row_threads.
template <typename E, int N, int P>
__device__ __forceinline__ void load_row(Bits<E, N> (&r)[P], const void *data, int64_t stride, int64_t t, bool live, int in,
                                         int row_threads, int d) {
    const E *row = static_cast<const E *>(data) + t * stride;
#pragma unroll
    for (int p = 0; p < P; ++p) {
        const int i = (in + p * row_threads) * N;
        r[p] = Bits<E, N>{};
        if (live && i < d) load_bits(row + i, r[p]);
    }
}

// Each row's threads load the next row while they work on one.
template <typename E, int N, int P, int MOST>
__global__ void __launch_bounds__(MOST) add_norm_kernel(const __grid_constant__ NormArgs a, int row_threads) {
    __shared__ float2 sums[32];
    const int in = threadIdx.x % row_threads, rows = MOST / row_threads;
    const int64_t step = (int64_t)gridDim.x * rows;
    int64_t t = (int64_t)blockIdx.x * rows + threadIdx.x / row_threads;
    Bits<E, N> w[P], x[P], delta[P];
    if (a.w) load_row(w, a.w, 0, 0, true, in, row_threads, a.d);
    load_row(x, a.x, a.xs, t, t < a.T, in, row_threads, a.d);
    if (a.delta) load_row(delta, a.delta, a.deltas, t, t < a.T, in, row_threads, a.d);
    // every thread of the block makes the same number of turns
    for (int64_t t0 = (int64_t)blockIdx.x * rows; t0 < a.T; t0 += step, t += step) {
        const bool live = t < a.T;
        Piece<E, N> v[P];
        float sum = 0.f;
#pragma unroll
        for (int p = 0; p < P; ++p) {
            v[p] = values(x[p]);
            if (a.delta) {
                const Piece<E, N> more = values(delta[p]);
#pragma unroll
                for (int j = 0; j < N; ++j) {
                    v[p].v[j] += more.v[j];
                    if (sizeof(E) == 2) v[p].v[j] = __bfloat162float(__float2bfloat16_rn(v[p].v[j]));
                }
            }
#pragma unroll
            for (int j = 0; j < N; ++j) sum = fmaf(v[p].v[j], v[p].v[j], sum);
        }
        load_row(x, a.x, a.xs, t + step, t + step < a.T, in, row_threads, a.d);
        if (a.delta) load_row(delta, a.delta, a.deltas, t + step, t + step < a.T, in, row_threads, a.d);
        sum = row_sums(make_float2(sum, 0.f), row_threads, sums).x;
        const float r = rsqrtf(sum / a.d + a.eps);
        E *s = static_cast<E *>(a.s) + t * a.ss, *y = static_cast<E *>(a.y) + t * a.ys;
#pragma unroll
        for (int p = 0; p < P; ++p) {
            const int i = (in + p * row_threads) * N;
            if (!live || i >= a.d) continue;
            if (a.s) store_piece(s + i, v[p]);
            const Piece<E, N> k = values(w[p]);
#pragma unroll
            for (int j = 0; j < N; ++j) v[p].v[j] = v[p].v[j] * r * (a.w ? k.v[j] : 1.f);
            store_piece(y + i, v[p]);
        }
    }
}

__device__ __forceinline__ void copy_piece(void *to, const void *from) {
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(tc::smem_addr(to)), "l"(from) : "memory");
}

// Where a thread's pieces of a row's three rows are until they are used: pieces of
// 16 bytes in places of its own in shared memory, kStages rows on their way, which
// its registers would not hold; single values in registers, read when they are used.
template <typename E, int N, int P, int MOST>
struct GradRows {
    static constexpr bool kCopied = N > 1;
    static constexpr int kStages = (P == 4 ? 2 : 3) - (MOST == 1024);  // two blocks an SM, one of the widest rows
    static constexpr size_t kBytes = kCopied ? (size_t)kStages * 3 * P * MOST * 16 : 0;
    uint8_t *mem;
    int in, row_threads, slot = 0, filled = 0;
    Bits<E, N> now[kCopied ? 1 : 3][kCopied ? 1 : P];
    __device__ __forceinline__ uint8_t *place(int at, int array, int p) const {
        return mem + (((at * 3 + array) * P + p) * MOST + threadIdx.x) * 16;
    }
    __device__ __forceinline__ void init() {
        if constexpr (kCopied)  // places behind the row's end stay 0
            for (int k = 0; k < kStages * 3 * P; ++k)
                *reinterpret_cast<uint4 *>(mem + (k * MOST + threadIdx.x) * 16) = make_uint4(0, 0, 0, 0);
    }
    // Asks for row t.
    __device__ __forceinline__ void ask(const NormArgs &a, int64_t t) {
        if constexpr (kCopied) {
            if (t < a.T) {
                const E *s = static_cast<const E *>(a.x) + t * a.xs, *dy = static_cast<const E *>(a.dy) + t * a.dys;
                const E *ds = static_cast<const E *>(a.ds) + t * a.dss;
#pragma unroll
                for (int p = 0; p < P; ++p) {
                    const int i = (in + p * row_threads) * N;
                    if (i >= a.d) continue;
                    copy_piece(place(filled, 0, p), s + i);
                    copy_piece(place(filled, 1, p), dy + i);
                    if (a.ds) copy_piece(place(filled, 2, p), ds + i);
                }
            }
            asm volatile("cp.async.commit_group;" ::: "memory");
            filled = filled + 1 == kStages ? 0 : filled + 1;
        }
    }
    // The oldest row asked for, t, is there.
    __device__ __forceinline__ void take(const NormArgs &a, int64_t t) {
        if constexpr (kCopied) {
            asm volatile("cp.async.wait_group %0;" ::"n"(kStages - 1) : "memory");
        } else {
            load_row(now[0], a.x, a.xs, t, t < a.T, in, row_threads, a.d);
            load_row(now[1], a.dy, a.dys, t, t < a.T, in, row_threads, a.d);
            if (a.ds) load_row(now[2], a.ds, a.dss, t, t < a.T, in, row_threads, a.d);
        }
    }
    __device__ __forceinline__ Piece<E, N> get(int array, int p) const {
        if constexpr (kCopied) {
            Bits<E, N> b;
            b.w = *reinterpret_cast<const uint4 *>(place(slot, array, p));
            return values(b);
        } else {
            return values(now[array][p]);
        }
    }
    __device__ __forceinline__ void next() { slot = slot + 1 == kStages ? 0 : slot + 1; }
};

template <typename E, int N, int P, int MOST>
__global__ void __launch_bounds__(MOST, N > 1 && MOST == 256 ? 2 : 1)
    add_norm_grad_kernel(const __grid_constant__ NormArgs a, int row_threads) {
    __shared__ float2 sums[32];
    extern __shared__ __align__(16) uint8_t mem[];
    tc::start_next();
    const int in = threadIdx.x % row_threads, rows = MOST / row_threads;
    const int64_t step = (int64_t)gridDim.x * rows;
    int64_t t = (int64_t)blockIdx.x * rows + threadIdx.x / row_threads;
    float dw[P][N];
#pragma unroll
    for (int p = 0; p < P; ++p)
#pragma unroll
        for (int j = 0; j < N; ++j) dw[p][j] = 0.f;
    Bits<E, N> w[P];
    if (a.w) load_row(w, a.w, 0, 0, true, in, row_threads, a.d);
    GradRows<E, N, P, MOST> row{mem, in, row_threads};
    constexpr int kStages = GradRows<E, N, P, MOST>::kStages;
    row.init();
    for (int k = 0; k < kStages - 1; ++k) row.ask(a, t + k * step);
    // every thread of the block makes the same number of turns
    for (int64_t t0 = (int64_t)blockIdx.x * rows; t0 < a.T; t0 += step, t += step) {
        const bool live = t < a.T;
        row.ask(a, t + (kStages - 1) * step);
        row.take(a, t);
        float sq = 0.f, us = 0.f;
#pragma unroll
        for (int p = 0; p < P; ++p) {
            const Piece<E, N> v = row.get(0, p), g = row.get(1, p), k = values(w[p]);
#pragma unroll
            for (int j = 0; j < N; ++j) {
                sq = fmaf(v.v[j], v.v[j], sq);
                us = fmaf(a.w ? g.v[j] * k.v[j] : g.v[j], v.v[j], us);
            }
        }
        const float2 both = row_sums(make_float2(sq, us), row_threads, sums);
        // with h = total r: factors of the result's own size, where r^3 leaves fp32 at rows beyond 1e14 or below 1e-13
        const float r = rsqrtf(both.x / a.d + a.eps), along = r * (both.y / a.d);  // mean(u h)
        E *dx = static_cast<E *>(a.dx) + t * a.dxs;
#pragma unroll
        for (int p = 0; p < P; ++p) {
            const int i = (in + p * row_threads) * N;
            if (!live || i >= a.d) continue;
            Piece<E, N> v = row.get(0, p), rest;
            const Piece<E, N> g = row.get(1, p), k = values(w[p]);
            if (a.ds) rest = row.get(2, p);
#pragma unroll
            for (int j = 0; j < N; ++j) {
                const float h = v.v[j] * r;
                dw[p][j] = fmaf(g.v[j], h, dw[p][j]);
                v.v[j] = fmaf(r, fmaf(-along, h, a.w ? g.v[j] * k.v[j] : g.v[j]), a.ds ? rest.v[j] : 0.f);
            }
            store_piece(dx + i, v);
        }
        row.next();
    }
    if (!a.part) return;
    // the block's rows one after the other
    float *columns = reinterpret_cast<float *>(mem);  // [rows][d]
    asm volatile("cp.async.wait_all;" ::: "memory");
    __syncthreads();
#pragma unroll
    for (int p = 0; p < P; ++p) {
        const int i = (in + p * row_threads) * N;
        float *to = columns + (int)threadIdx.x / row_threads * a.d + i;
        if (i >= a.d) continue;
        if constexpr (N == 1) {
            *to = dw[p][0];
        } else {
#pragma unroll
            for (int j = 0; j < N; j += 4)
                *reinterpret_cast<float4 *>(to + j) = make_float4(dw[p][j], dw[p][j + 1], dw[p][j + 2], dw[p][j + 3]);
        }
    }
    __syncthreads();
    for (int i = threadIdx.x; i < a.d; i += MOST) {
        float sum = columns[i];
        for (int q = 1; q < rows; ++q) sum += columns[q * a.d + i];
        a.part[(int64_t)blockIdx.x * a.d + i] = sum;
    }
}

// 32 columns of all blocks' sums: 32 threads a column, each its blocks in
// order, then the threads.
__global__ void __launch_bounds__(1024) add_norm_columns_kernel(const NormArgs a) {
    __shared__ float sums[32][33];
    tc::wait_previous();
    const int lane = threadIdx.x & 31, slice = threadIdx.x / 32, i = blockIdx.x * 32 + lane;
    float v = 0.f;
    if (i < a.d)
        for (int b = slice; b < a.blocks; b += 32) v += a.part[(int64_t)b * a.d + i];
    sums[slice][lane] = v;
    __syncthreads();
    v = sums[lane][slice];
#pragma unroll
    for (int k = 16; k > 0; k /= 2) v += __shfl_down_sync(kFull, v, k);
    const int mine = blockIdx.x * 32 + slice;
    if (lane == 0 && mine < a.d) a.dw[mine] = v;
}

// ---- host side ------------------------------------------------------------------

// Blocks of a kernel that an SM holds at a time.
int resident_blocks(const void *kernel, int threads, size_t smem) {
    int n = 0;
    if (allow_smem(kernel, smem) != cudaSuccess ||
        cudaOccupancyMaxActiveBlocksPerMultiprocessor(&n, kernel, threads, smem) != cudaSuccess) {
        cudaGetLastError();
        n = 0;
    }
    return std::max(n, 1);
}

// Threads that share a row, and the pieces of each of them: a warp where its
// lanes can hold the row (4 pieces of 16 bytes each, 16 of one value), then up
// to 8 warps, and 32 for the widest rows. Of short rows a warp has several, as one
// would leave most lanes idle (1000000 x 64 bf16: 84 us and 82 for the gradient, 212
// and 295 with a warp a row).
struct RowShape {
    int threads, pieces;
    RowShape(int row_pieces, int most) {
        int warps = 1;
        while (32 * warps * most < row_pieces) warps = warps < 8 ? 2 * warps : 32;
        const int each = (row_pieces + 32 * warps - 1) / (32 * warps);
        pieces = each;
        if (most > 4)  // of one value: 1, 2, 4, 8 or 16
            for (pieces = 1; pieces < each;) pieces *= 2;
        threads = 32 * warps;
        if (pieces == 1)
            for (threads = 4; threads < row_pieces && threads < 32;) threads *= 2;
    }
};

template <typename E, int N, int P, int MOST>
dpb_status launch_grad(NormArgs &a, const RowShape &r, cudaStream_t s) {
    const int rows = MOST / r.threads;
    constexpr size_t kSmem = std::max(GradRows<E, N, P, MOST>::kBytes, (size_t)MOST * P * N * 4);
    const void *kernel = reinterpret_cast<const void *>(add_norm_grad_kernel<E, N, P, MOST>);
    const cudaError_t e = allow_smem(kernel, kSmem);
    if (e != cudaSuccess) return launch_status(e, "add_norm_backward");
    static const int resident = resident_blocks(kernel, MOST, kSmem);
    a.blocks = (int)std::min<int64_t>((a.T + rows - 1) / rows, (int64_t)std::min(resident, kGradBlocks) * sms_of_device());
    add_norm_grad_kernel<E, N, P, MOST><<<a.blocks, MOST, kSmem, s>>>(a, r.threads);
    return launch_status(cudaGetLastError(), "add_norm_backward");
}

template <typename E, int N, int P, int MOST>
dpb_status launch(NormArgs &a, const RowShape &r, bool grad, cudaStream_t s) {
    const int rows = MOST / r.threads;
    if (!grad) {
        static const int resident = resident_blocks(reinterpret_cast<const void *>(add_norm_kernel<E, N, P, MOST>), MOST, 0);
        const int64_t blocks = std::min<int64_t>((a.T + rows - 1) / rows, (int64_t)resident * sms_of_device());
        add_norm_kernel<E, N, P, MOST><<<(unsigned)blocks, MOST, 0, s>>>(a, r.threads);
        return launch_status(cudaGetLastError(), "add_norm");
    }
    return launch_grad<E, N, P, MOST>(a, r, s);
}

template <typename E, int N>
dpb_status dispatch(NormArgs &a, bool grad, cudaStream_t s) {
    const RowShape r((a.d + N - 1) / N, N == 1 ? 16 : 4);
    if (r.threads > 256) {  // 2 or more pieces: what 8 warps cannot hold
        if constexpr (N == 8) return launch<E, N, 2, 1024>(a, r, grad, s);
        if constexpr (N == 4) return r.pieces <= 2 ? launch<E, N, 2, 1024>(a, r, grad, s) : launch<E, N, 4, 1024>(a, r, grad, s);
        if constexpr (N == 1) return r.pieces <= 8 ? launch<E, N, 8, 1024>(a, r, grad, s) : launch<E, N, 16, 1024>(a, r, grad, s);
    }
    if (r.pieces == 1) return launch<E, N, 1, 256>(a, r, grad, s);
    if (r.pieces == 2) return launch<E, N, 2, 256>(a, r, grad, s);
    if constexpr (N > 1)
        if (r.pieces == 3) return launch<E, N, 3, 256>(a, r, grad, s);
    if (r.pieces == 4) return launch<E, N, 4, 256>(a, r, grad, s);
    if constexpr (N == 1) return r.pieces == 8 ? launch<E, N, 8, 256>(a, r, grad, s) : launch<E, N, 16, 256>(a, r, grad, s);
    return fail(DPB_ERR_UNSUPPORTED, "dim is too large");
}

dpb_status run(NormArgs &a, int dtype, bool pieces, bool grad, cudaStream_t s) {
    using bf16 = __nv_bfloat16;
    if (dtype == DPB_F32) return pieces && a.d % 4 == 0 ? dispatch<float, 4>(a, grad, s) : dispatch<float, 1>(a, grad, s);
    return pieces && a.d % 8 == 0 ? dispatch<bf16, 8>(a, grad, s) : dispatch<bf16, 1>(a, grad, s);
}

dpb_status check_config(const dpb_norm_config *c) {
    if (!c) return fail(DPB_ERR_INVALID_ARG, "cfg is NULL");
    if (c->dtype != DPB_F32 && c->dtype != DPB_BF16) return fail(DPB_ERR_INVALID_ARG, "dtype must be DPB_F32 or DPB_BF16");
    if (c->tokens < 0 || c->dim < 1) return fail(DPB_ERR_INVALID_ARG, "a size is too small");
    if (c->tokens > (1ll << 40)) return fail(DPB_ERR_UNSUPPORTED, "at most 2^40 tokens");
    if (c->dim > kMostDim) return fail(DPB_ERR_UNSUPPORTED, "dim must be at most %d", kMostDim);
    if (!(c->eps >= 0.f) || !(c->eps <= 3.402823466e38f)) return fail(DPB_ERR_INVALID_ARG, "eps must be at least 0 and finite");
    return DPB_OK;
}

dpb_status check_rows(const dpb_norm_config *c, const dpb_rows *r, const char *name) {
    const int elem = c->dtype == DPB_F32 ? 4 : 2;
    if (!r) return fail(DPB_ERR_INVALID_ARG, "%s is NULL", name);
    DPB_CHECK(need(r->data, name, elem));
    if (c->tokens > 1 && r->stride < c->dim) return fail(DPB_ERR_INVALID_ARG, "the stride of %s must be at least dim", name);
    return DPB_OK;
}
bool rows_by_pieces(const dpb_norm_config *c, const dpb_rows *r) {
    return !r || by_pieces(r->data, r->stride, c->tokens, c->dtype == DPB_F32 ? 4 : 2);
}

// Blocks of the gradient, at most, each with a part of dw.
int64_t most_blocks(const dpb_norm_config *c) { return std::min<int64_t>(c->tokens, (int64_t)kGradBlocks * sms_of_device()); }

}  // namespace
}  // namespace dpb

using namespace dpb;

extern "C" {

dpb_status dpb_add_norm(const dpb_norm_config *cfg, const dpb_rows *x, const dpb_rows *delta, const void *weight,
                        const dpb_rows *y, const dpb_rows *total, void *stream) {
    DPB_CHECK(check_config(cfg));
    if (cfg->tokens == 0) return DPB_OK;
    DPB_CHECK(check_rows(cfg, x, "x"));
    if (delta) DPB_CHECK(check_rows(cfg, delta, "delta"));
    DPB_CHECK(check_rows(cfg, y, "y"));
    if (total) DPB_CHECK(check_rows(cfg, total, "total"));
    const int elem = cfg->dtype == DPB_F32 ? 4 : 2;
    if (weight) DPB_CHECK(need(weight, "weight", elem));
    NormArgs a{};
    a.x = x->data, a.xs = x->stride;
    if (delta) a.delta = delta->data, a.deltas = delta->stride;
    a.w = weight;
    a.y = y->data, a.ys = y->stride;
    if (total) a.s = total->data, a.ss = total->stride;
    a.T = cfg->tokens, a.d = cfg->dim, a.eps = cfg->eps;
    const bool pieces = rows_by_pieces(cfg, x) && rows_by_pieces(cfg, delta) && rows_by_pieces(cfg, y) &&
                        rows_by_pieces(cfg, total) && by_pieces(weight, 0, 1, elem);
    return run(a, cfg->dtype, pieces, false, static_cast<cudaStream_t>(stream));
}

dpb_status dpb_norm_workspace_size(const dpb_norm_config *cfg, size_t *bytes) {
    DPB_CHECK(check_config(cfg));
    if (!bytes) return fail(DPB_ERR_INVALID_ARG, "bytes is NULL");
    *bytes = ((size_t)most_blocks(cfg) * cfg->dim * 4 + 255) / 256 * 256;
    return DPB_OK;
}

dpb_status dpb_add_norm_backward(const dpb_norm_config *cfg, const dpb_rows *total, const dpb_rows *grad_y,
                                 const dpb_rows *grad_total, const void *weight, const dpb_rows *grad_x,
                                 float *grad_weight, void *workspace, size_t workspace_bytes, void *stream) {
    DPB_CHECK(check_config(cfg));
    const cudaStream_t s = static_cast<cudaStream_t>(stream);
    if (grad_weight) DPB_CHECK(need(grad_weight, "grad_weight", 4));
    if (cfg->tokens == 0) {
        if (!grad_weight) return DPB_OK;
        return launch_status(cudaMemsetAsync(grad_weight, 0, (size_t)cfg->dim * 4, s), "add_norm_backward");
    }
    DPB_CHECK(check_rows(cfg, total, "total"));
    DPB_CHECK(check_rows(cfg, grad_y, "grad_y"));
    if (grad_total) DPB_CHECK(check_rows(cfg, grad_total, "grad_total"));
    DPB_CHECK(check_rows(cfg, grad_x, "grad_x"));
    const int elem = cfg->dtype == DPB_F32 ? 4 : 2;
    if (weight) DPB_CHECK(need(weight, "weight", elem));
    NormArgs a{};
    a.x = total->data, a.xs = total->stride;
    a.dy = grad_y->data, a.dys = grad_y->stride;
    if (grad_total) a.ds = grad_total->data, a.dss = grad_total->stride;
    a.w = weight;
    a.dx = grad_x->data, a.dxs = grad_x->stride;
    a.T = cfg->tokens, a.d = cfg->dim, a.eps = cfg->eps;
    if (grad_weight) {
        DPB_CHECK(need_workspace(workspace, workspace_bytes, (size_t)most_blocks(cfg) * a.d * 4));
        a.dw = grad_weight;
        a.part = static_cast<float *>(workspace);
    }
    const bool pieces = rows_by_pieces(cfg, total) && rows_by_pieces(cfg, grad_y) && rows_by_pieces(cfg, grad_total) &&
                        rows_by_pieces(cfg, grad_x) && by_pieces(weight, 0, 1, elem);
    DPB_CHECK(run(a, cfg->dtype, pieces, true, s));
    if (!grad_weight) return DPB_OK;
    return launch_status(launch_early(add_norm_columns_kernel, dim3((a.d + 31) / 32), 1024, 0, s, a), "add_norm_backward (weight)");
}

}  // extern "C"
