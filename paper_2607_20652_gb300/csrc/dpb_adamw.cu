// dpb_adamw.cu -- one AdamW step of many tensors in place, states in fp32 or
// in 8 bits.
//
// Bound by memory: each parameter, gradient and state is read once and the
// first three kinds written once. The tensors' addresses travel as a kernel
// argument (no table to copy to the device first), so a step is one launch
// for every kMany tensors. A block takes 512 values of one tensor (or some rounds
// of 512), found by bisection in that argument; a warp takes 256 of them, 8 a
// lane, so that a block of 8-bit states is one warp's, its scale a warp maximum.
#include <algorithm>
#include <cmath>
#include <cuda_bf16.h>
#include <cuda_fp8.h>

#include <type_traits>

#include "dpb_checks.h"
#include "dpb_device.cuh"

namespace dpb {
namespace {

constexpr int kPer = 8;                    // values a thread
// Rounds a block: 32-bit states keep enough loads in flight with one (203 M bf16
// parameters: 632 us). 8-bit ones compute longer on fewer bytes, so a block loads
// its next round while it computes one, and its start is spread over up to eight
// (203 M bf16 parameters: 434 us; while that took 457, one round of 256 threads
// 547, four of 128 threads 475) as long as there are some waves of blocks (14 M
// fp32 parameters: 56 us; 57 with eight).
constexpr int kThreads = 64;
constexpr int kRound = kThreads * kPer;    // values a block takes at a time
constexpr int kMostRounds = 8, kWaves = 6, kResident = 152 * 14;
constexpr int kBlock = 32 * kPer;          // values that share a scale
constexpr float kTop = 448.f;              // largest e4m3 value
constexpr float kLargest = 3.402823466e38f;  // largest finite fp32 value
constexpr int kFew = 40, kMany = 440;      // tensors a launch (4 KB and 32 KB of kernel arguments)

struct Tensor {
    void *p;
    const void *g;
    void *m, *v;
    float *ms, *vs;
    int64_t n;
    int64_t at;       // first value's place in the list, each tensor padded to kBlock
};

template <int N>
struct Table {
    int64_t first[N + 1];  // first chunk of each tensor; first[count] = chunks in all
    Tensor t[N];
    uint8_t wide[N];  // every pointer aligned for whole vectors
    int count;
    int chunk;  // values a block
};

struct Hyper {
    float rate, b1, c1, b2, c2, eps, decay, fix2;  // rate: lr / (1 - beta1^step); fix2: (1 - beta2^step)^-1/2
    uint32_t key;
    const float *grad_scale;
    float zero;  // -0
};

// The lowbias32 integer hash of the hash-prospector project: two rounds of
// xor-shift and multiply.
__host__ __device__ __forceinline__ uint32_t mix32(uint32_t x) {
    x ^= x >> 16;
    x *= 0x7feb352du;
    x ^= x >> 15;
    x *= 0x846ca68bu;
    return x ^ (x >> 16);
}

__device__ __forceinline__ float rcp_approx(float x) {
    float y;
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
// Two fp32 values in one register pair, and the packed multiply and add
// (one instruction for both).
struct F2 {
    uint64_t u;
    __device__ __forceinline__ F2() : u(0) {}
    __device__ __forceinline__ F2(float a, float b) { asm("mov.b64 %0, {%1, %2};" : "=l"(u) : "f"(a), "f"(b)); }
    __device__ __forceinline__ float2 get() const {
        float2 r;
        asm("mov.b64 {%0, %1}, %2;" : "=f"(r.x), "=f"(r.y) : "l"(u));
        return r;
    }
};
__device__ __forceinline__ F2 operator*(F2 a, F2 b) {
    F2 r;
    asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r.u) : "l"(a.u), "l"(b.u));
    return r;
}
__device__ __forceinline__ F2 operator+(F2 a, F2 b) {
    F2 r;
    asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r.u) : "l"(a.u), "l"(b.u));
    return r;
}

// a b, rounded by itself whatever is added to it: the compiler may make one
// multiply-add of a packed product and the add that follows it, but not of this
// (zero: -0, from memory, so that it does not see that nothing is added).
__device__ __forceinline__ F2 product(F2 a, F2 b, F2 zero) {
    F2 r;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r.u) : "l"(a.u), "l"(b.u), "l"(zero.u));
    return r;
}

// A value scaled to |y| <= 448 is rounded to one of its two e4m3 neighbours,
// away from zero with the probability of its place between them (r: 16 random
// bits). From 2^-6 on a code keeps 3 bits after the
// leading one, so adding the random bits just below them and cutting them off
// rounds the magnitude; what passes 448 is brought back by the saturating
// conversion.
__device__ __forceinline__ float round_normal(float y, uint32_t r) {
    return __uint_as_float((__float_as_uint(y) + r * 16u) & 0xfff00000u);
}
// Below 2^-6 the codes are multiples of 2^-9. A NaN stays one.
__device__ __forceinline__ float round_small(float y, uint32_t r) {
    const float t = __fadd_rn(fabsf(y) * 512.f, (float)r * (1.f / 65536.f));
    return copysignf(floorf(t) * (1.f / 512.f), y);
}
__device__ __forceinline__ float round_any(float y, uint32_t r) {
    return fabsf(y) >= 0.015625f ? round_normal(y, r) : round_small(y, r);
}
// The smallest of three; a NaN if one of them is.
__device__ __forceinline__ float min_or_nan(float a, float b, float c) {
    float r;
    asm("min.NaN.f32 %0, %1, %2, %3;" : "=f"(r) : "f"(a), "f"(b), "f"(c));
    return r;
}
__device__ __forceinline__ float max3(float a, float b, float c) {
    float r;
    asm("max.f32 %0, %1, %2, %3;" : "=f"(r) : "f"(a), "f"(b), "f"(c));
    return r;
}

// The warp's largest of values >= 0 that are no NaN: their bits as integers are
// in the same order, and integers have an instruction for it.
__device__ __forceinline__ float warp_max(float v) {
    return __uint_as_float(__reduce_max_sync(kFull, __float_as_uint(v)));
}

// Scale of a block with largest magnitude `top`, and what its values are
// multiplied with before rounding. Blocks below 1e-30 are stored as zero.
__device__ __forceinline__ float block_scale(float top, float *inv) {
    const bool live = top >= 1e-30f;
    *inv = live ? __fmul_rn(__frcp_rn(top), kTop) : 0.f;
    return live ? top * (1.f / kTop) : 0.f;
}

// kPer values as they lie in memory.
template <typename T>
struct Raw8 {
    uint32_t w[kPer * sizeof(T) / 4];
};

template <typename T, bool WIDE>
__device__ __forceinline__ void load8(const T *p, int left, Raw8<T> &r) {
    constexpr int W = kPer * sizeof(T) / 4;
    if (WIDE && left >= kPer) {
        if constexpr (W >= 4) {
#pragma unroll
            for (int i = 0; i < W; i += 4) {
                const uint4 u = __ldcs(reinterpret_cast<const uint4 *>(p) + i / 4);
                r.w[i] = u.x, r.w[i + 1] = u.y, r.w[i + 2] = u.z, r.w[i + 3] = u.w;
            }
        } else {
            const uint2 u = __ldcs(reinterpret_cast<const uint2 *>(p));
            r.w[0] = u.x, r.w[1] = u.y;
        }
    } else {
#pragma unroll
        for (int i = 0; i < W; ++i) r.w[i] = 0u;
#pragma unroll
        for (int i = 0; i < kPer; ++i)
            if (i < left) {
                constexpr int per = 4 / sizeof(T);
                uint32_t u;
                if constexpr (sizeof(T) == 4)
                    u = reinterpret_cast<const uint32_t *>(p)[i];
                else if constexpr (sizeof(T) == 2)
                    u = reinterpret_cast<const uint16_t *>(p)[i];
                else
                    u = reinterpret_cast<const uint8_t *>(p)[i];
                r.w[i / per] |= u << (8 * sizeof(T) * (i % per));
            }
    }
}

__device__ __forceinline__ F2 two_values(const Raw8<float> &r, int i) {
    return F2(__uint_as_float(r.w[i]), __uint_as_float(r.w[i + 1]));
}
__device__ __forceinline__ F2 two_values(const Raw8<__nv_bfloat16> &r, int i) {
    return F2(__uint_as_float(r.w[i / 2] << 16), __uint_as_float(r.w[i / 2] & 0xffff0000u));
}
__device__ __forceinline__ F2 two_values(const Raw8<uint8_t> &r, int i) {
    const __half2_raw h = __nv_cvt_fp8x2_to_halfraw2((__nv_fp8x2_storage_t)(r.w[i / 4] >> (8 * (i & 2))), __NV_E4M3);
    const float2 f = __half22float2(__half2(h));
    return F2(f.x, f.y);
}

template <typename T, bool WIDE>
__device__ __forceinline__ void store8(T *p, int left, const float (&v)[kPer]) {
    if (WIDE && left >= kPer) {
        if constexpr (sizeof(T) == 4) {
            __stcs(reinterpret_cast<float4 *>(p), make_float4(v[0], v[1], v[2], v[3]));
            __stcs(reinterpret_cast<float4 *>(p) + 1, make_float4(v[4], v[5], v[6], v[7]));
        } else {
            uint32_t w[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const __nv_bfloat162 b = __floats2bfloat162_rn(v[2 * i], v[2 * i + 1]);
                w[i] = *reinterpret_cast<const uint32_t *>(&b);
            }
            __stcs(reinterpret_cast<uint4 *>(p), make_uint4(w[0], w[1], w[2], w[3]));
        }
    } else {
#pragma unroll
        for (int i = 0; i < kPer; ++i)
            if (i < left) st_elem(p, i, v[i]);
    }
}

// The values are already on the e4m3 grid (or above 448): the conversion is exact.
template <bool WIDE>
__device__ __forceinline__ void store_codes(uint8_t *p, int left, const float (&v)[kPer]) {
    uint32_t w[2] = {0u, 0u};
#pragma unroll
    for (int i = 0; i < 4; ++i)
        w[i / 2] |= (uint32_t)__nv_cvt_float2_to_fp8x2(make_float2(v[2 * i], v[2 * i + 1]), __NV_SATFINITE, __NV_E4M3)
                    << (16 * (i & 1));
    if (WIDE && left >= kPer) {
        __stcs(reinterpret_cast<uint2 *>(p), make_uint2(w[0], w[1]));
    } else {
#pragma unroll
        for (int i = 0; i < kPer; ++i)
            if (i < left) p[i] = (uint8_t)(w[i / 4] >> (8 * (i & 3)));
    }
}

// What a thread loads of kPer values.
template <typename T, bool F8>
struct Loaded {
    using S = std::conditional_t<F8, uint8_t, float>;
    Raw8<T> p, g;
    Raw8<S> m, v;
    float ms, vs;
};

template <typename T, bool F8, bool WIDE>
__device__ __forceinline__ void load_values(const Tensor &t, int64_t i0, Loaded<T, F8> &r) {
    using S = typename Loaded<T, F8>::S;
    const int left = (int)min((int64_t)kPer, max((int64_t)0, t.n - i0));
    if (F8) r.ms = t.ms[i0 / kBlock], r.vs = t.vs[i0 / kBlock];
    load8<T, WIDE>(static_cast<const T *>(t.g) + i0, left, r.g);
    load8<S, WIDE>(static_cast<const S *>(t.m) + i0, left, r.m);
    load8<S, WIDE>(static_cast<const S *>(t.v) + i0, left, r.v);
    load8<T, WIDE>(static_cast<const T *>(t.p) + i0, left, r.p);
}

// Every product and sum of the states is rounded by itself, as its formula is
// written, so that the 8-bit codes are the same wherever that formula is
// computed in fp32.
template <typename T, bool F8, bool WIDE>
__device__ __forceinline__ void step_values(const Tensor &t, int64_t i0, const Hyper &h, float gs,
                                            const Loaded<T, F8> &in) {
    const int left = (int)min((int64_t)kPer, max((int64_t)0, t.n - i0));
    const int lane = threadIdx.x & 31;
    float p[kPer], m[kPer], v[kPer];
    T *pp = static_cast<T *>(t.p) + i0;
    uint8_t *m8 = static_cast<uint8_t *>(t.m) + i0, *v8 = static_cast<uint8_t *>(t.v) + i0;
    float *mf = static_cast<float *>(t.m) + i0, *vf = static_cast<float *>(t.v) + i0;
    const int64_t blk = i0 / kBlock;
    float ms, vs;
    float tm = 0.f, tv = 0.f;  // largest magnitudes of this lane
    const F2 zero(h.zero, h.zero);
#pragma unroll
    for (int i = 0; i < kPer; i += 2) {
        F2 gi = two_values(in.g, i), mi = two_values(in.m, i), vi = two_values(in.v, i);
        if (h.grad_scale) gi = gi * F2(gs, gs);
        if constexpr (F8) {
            mi = mi * F2(in.ms, in.ms);
            vi = vi * F2(in.vs, in.vs);
            vi = vi * vi;
        }
        mi = product(mi, F2(h.b1, h.b1), zero) + product(gi, F2(h.c1, h.c1), zero);
        vi = product(vi, F2(h.b2, h.b2), zero) + product(gi * F2(h.c2, h.c2), gi, zero);
        const float2 m2 = mi.get(), v2 = vi.get();
        const F2 root(__fsqrt_rn(v2.x), __fsqrt_rn(v2.y));
        const float2 den = (root * F2(h.fix2, h.fix2) + F2(h.eps, h.eps)).get();
        const float2 p2 = (two_values(in.p, i) * F2(h.decay, h.decay) +
                           mi * F2(-h.rate, -h.rate) * F2(rcp_approx(den.x), rcp_approx(den.y)))
                              .get();
        p[i] = p2.x, p[i + 1] = p2.y;
        m[i] = m2.x, m[i + 1] = m2.y;
        const float2 s2 = F8 ? root.get() : v2;
        v[i] = s2.x, v[i + 1] = s2.y;
        if (F8) {
            tm = max3(tm, fabsf(m[i]), fabsf(m[i + 1]));
            tv = max3(tv, v[i], v[i + 1]);
        }
    }
    store8<T, WIDE>(pp, left, p);
    if constexpr (F8) {
        tm = warp_max(tm);
        tv = warp_max(tv);
        if (max3(tm, tv, 0.f) > kLargest) {
            // The codes have no infinity: it is stored as NaN, and the block's scale is
            // that of its finite values, so that they keep theirs. (All lanes: tm, tv
            // are the warp's.)
            tm = tv = 0.f;
#pragma unroll
            for (int i = 0; i < kPer; ++i) {
                if (fabsf(m[i]) > kLargest) m[i] = __int_as_float(0x7fffffff);
                if (v[i] > kLargest) v[i] = __int_as_float(0x7fffffff);
                tm = fmaxf(tm, fabsf(m[i]));
                tv = fmaxf(tv, v[i]);
            }
            tm = warp_max(tm);
            tv = warp_max(tv);
        }
        float im, iv;
        ms = block_scale(tm, &im);
        vs = block_scale(tv, &iv);
        const uint64_t at = (uint64_t)(t.at + i0);
        // the value's place (a multiple of kPer, and its place among the kPer) with the key
        const uint32_t key = (uint32_t)at ^ (h.key + 0x9e3779b9u * (uint32_t)(at >> 32));
        uint32_t r[kPer];
        float low = 1.f;  // smallest magnitude of this lane, scaled
#pragma unroll
        for (int i = 0; i < kPer; i += 2) {
            const float2 m2 = (F2(m[i], m[i + 1]) * F2(im, im)).get(), v2 = (F2(v[i], v[i + 1]) * F2(iv, iv)).get();
            m[i] = m2.x, m[i + 1] = m2.y;
            v[i] = v2.x, v[i + 1] = v2.y;
            low = min_or_nan(min_or_nan(low, fabsf(m2.x), fabsf(m2.y)), v2.x, v2.y);
        }
#pragma unroll
        for (int i = 0; i < kPer; ++i) r[i] = mix32(key ^ (uint32_t)i);
        // magnitudes below the normal codes (under 2^-6 / 448 of the block's
        // largest) and NaNs are rare: one test for all of the lane's values
        if (low >= 0.015625f) {
#pragma unroll
            for (int i = 0; i < kPer; ++i) {
                m[i] = round_normal(m[i], r[i] & 0xffffu);
                v[i] = round_normal(v[i], r[i] >> 16);
            }
        } else {
#pragma unroll
            for (int i = 0; i < kPer; ++i) {
                const uint32_t rm = r[i] & 0xffffu, rv = r[i] >> 16;
                m[i] = round_any(m[i], rm);
                const float y = v[i], q = round_any(y, rv);
                v[i] = y > 0.f ? fmaxf(q, 1.f / 512.f) : q;  // 2^-9, the smallest code
            }
        }
        store_codes<WIDE>(m8, left, m);
        store_codes<WIDE>(v8, left, v);
        if (lane == 0) t.ms[blk] = ms, t.vs[blk] = vs;
    } else {
        store8<float, WIDE>(mf, left, m);
        store8<float, WIDE>(vf, left, v);
    }
}

// The next values' loads are under way while these are computed.
template <typename T, bool F8, bool WIDE>
__device__ __forceinline__ void step_chunk(const Tensor t, int64_t i0, int chunk, const Hyper &h, float gs) {
    const int64_t end = min(i0 + chunk, (t.n + kBlock - 1) / kBlock * kBlock);  // whole warps
    if (i0 >= end) return;
    Loaded<T, F8> a;
    load_values<T, F8, WIDE>(t, i0, a);
    if constexpr (!F8) {  // one round
        step_values<T, F8, WIDE>(t, i0, h, gs, a);
    } else {
        Loaded<T, F8> b;
#pragma unroll 1
        for (int64_t i = i0; i < end; i += kRound) {
            const bool more = i + kRound < end;
            if (more) load_values<T, F8, WIDE>(t, i + kRound, b);
            step_values<T, F8, WIDE>(t, i, h, gs, a);
            if (more) a = b;
        }
    }
}

template <typename T, bool F8, int N>
__global__ void __launch_bounds__(kThreads, 14) adamw_kernel(const __grid_constant__ Table<N> tab, const Hyper h) {
    const int64_t chunk = blockIdx.x;
    int lo = 0, hi = tab.count;  // first[lo] <= chunk < first[hi]
    while (hi - lo > 1) {
        const int mid = (lo + hi) / 2;
        if (tab.first[mid] <= chunk)
            lo = mid;
        else
            hi = mid;
    }
    const float gs = h.grad_scale ? *h.grad_scale : 1.f;
    if (!(fabsf(gs) <= kLargest)) return;
    const int64_t i0 = (chunk - tab.first[lo]) * tab.chunk + (int64_t)threadIdx.x * kPer;
    if (tab.wide[lo])
        step_chunk<T, F8, true>(tab.t[lo], i0, tab.chunk, h, gs);
    else
        step_chunk<T, F8, false>(tab.t[lo], i0, tab.chunk, h, gs);
}

template <typename T, bool F8, int N>
cudaError_t launch_group(const dpb_adamw_tensor *ts, int n, int64_t at, int rounds, const Hyper &h, cudaStream_t s) {
    Table<N> tab;
    tab.chunk = rounds * kRound;
    tab.count = 0;
    tab.first[0] = 0;
    const size_t sa = F8 ? 8 : 16;
    for (int i = 0; i < n; ++i) {
        const dpb_adamw_tensor &x = ts[i];
        const int64_t padded = (x.count + kBlock - 1) / kBlock * kBlock;
        if (x.count > 0) {
            const int c = tab.count++;
            tab.t[c] = {x.param, x.grad, x.exp_avg, x.exp_avg_sq, x.exp_avg_scale, x.exp_avg_sq_scale, x.count, at};
            tab.wide[c] = is_aligned(x.param, 16) && is_aligned(x.grad, 16) && is_aligned(x.exp_avg, sa) &&
                          is_aligned(x.exp_avg_sq, sa);
            tab.first[c + 1] = tab.first[c] + (x.count + tab.chunk - 1) / tab.chunk;
        }
        at += padded;
    }
    if (tab.count == 0) return cudaSuccess;
    if (tab.first[tab.count] > 0x7fffffffll) return cudaErrorInvalidConfiguration;
    adamw_kernel<T, F8, N><<<(unsigned)tab.first[tab.count], kThreads, 0, s>>>(tab, h);
    return cudaGetLastError();
}

template <typename T, bool F8>
cudaError_t launch_adamw(const dpb_adamw_tensor *ts, int n, const Hyper &h, cudaStream_t s) {
    int64_t at = 0, all = 0;
    for (int i = 0; i < n; ++i) all += ts[i].count;
    const int rounds = F8 ? (int)std::min<int64_t>(kMostRounds, 1 + all / ((int64_t)kWaves * kResident * kRound)) : 1;
    for (int i = 0; i < n; i += kMany) {
        const int k = std::min(kMany, n - i);
        const cudaError_t e = k <= kFew ? launch_group<T, F8, kFew>(ts + i, k, at, rounds, h, s)
                                        : launch_group<T, F8, kMany>(ts + i, k, at, rounds, h, s);
        if (e != cudaSuccess) return e;
        for (int j = 0; j < k; ++j) at += (ts[i + j].count + kBlock - 1) / kBlock * kBlock;
    }
    return cudaSuccess;
}

dpb_status check_adamw(const dpb_adamw_config *c, const dpb_adamw_tensor *ts, int32_t n) {
    if (!c) return fail(DPB_ERR_INVALID_ARG, "cfg is NULL");
    if (n < 0 || (n > 0 && !ts)) return fail(DPB_ERR_INVALID_ARG, "n < 0 or tensors is NULL");
    if (c->dtype != DPB_F32 && c->dtype != DPB_BF16) return fail(DPB_ERR_INVALID_ARG, "unknown dtype %d", c->dtype);
    if (c->state_bits != 32 && c->state_bits != 8) return fail(DPB_ERR_INVALID_ARG, "state_bits must be 32 or 8");
    if (!(c->beta1 >= 0 && c->beta1 < 1) || !(c->beta2 >= 0 && c->beta2 < 1))
        return fail(DPB_ERR_INVALID_ARG, "betas must lie in [0, 1)");
    if (!(c->lr >= 0) || !(c->eps >= 0) || !(c->weight_decay >= 0) || !std::isfinite(c->lr) ||
        !std::isfinite(c->eps) || !std::isfinite(c->weight_decay))
        return fail(DPB_ERR_INVALID_ARG, "lr, eps and weight_decay must be finite and not negative");
    if (c->step < 1) return fail(DPB_ERR_INVALID_ARG, "step must be at least 1");
    if (c->grad_scale) DPB_CHECK(need(c->grad_scale, "grad_scale", 4));
    const size_t e = c->dtype == DPB_F32 ? 4 : 2;
    for (int i = 0; i < n; ++i) {
        const dpb_adamw_tensor &t = ts[i];
        if (t.count < 0) return fail(DPB_ERR_INVALID_ARG, "tensor %d has a negative count", i);
        if (t.count == 0) continue;
        const size_t se = c->state_bits == 32 ? 4 : 1;
        DPB_CHECK(need(t.param, "param", e));
        DPB_CHECK(need(t.grad, "grad", e));
        DPB_CHECK(need(t.exp_avg, "exp_avg", se));
        DPB_CHECK(need(t.exp_avg_sq, "exp_avg_sq", se));
        if (c->state_bits == 8) {
            DPB_CHECK(need(t.exp_avg_scale, "exp_avg_scale", 4));
            DPB_CHECK(need(t.exp_avg_sq_scale, "exp_avg_sq_scale", 4));
        }
    }
    return DPB_OK;
}

}  // namespace
}  // namespace dpb

using namespace dpb;

extern "C" dpb_status dpb_adamw_step(const dpb_adamw_config *cfg, const dpb_adamw_tensor *tensors, int32_t n,
                                     void *stream) {
    DPB_CHECK(check_adamw(cfg, tensors, n));
    if (n == 0) return DPB_OK;
    Hyper h;
    h.rate = (float)(cfg->lr / (1.0 - std::pow(cfg->beta1, (double)cfg->step)));
    h.b1 = (float)cfg->beta1;
    h.c1 = (float)(1.0 - cfg->beta1);
    h.b2 = (float)cfg->beta2;
    h.zero = -0.f;
    h.c2 = (float)(1.0 - cfg->beta2);
    // the reciprocal takes a denormal for 0, and 0 x inf would be NaN where nothing was ever summed
    h.eps = cfg->eps > 0 ? std::max((float)cfg->eps, 1.17549435e-38f) : 0.f;
    h.decay = (float)(1.0 - cfg->lr * cfg->weight_decay);
    h.fix2 = (float)(1.0 / std::sqrt(1.0 - std::pow(cfg->beta2, (double)cfg->step)));
    h.key = mix32((uint32_t)cfg->seed ^
                  mix32((uint32_t)cfg->step + 0x9e3779b9u * (1u + (uint32_t)(cfg->seed >> 32))));
    h.grad_scale = cfg->grad_scale;
    const cudaStream_t s = static_cast<cudaStream_t>(stream);
    const bool f8 = cfg->state_bits == 8;
    const cudaError_t e = cfg->dtype == DPB_F32 ? (f8 ? launch_adamw<float, true>(tensors, n, h, s)
                                                      : launch_adamw<float, false>(tensors, n, h, s))
                                                : (f8 ? launch_adamw<__nv_bfloat16, true>(tensors, n, h, s)
                                                      : launch_adamw<__nv_bfloat16, false>(tensors, n, h, s));
    return launch_status(e, "adamw");
}
