// dpb_rope.cu -- RMS norm of query and key heads with the position rotation
// in the same pass, and its gradient.
//
// Bound by memory: a head is read once and written once (the gradient reads
// two and writes one), some ten operations a value. A warp takes one token,
// so the token's cos and sin, and their products with the weights, are made
// once for all of its heads, and several heads at a time: a head of D values
// takes D / 8 lanes (rounded up to a power of two) with 8 values each, and its
// sums are shuffles among them. The 8 values of a lane are 4 rotation pairs,
// so no value crosses lanes for the rotation: (i .. i + 3) and
// (i + R/2 .. i + R/2 + 3) in the half layout (two accesses of 4 values), 8 in
// a row in the interleaved one and beyond the rotated part. The pairs' first
// and second values are kept apart, so that both layouts run the same packed
// arithmetic (two values an instruction). Head widths or rotated parts that
// are no multiple of 8, and rows that are not aligned to 4 values, take the
// same code with one pair of values a lane and scalar accesses.
#include <algorithm>
#include <cuda_bf16.h>

#include "dpb_checks.h"
#include "dpb_device.cuh"

namespace dpb {
namespace {

constexpr int kWarps = 8;
// Heads of a lane group whose loads are in flight together, and the blocks an
// SM that the registers are held to: 65536 tokens of 12 + 12 heads of 64 take
// 71 us at (3, 4), 78 at (3, 3), 87 at (4, 4); the gradient of 49999 tokens of
// 16 + 4 heads of 128 143 us at (4, 2), 151 at (3, 2), 184 at (3, 3).
constexpr int kBatch = 3, kBlocks = 4;
constexpr int kBatchGrad = 4, kBlocksGrad = 2;
constexpr int kMaxDim = 256;
constexpr int kMaxBlocks = 152 * 8;  // partial sums of the weight gradients: one row a block

struct Heads {
    char *p;
    int64_t ts, hs;  // strides in elements
    int n;           // heads
};

struct RopeArgs {
    Heads q, k, gq, gk, oq, ok;  // inputs, output gradients (backward), outputs
    const void *wq, *wk;
    const float *cos_tab, *sin_tab;
    const int32_t *pos;
    int64_t T;
    int D, R, pos_n, gl;  // gl: lanes of a head
    int interleaved, normalise;
    float eps;
    float *part;          // [blocks][2][D] partial weight gradients
    int32_t *status;
};

// ---- VEC values of one kind (a pair's first or second) a lane ----------------

template <int VEC>
struct Vals;
template <>
struct Vals<4> {
    uint64_t x[2];
};
template <>
struct Vals<1> {
    float x;
};

__device__ __forceinline__ uint64_t two(float a, float b) {
    uint64_t r;
    asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(a), "f"(b));
    return r;
}
__device__ __forceinline__ float2 apart(uint64_t u) {
    float2 r;
    asm("mov.b64 {%0, %1}, %2;" : "=f"(r.x), "=f"(r.y) : "l"(u));
    return r;
}
__device__ __forceinline__ Vals<4> all4(float v) { return {{two(v, v), two(v, v)}}; }
__device__ __forceinline__ Vals<4> set4(float a, float b, float c, float d) { return {{two(a, b), two(c, d)}}; }
__device__ __forceinline__ Vals<4> operator*(const Vals<4> &a, const Vals<4> &b) {
    Vals<4> r;
#pragma unroll
    for (int i = 0; i < 2; ++i) asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r.x[i]) : "l"(a.x[i]), "l"(b.x[i]));
    return r;
}
__device__ __forceinline__ Vals<4> madd(const Vals<4> &a, const Vals<4> &b, const Vals<4> &c) {
    Vals<4> r;
#pragma unroll
    for (int i = 0; i < 2; ++i)
        asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r.x[i]) : "l"(a.x[i]), "l"(b.x[i]), "l"(c.x[i]));
    return r;
}
__device__ __forceinline__ float total(const Vals<4> &a) {
    const float2 u = apart(a.x[0]), v = apart(a.x[1]);
    return (u.x + u.y) + (v.x + v.y);
}
__device__ __forceinline__ Vals<1> operator*(const Vals<1> &a, const Vals<1> &b) { return {a.x * b.x}; }
__device__ __forceinline__ Vals<1> madd(const Vals<1> &a, const Vals<1> &b, const Vals<1> &c) {
    return {fmaf(a.x, b.x, c.x)};
}
__device__ __forceinline__ float total(const Vals<1> &a) { return a.x; }
template <int VEC>
__device__ __forceinline__ Vals<VEC> all(float v) {
    if constexpr (VEC == 4)
        return all4(v);
    else
        return {v};
}
template <int VEC, typename F>
__device__ __forceinline__ void each_value(const Vals<VEC> &v, F f) {
    if constexpr (VEC == 4) {
        const float2 a = apart(v.x[0]), b = apart(v.x[1]);
        f(0, a.x), f(1, a.y), f(2, b.x), f(3, b.y);
    } else {
        f(0, v.x);
    }
}
template <int VEC, typename F>
__device__ __forceinline__ Vals<VEC> map_values(const Vals<VEC> &v, F f) {
    if constexpr (VEC == 4) {
        const float2 a = apart(v.x[0]), b = apart(v.x[1]);
        return set4(f(a.x), f(a.y), f(b.x), f(b.y));
    } else {
        return {f(v.x)};
    }
}

// ---- access --------------------------------------------------------------------

// VEC values as they lie in memory: loads keep these until they are used.
template <typename T, int VEC>
struct RawVec {
    using type = T;
};
template <>
struct RawVec<float, 4> {
    using type = float4;
};
template <>
struct RawVec<__nv_bfloat16, 4> {
    using type = uint2;
};
template <typename T, int VEC>
struct Raw {
    typename RawVec<T, VEC>::type a, b;
};

__device__ __forceinline__ float low_bf16(uint32_t u) { return __uint_as_float(u << 16); }
__device__ __forceinline__ float high_bf16(uint32_t u) { return __uint_as_float(u & 0xffff0000u); }
__device__ __forceinline__ uint32_t pack_two(float lo, float hi) {
    const __nv_bfloat162 v = __floats2bfloat162_rn(lo, hi);
    return *reinterpret_cast<const uint32_t *>(&v);
}

// A lane's 2 VEC values of a head as (first, second) of its pairs. MIX: the
// pairs are neighbours in memory.
template <bool MIX>
__device__ __forceinline__ void unpack(const Raw<float, 4> &r, Vals<4> &a, Vals<4> &b) {
    a = MIX ? set4(r.a.x, r.a.z, r.b.x, r.b.z) : set4(r.a.x, r.a.y, r.a.z, r.a.w);
    b = MIX ? set4(r.a.y, r.a.w, r.b.y, r.b.w) : set4(r.b.x, r.b.y, r.b.z, r.b.w);
}
template <bool MIX>
__device__ __forceinline__ void unpack(const Raw<__nv_bfloat16, 4> &r, Vals<4> &a, Vals<4> &b) {
    if (MIX) {
        a = set4(low_bf16(r.a.x), low_bf16(r.a.y), low_bf16(r.b.x), low_bf16(r.b.y));
        b = set4(high_bf16(r.a.x), high_bf16(r.a.y), high_bf16(r.b.x), high_bf16(r.b.y));
    } else {
        a = set4(low_bf16(r.a.x), high_bf16(r.a.x), low_bf16(r.a.y), high_bf16(r.a.y));
        b = set4(low_bf16(r.b.x), high_bf16(r.b.x), low_bf16(r.b.y), high_bf16(r.b.y));
    }
}
template <bool MIX, typename T>
__device__ __forceinline__ void unpack(const Raw<T, 1> &r, Vals<1> &a, Vals<1> &b) {
    a.x = (float)r.a;
    b.x = (float)r.b;
}
template <bool MIX>
__device__ __forceinline__ void pack(const Vals<4> &a, const Vals<4> &b, Raw<float, 4> &r) {
    const float2 a0 = apart(a.x[0]), a1 = apart(a.x[1]), b0 = apart(b.x[0]), b1 = apart(b.x[1]);
    r.a = MIX ? make_float4(a0.x, b0.x, a0.y, b0.y) : make_float4(a0.x, a0.y, a1.x, a1.y);
    r.b = MIX ? make_float4(a1.x, b1.x, a1.y, b1.y) : make_float4(b0.x, b0.y, b1.x, b1.y);
}
template <bool MIX>
__device__ __forceinline__ void pack(const Vals<4> &a, const Vals<4> &b, Raw<__nv_bfloat16, 4> &r) {
    const float2 a0 = apart(a.x[0]), a1 = apart(a.x[1]), b0 = apart(b.x[0]), b1 = apart(b.x[1]);
    r.a = MIX ? make_uint2(pack_two(a0.x, b0.x), pack_two(a0.y, b0.y)) : make_uint2(pack_two(a0.x, a0.y), pack_two(a1.x, a1.y));
    r.b = MIX ? make_uint2(pack_two(a1.x, b1.x), pack_two(a1.y, b1.y)) : make_uint2(pack_two(b0.x, b0.y), pack_two(b1.x, b1.y));
}
template <bool MIX, typename T>
__device__ __forceinline__ void pack(const Vals<1> &a, const Vals<1> &b, Raw<T, 1> &r) {
    r.a = (T)a.x;
    r.b = (T)b.x;
}

// A lane's share of a head: UPL units of VEC pairs. Unit u covers, in the
// rotated part of the half layout, VEC u .. and VEC u + R/2 ..; else the 2 VEC
// values from 2 VEC u on. MIX says that these are neighbouring pairs; beyond
// the rotated part (rotated by nothing) the pairing does not matter.
template <typename T, int VEC, int UPL, bool MIX>
struct Lane {
    using R = typename RawVec<T, VEC>::type;
    int oa[UPL], ob[UPL];  // first elements of the two runs of VEC values
    bool on[UPL], rot[UPL];

    __device__ __forceinline__ Lane(const RopeArgs &g, int u0) {
#pragma unroll
        for (int j = 0; j < UPL; ++j) {
            const int u = u0 + 32 * j;
            on[j] = 2 * VEC * u < g.D;
            rot[j] = 2 * VEC * u < g.R;
            const bool half = rot[j] && !MIX;
            oa[j] = half ? VEC * u : 2 * VEC * u;
            ob[j] = half ? VEC * u + g.R / 2 : 2 * VEC * u + VEC;
        }
    }
    __device__ __forceinline__ void load(const T *row, bool ok, Raw<T, VEC> (&s)[UPL]) const {
#pragma unroll
        for (int j = 0; j < UPL; ++j) {
            s[j].a = R{};
            s[j].b = R{};
            if (ok && on[j]) {
                s[j].a = *reinterpret_cast<const R *>(row + oa[j]);
                s[j].b = *reinterpret_cast<const R *>(row + ob[j]);
            }
        }
    }
    __device__ __forceinline__ void store(T *row, const Vals<VEC> (&a)[UPL], const Vals<VEC> (&b)[UPL]) const {
#pragma unroll
        for (int j = 0; j < UPL; ++j)
            if (on[j]) {
                Raw<T, VEC> r;
                pack<MIX>(a[j], b[j], r);
                *reinterpret_cast<R *>(row + oa[j]) = r.a;
                *reinterpret_cast<R *>(row + ob[j]) = r.b;
            }
    }
    // Position p's cos and sin of this lane's pairs (pairs VEC u .. VEC u +
    // VEC - 1 in both layouts); 1 and 0 where nothing turns.
    __device__ __forceinline__ void angles(const RopeArgs &g, int64_t p, int u0, Vals<VEC> (&c)[UPL],
                                           Vals<VEC> (&n)[UPL]) const {
        const bool good = p >= 0 && p < g.pos_n;
        if (g.R > 0 && !good && (threadIdx.x & 31) == 0) set_status(g.status, DPB_DEV_BAD_LENGTH);
#pragma unroll
        for (int j = 0; j < UPL; ++j) {
            c[j] = all<VEC>(1.f);
            n[j] = all<VEC>(0.f);
            if (good && rot[j]) {
                const int64_t at = p * (g.R / 2) + VEC * (u0 + 32 * j);
                if constexpr (VEC == 4) {
                    const float4 x = __ldg(reinterpret_cast<const float4 *>(g.cos_tab + at));
                    const float4 y = __ldg(reinterpret_cast<const float4 *>(g.sin_tab + at));
                    c[j] = set4(x.x, x.y, x.z, x.w);
                    n[j] = set4(y.x, y.y, y.z, y.w);
                } else {
                    c[j].x = __ldg(g.cos_tab + at);
                    n[j].x = __ldg(g.sin_tab + at);
                }
            }
        }
    }
    __device__ __forceinline__ void weights(const void *w, Vals<VEC> (&a)[UPL], Vals<VEC> (&b)[UPL]) const {
#pragma unroll
        for (int j = 0; j < UPL; ++j) a[j] = b[j] = all<VEC>(1.f);
        if (!w) return;
        Raw<T, VEC> r[UPL];
        load(static_cast<const T *>(w), true, r);
#pragma unroll
        for (int j = 0; j < UPL; ++j) unpack<MIX>(r[j], a[j], b[j]);
    }
};

// Sum over the lanes of a head: GL of them, or (GL = 0) gl.
template <int GL>
__device__ __forceinline__ float group_sum(float v, int gl) {
    if constexpr (GL > 0) {
#pragma unroll
        for (int o = GL / 2; o > 0; o >>= 1) v += __shfl_xor_sync(kFull, v, o);
    } else {
        for (int o = gl / 2; o > 0; o >>= 1) v += __shfl_xor_sync(kFull, v, o);
    }
    return v;
}

__device__ __forceinline__ int64_t position(const RopeArgs &g, int64_t t) {
    return g.R > 0 && g.pos && t < g.T ? (int64_t)g.pos[t] : t;
}

template <int VEC>
__device__ __forceinline__ Vals<VEC> negative(const Vals<VEC> &v) {
    return map_values<VEC>(v, [](float x) { return -x; });
}

// A lane group's heads of one kind: h = grp, grp + groups, ..., taken in
// batches of B whose loads are in flight together.
template <typename T>
struct Walk {
    T *at;
    int64_t step;  // to the group's next head
    __device__ __forceinline__ Walk(const Heads &h, int64_t t, int grp, int groups)
        : at(reinterpret_cast<T *>(h.p) + t * h.ts + grp * h.hs), step(groups * h.hs) {}
};

// With P = w cos and Q = w sin, the rotated, weighted and normalised pair is
//   r (x_a P_a - x_b Q_b),  r (x_b P_b + x_a Q_a).
template <typename T, int VEC, int UPL, bool MIX, int GL>
__global__ void __launch_bounds__(32 * kWarps, VEC == 4 ? kBlocks : 1) norm_rope_kernel(
    const __grid_constant__ RopeArgs g) {
    const int gl = GL > 0 ? GL : g.gl;
    const int lane = threadIdx.x & 31, u0 = lane & (gl - 1), grp = lane / gl, groups = 32 / gl;
    const Lane<T, VEC, UPL, MIX> ln(g, u0);
    const float inv_d = 1.f / (float)g.D;
    const int64_t step = (int64_t)gridDim.x * kWarps;
    int64_t t = (int64_t)blockIdx.x * kWarps + threadIdx.x / 32;
    int64_t p = position(g, t);
    for (; t < g.T; t += step) {
        const int64_t next = position(g, t + step);
#pragma unroll
        for (int s = 0; s < 2; ++s) {
            const Heads &in = s ? g.k : g.q;
            Walk<const T> src(in, t, grp, groups);
            Walk<T> dst(s ? g.ok : g.oq, t, grp, groups);
            // weights and angles are read for either kind (from the L1 cache)
            // rather than held in registers, which more warps need
            Vals<VEC> pa[UPL], pb[UPL], qa[UPL], qb[UPL];
            for (int h0 = grp; h0 - grp < in.n; h0 += groups * kBatch) {
                Raw<T, VEC> raw[kBatch][UPL];
#pragma unroll
                for (int e = 0; e < kBatch; ++e) {
                    ln.load(src.at, h0 + e * groups < in.n, raw[e]);
                    src.at += src.step;
                }
                if (h0 == grp) {  // behind the first heads' loads
                    Vals<VEC> c[UPL], n[UPL], a[UPL], b[UPL];
                    ln.angles(g, p, u0, c, n);
                    ln.weights(s ? g.wk : g.wq, a, b);
#pragma unroll
                    for (int j = 0; j < UPL; ++j) {
                        pa[j] = a[j] * c[j];
                        pb[j] = b[j] * c[j];
                        qa[j] = a[j] * n[j];
                        qb[j] = negative<VEC>(b[j] * n[j]);
                    }
                }
#pragma unroll
                for (int e = 0; e < kBatch; ++e) {
                    const int h = h0 + e * groups;
                    if (h - grp >= in.n) break;
                    Vals<VEC> ya[UPL], yb[UPL], ss = all<VEC>(0.f);
#pragma unroll
                    for (int j = 0; j < UPL; ++j) {
                        Vals<VEC> xa, xb;
                        unpack<MIX>(raw[e][j], xa, xb);
                        ss = madd(xb, xb, j ? madd(xa, xa, ss) : xa * xa);
                        ya[j] = madd(xb, qb[j], xa * pa[j]);
                        yb[j] = madd(xa, qa[j], xb * pb[j]);
                    }
                    if (g.normalise) {
                        const Vals<VEC> f = all<VEC>(rsqrtf(group_sum<GL>(total(ss), gl) * inv_d + g.eps));
#pragma unroll
                        for (int j = 0; j < UPL; ++j) {
                            ya[j] = ya[j] * f;
                            yb[j] = yb[j] * f;
                        }
                    }
                    if (h < in.n) ln.store(dst.at, ya, yb);
                    dst.at += dst.step;
                }
            }
        }
        p = next;
    }
}

// The gradient: g rotated back, u = w g, n = x r; dx = r (u - n mean(u n)), and
// g n to the weight's.
template <typename T, int VEC, int UPL, bool MIX, int GL>
__global__ void __launch_bounds__(32 * kWarps, VEC == 4 ? kBlocksGrad : 1) norm_rope_grad_kernel(
    const __grid_constant__ RopeArgs g) {
    __shared__ float part[kWarps][2][kMaxDim];
    const int gl = GL > 0 ? GL : g.gl;
    const int lane = threadIdx.x & 31, u0 = lane & (gl - 1), grp = lane / gl, groups = 32 / gl;
    const int warp = threadIdx.x / 32;
    const Lane<T, VEC, UPL, MIX> ln(g, u0);
    const float inv_d = 1.f / (float)g.D;
    Vals<VEC> wa[2][UPL], wb[2][UPL], da[2][UPL], db[2][UPL];
    ln.weights(g.wq, wa[0], wb[0]);
    ln.weights(g.wk, wa[1], wb[1]);
#pragma unroll
    for (int j = 0; j < UPL; ++j) da[0][j] = db[0][j] = da[1][j] = db[1][j] = all<VEC>(0.f);
    const int64_t step = (int64_t)gridDim.x * kWarps;
    int64_t t = (int64_t)blockIdx.x * kWarps + warp;
    int64_t p = position(g, t);
    for (; t < g.T; t += step) {
        Vals<VEC> c[UPL], n[UPL], m[UPL];
        bool first = true;
        // q's heads, then k's: each kind adds to its own weight gradient
#pragma unroll
        for (int s = 0; s < 2; ++s) {
            const Heads &in = s ? g.k : g.q;
            Walk<const T> xs(in, t, grp, groups), ys(s ? g.gk : g.gq, t, grp, groups);
            Walk<T> os(s ? g.ok : g.oq, t, grp, groups);
            for (int h0 = grp; h0 - grp < in.n; h0 += groups * kBatchGrad) {
                Raw<T, VEC> rx[kBatchGrad][UPL], ry[kBatchGrad][UPL];
#pragma unroll
                for (int e = 0; e < kBatchGrad; ++e) {
                    const int h = h0 + e * groups;
                    ln.load(xs.at, g.normalise && h < in.n, rx[e]);
                    ln.load(ys.at, h < in.n, ry[e]);
                    xs.at += xs.step;
                    ys.at += ys.step;
                }
                if (first) {
                    ln.angles(g, p, u0, c, n);
#pragma unroll
                    for (int j = 0; j < UPL; ++j) m[j] = negative<VEC>(n[j]);
                    p = position(g, t + step);
                    first = false;
                }
#pragma unroll
                for (int e = 0; e < kBatchGrad; ++e) {
                    const int h = h0 + e * groups;
                    if (h - grp >= in.n) break;
                    Vals<VEC> xa[UPL], xb[UPL], ga[UPL], gb[UPL], ua[UPL], ub[UPL];
                    Vals<VEC> ss = all<VEC>(0.f), sp = all<VEC>(0.f);  // sums of x^2 and of u x
#pragma unroll
                    for (int j = 0; j < UPL; ++j) {
                        Vals<VEC> ya, yb;
                        unpack<MIX>(ry[e][j], ya, yb);
                        unpack<MIX>(rx[e][j], xa[j], xb[j]);
                        ga[j] = madd(yb, n[j], ya * c[j]);
                        gb[j] = madd(ya, m[j], yb * c[j]);
                        ua[j] = ga[j] * wa[s][j];
                        ub[j] = gb[j] * wb[s][j];
                        ss = madd(xb[j], xb[j], j ? madd(xa[j], xa[j], ss) : xa[j] * xa[j]);
                        sp = madd(xb[j], ub[j], j ? madd(xa[j], ua[j], sp) : xa[j] * ua[j]);
                    }
                    if (g.normalise) {
                        const float x2 = group_sum<GL>(total(ss), gl), ux = group_sum<GL>(total(sp), gl);
                        // a lane group without a head adds 0 x r: r must not be infinite there, whatever eps
                        const float r = rsqrtf((h < in.n ? x2 : 1.f) * inv_d + g.eps);
                        // r^3 by itself leaves fp32 at heads beyond 1e14, and without an eps below 1e-13
                        const Vals<VEC> r4 = all<VEC>(r), less = all<VEC>(-r * (ux * inv_d));
#pragma unroll
                        for (int j = 0; j < UPL; ++j) {
                            const Vals<VEC> na = xa[j] * r4, nb = xb[j] * r4;
                            da[s][j] = madd(ga[j], na, da[s][j]);
                            db[s][j] = madd(gb[j], nb, db[s][j]);
                            ua[j] = madd(na, less, ua[j]) * r4;
                            ub[j] = madd(nb, less, ub[j]) * r4;
                        }
                    }
                    if (h < in.n) ln.store(os.at, ua, ub);
                    os.at += os.step;
                }
            }
        }
    }
    if (!g.part) return;
    // the lanes of the warp's groups that hold the same values, then the
    // block's warps, always in the same order
    for (int o = gl; o < 32; o <<= 1)
#pragma unroll
        for (int s = 0; s < 2; ++s)
#pragma unroll
            for (int j = 0; j < UPL; ++j) {
                auto add = [&](float x) { return x + __shfl_xor_sync(kFull, x, o); };
                da[s][j] = map_values<VEC>(da[s][j], add);
                db[s][j] = map_values<VEC>(db[s][j], add);
            }
    if (grp == 0)
#pragma unroll
        for (int s = 0; s < 2; ++s)
#pragma unroll
            for (int j = 0; j < UPL; ++j)
                if (ln.on[j]) {
                    // where a pair's values lie: neighbours, or in two runs
                    each_value<VEC>(da[s][j], [&](int i, float x) { part[warp][s][MIX && VEC > 1 ? ln.oa[j] + 2 * i : ln.oa[j] + i] = x; });
                    each_value<VEC>(db[s][j], [&](int i, float x) { part[warp][s][MIX && VEC > 1 ? ln.oa[j] + 2 * i + 1 : ln.ob[j] + i] = x; });
                }
    __syncthreads();
    for (int e = threadIdx.x; e < 2 * g.D; e += blockDim.x) {
        const int s = e >= g.D, i = e - s * g.D;
        float v = 0.f;
#pragma unroll
        for (int v8 = 0; v8 < kWarps; ++v8) v += part[v8][s][i];
        g.part[((int64_t)blockIdx.x * 2 + s) * g.D + i] = v;
    }
}

// Sums the blocks' partial weight gradients: 32 columns a block, 32 rows at a
// time, in a fixed order.
__global__ void __launch_bounds__(1024) weight_grad_kernel(const float *part, int rows, int D, float *dq, float *dk) {
    __shared__ float s[32][33];
    const int col = blockIdx.x * 32 + (threadIdx.x & 31), r0 = threadIdx.x / 32;
    float v = 0.f;
    if (col < 2 * D)
        for (int r = r0; r < rows; r += 32) v += part[(int64_t)r * 2 * D + col];
    s[r0][threadIdx.x & 31] = v;
    __syncthreads();
    if (r0 == 0 && col < 2 * D) {
        float sum = 0.f;
        for (int r = 0; r < 32; ++r) sum += s[r][threadIdx.x & 31];
        float *out = col < D ? dq : dk;
        if (out) out[col < D ? col : col - D] = sum;
    }
}

dpb_status check_heads(const dpb_heads *h, const char *name, int n, size_t elem, Heads *out) {
    *out = Heads{nullptr, 0, 0, n};
    if (n == 0) return DPB_OK;
    if (!h) return fail(DPB_ERR_INVALID_ARG, "%s is NULL", name);
    DPB_CHECK(need(h->data, name, elem));
    *out = Heads{static_cast<char *>(h->data), h->token_stride, h->head_stride, n};
    return DPB_OK;
}

// Rows whose every run of 4 values is aligned for one access.
bool rows_by_four(const Heads &h, size_t elem) {
    return h.n == 0 || (is_aligned(h.p, 4 * elem) && h.ts % 4 == 0 && h.hs % 4 == 0);
}

dpb_status check_config(const dpb_rope_config *c) {
    if (!c) return fail(DPB_ERR_INVALID_ARG, "cfg is NULL");
    if (c->tokens < 0 || c->heads_q < 0 || c->heads_k < 0 || c->heads_q > 65535 || c->heads_k > 65535)
        return fail(DPB_ERR_INVALID_ARG, "tokens or heads out of range");
    if (c->head_dim < 2 || c->head_dim > kMaxDim || c->head_dim % 2)
        return fail(DPB_ERR_UNSUPPORTED, "head_dim must be even, in [2, %d]", kMaxDim);
    if (c->rot_dim < 0 || c->rot_dim > c->head_dim || c->rot_dim % 2)
        return fail(DPB_ERR_INVALID_ARG, "rot_dim must be even, in [0, head_dim]");
    if (c->rot_dim > 0 && c->positions_n < 1) return fail(DPB_ERR_INVALID_ARG, "positions_n must be at least 1");
    if (c->dtype != DPB_F32 && c->dtype != DPB_BF16) return fail(DPB_ERR_INVALID_ARG, "unknown dtype %d", c->dtype);
    DPB_CHECK(check_slot(c->status_slot));
    if (c->normalise && !(c->eps >= 0.f)) return fail(DPB_ERR_INVALID_ARG, "eps must not be negative");
    return DPB_OK;
}

size_t rope_workspace(const dpb_rope_config *c) {
    return kStatusBytes + sizeof(float) * 2 * (size_t)c->head_dim * kMaxBlocks;
}

struct Call {
    RopeArgs a{};
    bool four = true;
};

dpb_status make_call(const dpb_rope_config *c, const dpb_heads *q, const dpb_heads *k, const dpb_heads *gq,
                     const dpb_heads *gk, const void *wq, const void *wk, const float *ct, const float *st,
                     const int32_t *pos, const dpb_heads *oq, const dpb_heads *ok, void *ws, size_t ws_bytes,
                     bool backward, Call *out) {
    const size_t e = c->dtype == DPB_F32 ? 4 : 2;
    if (!c->normalise && (wq || wk)) return fail(DPB_ERR_INVALID_ARG, "weights are given but normalise is 0");
    RopeArgs &a = out->a;
    const bool in = !backward || c->normalise;  // without a norm the gradient needs no input
    DPB_CHECK(check_heads(q, "q", in ? c->heads_q : 0, e, &a.q));
    DPB_CHECK(check_heads(k, "k", in ? c->heads_k : 0, e, &a.k));
    DPB_CHECK(check_heads(gq, "grad_q_out", backward ? c->heads_q : 0, e, &a.gq));
    DPB_CHECK(check_heads(gk, "grad_k_out", backward ? c->heads_k : 0, e, &a.gk));
    DPB_CHECK(check_heads(oq, "q output", c->heads_q, e, &a.oq));
    DPB_CHECK(check_heads(ok, "k output", c->heads_k, e, &a.ok));
    a.q.n = c->heads_q;
    a.k.n = c->heads_k;
    if (c->rot_dim > 0) {
        DPB_CHECK(need(ct, "cos_tab", 4));
        DPB_CHECK(need(st, "sin_tab", 4));
    }
    if (wq) DPB_CHECK(need(wq, "weight_q", e));
    if (wk) DPB_CHECK(need(wk, "weight_k", e));
    if (pos) DPB_CHECK(need(pos, "positions", 4));
    DPB_CHECK(place_status(c->status_slot, ws, ws_bytes, backward ? rope_workspace(c) : kStatusBytes, &a.status));
    a.wq = wq;
    a.wk = wk;
    a.cos_tab = ct;
    a.sin_tab = st;
    a.pos = pos;
    a.T = c->tokens;
    a.D = c->head_dim;
    a.R = c->rot_dim;
    a.pos_n = c->positions_n;
    a.interleaved = c->interleaved != 0;
    a.normalise = c->normalise != 0;
    a.eps = c->eps;
    out->four = c->head_dim % 8 == 0 && c->rot_dim % 8 == 0 && is_aligned(ct, 16) && is_aligned(st, 16) &&
                is_aligned(wq, 4 * e) && is_aligned(wk, 4 * e);
    const Heads *all[] = {&a.q, &a.k, &a.gq, &a.gk, &a.oq, &a.ok};
    for (const Heads *h : all) out->four = out->four && (!h->p || rows_by_four(*h, e));
    a.gl = 32;
    if (out->four)
        for (a.gl = 1; a.gl * 8 < c->head_dim; a.gl *= 2) {
        }
    return DPB_OK;
}

template <typename K>
int rope_blocks(K kernel) {
    int dev = 0, sms = 1, occ = 1;
    cudaGetDevice(&dev);
    cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev);
    cudaOccupancyMaxActiveBlocksPerMultiprocessor(&occ, kernel, 32 * kWarps, 0);
    return std::min(sms * std::max(occ, 1), kMaxBlocks);
}

template <typename T, int VEC, int UPL, bool MIX, int GL>
cudaError_t launch_kernels(const RopeArgs &a, bool backward, float *dwq, float *dwk, cudaStream_t s) {
    const int64_t wanted = (a.T + kWarps - 1) / kWarps;
    if (!backward) {
        static const int full = rope_blocks(norm_rope_kernel<T, VEC, UPL, MIX, GL>);
        norm_rope_kernel<T, VEC, UPL, MIX, GL><<<(int)std::min<int64_t>(wanted, full), 32 * kWarps, 0, s>>>(a);
        return cudaGetLastError();
    }
    static const int full = rope_blocks(norm_rope_grad_kernel<T, VEC, UPL, MIX, GL>);
    const int blocks = (int)std::min<int64_t>(wanted, full);
    if (blocks > 0) norm_rope_grad_kernel<T, VEC, UPL, MIX, GL><<<blocks, 32 * kWarps, 0, s>>>(a);
    if (a.part) weight_grad_kernel<<<(2 * a.D + 31) / 32, 1024, 0, s>>>(a.part, blocks, a.D, dwq, dwk);
    return cudaGetLastError();
}

// By type, by whether rows are read 4 values at a time, by layout, and by the
// lanes of a head: the usual two counts have their sums unrolled.
template <typename T, int VEC, int UPL, bool MIX>
cudaError_t launch_lanes(const Call &c, bool backward, float *dwq, float *dwk, cudaStream_t s) {
    if constexpr (VEC == 4) {
        if (c.a.gl == 8) return launch_kernels<T, VEC, UPL, MIX, 8>(c.a, backward, dwq, dwk, s);
        if (c.a.gl == 16) return launch_kernels<T, VEC, UPL, MIX, 16>(c.a, backward, dwq, dwk, s);
    }
    return launch_kernels<T, VEC, UPL, MIX, 0>(c.a, backward, dwq, dwk, s);
}

template <typename T, int VEC, int UPL>
cudaError_t launch_kind(const Call &c, bool backward, float *dwq, float *dwk, cudaStream_t s) {
    return c.a.interleaved ? launch_lanes<T, VEC, UPL, true>(c, backward, dwq, dwk, s)
                           : launch_lanes<T, VEC, UPL, false>(c, backward, dwq, dwk, s);
}

cudaError_t launch_rope(const Call &c, int dtype, bool backward, float *dwq, float *dwk, cudaStream_t s) {
    if (dtype == DPB_F32)
        return c.four ? launch_kind<float, 4, 1>(c, backward, dwq, dwk, s)
                      : launch_kind<float, 1, 4>(c, backward, dwq, dwk, s);
    return c.four ? launch_kind<__nv_bfloat16, 4, 1>(c, backward, dwq, dwk, s)
                  : launch_kind<__nv_bfloat16, 1, 4>(c, backward, dwq, dwk, s);
}

}  // namespace
}  // namespace dpb

using namespace dpb;

extern "C" {

dpb_status dpb_rope_workspace_size(const dpb_rope_config *cfg, size_t *bytes) {
    DPB_CHECK(check_config(cfg));
    if (!bytes) return fail(DPB_ERR_INVALID_ARG, "bytes is NULL");
    *bytes = rope_workspace(cfg);
    return DPB_OK;
}

dpb_status dpb_qk_norm_rope(const dpb_rope_config *cfg, const dpb_heads *q, const dpb_heads *k, const void *weight_q,
                            const void *weight_k, const float *cos_tab, const float *sin_tab,
                            const int32_t *positions, const dpb_heads *q_out, const dpb_heads *k_out, void *workspace,
                            size_t workspace_bytes, void *stream) {
    DPB_CHECK(check_config(cfg));
    if (cfg->tokens == 0) return DPB_OK;
    Call call;
    DPB_CHECK(make_call(cfg, q, k, nullptr, nullptr, weight_q, weight_k, cos_tab, sin_tab, positions, q_out, k_out,
                        workspace, workspace_bytes, false, &call));
    return launch_status(
        launch_rope(call, cfg->dtype, false, nullptr, nullptr, static_cast<cudaStream_t>(stream)), "qk_norm_rope");
}

dpb_status dpb_qk_norm_rope_backward(const dpb_rope_config *cfg, const dpb_heads *q, const dpb_heads *k,
                                     const dpb_heads *grad_q_out, const dpb_heads *grad_k_out, const void *weight_q,
                                     const void *weight_k, const float *cos_tab, const float *sin_tab,
                                     const int32_t *positions, const dpb_heads *grad_q, const dpb_heads *grad_k,
                                     float *grad_weight_q, float *grad_weight_k, void *workspace,
                                     size_t workspace_bytes, void *stream) {
    DPB_CHECK(check_config(cfg));
    const bool weights = grad_weight_q || grad_weight_k;
    if (weights && !cfg->normalise) return fail(DPB_ERR_INVALID_ARG, "weight gradients need normalise");
    if (grad_weight_q) DPB_CHECK(need(grad_weight_q, "grad_weight_q", 4));
    if (grad_weight_k) DPB_CHECK(need(grad_weight_k, "grad_weight_k", 4));
    if (cfg->tokens == 0 && !weights) return DPB_OK;
    Call call;
    if (cfg->tokens == 0) {  // no rows: the weight gradients are zero
        DPB_CHECK(need_workspace(workspace, workspace_bytes, rope_workspace(cfg)));
        call.a.D = cfg->head_dim;
        call.a.T = 0;
    } else {
        DPB_CHECK(make_call(cfg, q, k, grad_q_out, grad_k_out, weight_q, weight_k, cos_tab, sin_tab, positions, grad_q,
                            grad_k, workspace, workspace_bytes, true, &call));
    }
    if (weights) call.a.part = reinterpret_cast<float *>(static_cast<char *>(workspace) + kStatusBytes);
    return launch_status(
        launch_rope(call, cfg->dtype, true, grad_weight_q, grad_weight_k, static_cast<cudaStream_t>(stream)),
        "qk_norm_rope_backward");
}

}  // extern "C"
