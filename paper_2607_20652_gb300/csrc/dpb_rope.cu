// dpb_rope.cu -- RMS norm of query and key heads with the position rotation
// in the same pass, and its gradient.
//
// Bound by memory: a head is read once and written once (the gradient reads
// two and writes one), some ten operations a value. A warp takes one token,
// so the token's cos and sin are loaded once for all of its heads, and several
// heads at a time: a head of D values takes D / 8 lanes (rounded up to a
// power of two) with 8 values each, and its sums are shuffles among them.
// The 8 values of a lane are 4 rotation pairs, so no value crosses lanes for
// the rotation: (i .. i + 3) and (i + R/2 .. i + R/2 + 3) in the half layout
// (two accesses of 4 values), 8 in a row in the interleaved one and beyond
// the rotated part. Head widths or rotated parts that are no multiple of 8,
// and rows that are not aligned to 4 values, take the same code with one pair
// of values a lane and scalar accesses.
#include <algorithm>
#include <cuda_bf16.h>

#include "dpb_checks.h"
#include "dpb_device.cuh"

namespace dpb {
namespace {

constexpr int kWarps = 8;
constexpr int kBatch = 4;       // rounds (one head a lane group each) whose loads are in flight together
constexpr int kBatchGrad = 3;
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

template <int VEC>
__device__ __forceinline__ void unpack(const float4 &r, float (&v)[VEC]) {
    v[0] = r.x, v[1] = r.y, v[2] = r.z, v[3] = r.w;
}
template <int VEC>
__device__ __forceinline__ void unpack(const uint2 &r, float (&v)[VEC]) {
    v[0] = __uint_as_float(r.x << 16), v[1] = __uint_as_float(r.x & 0xffff0000u);
    v[2] = __uint_as_float(r.y << 16), v[3] = __uint_as_float(r.y & 0xffff0000u);
}
template <int VEC>
__device__ __forceinline__ void unpack(float r, float (&v)[VEC]) {
    v[0] = r;
}
template <int VEC>
__device__ __forceinline__ void unpack(__nv_bfloat16 r, float (&v)[VEC]) {
    v[0] = __bfloat162float(r);
}
template <typename T, int VEC>
__device__ __forceinline__ void store_vec(T *p, const float (&v)[VEC]) {
    if constexpr (VEC == 4)
        st4(p, make_float4(v[0], v[1], v[2], v[3]));
    else
        st_elem(p, 0, v[0]);
}

// A lane's share of a head: UPL units of VEC pairs (a, b). Unit u covers, in
// the rotated part of the half layout, a = VEC u .. and b = a + R/2 ..; else
// the 2 VEC values from 2 VEC u on, paired in turn when rotated.
template <int VEC, int UPL>
struct Share {
    float a[UPL][VEC], b[UPL][VEC];
};
template <typename T, int VEC, int UPL>
struct RawShare {
    typename RawVec<T, VEC>::type a[UPL], b[UPL];
};

template <typename T, int VEC, int UPL>
struct Lane {
    int oa[UPL], ob[UPL];  // first elements of the two runs of VEC values
    bool on[UPL], rot[UPL], inter;

    __device__ __forceinline__ Lane(const RopeArgs &g, int u0) {
        inter = g.interleaved;
#pragma unroll
        for (int j = 0; j < UPL; ++j) {
            const int u = u0 + 32 * j;
            on[j] = 2 * VEC * u < g.D;
            rot[j] = 2 * VEC * u < g.R;
            const bool half = rot[j] && !inter;
            oa[j] = half ? VEC * u : 2 * VEC * u;
            ob[j] = half ? VEC * u + g.R / 2 : 2 * VEC * u + VEC;
        }
    }
    __device__ __forceinline__ void load(const T *row, bool ok, RawShare<T, VEC, UPL> &s) const {
        using R = typename RawVec<T, VEC>::type;
#pragma unroll
        for (int j = 0; j < UPL; ++j) {
            s.a[j] = R{};
            s.b[j] = R{};
            if (ok && on[j]) {
                s.a[j] = *reinterpret_cast<const R *>(row + oa[j]);
                s.b[j] = *reinterpret_cast<const R *>(row + ob[j]);
            }
        }
    }
    __device__ __forceinline__ static void values(const RawShare<T, VEC, UPL> &r, Share<VEC, UPL> &s) {
#pragma unroll
        for (int j = 0; j < UPL; ++j) {
            unpack<VEC>(r.a[j], s.a[j]);
            unpack<VEC>(r.b[j], s.b[j]);
        }
    }
    __device__ __forceinline__ void store(T *row, bool ok, const Share<VEC, UPL> &s) const {
#pragma unroll
        for (int j = 0; j < UPL; ++j)
            if (ok && on[j]) {
                store_vec<T, VEC>(row + oa[j], s.a[j]);
                store_vec<T, VEC>(row + ob[j], s.b[j]);
            }
    }
    // The unit's VEC pairs are (a[i], b[i]) in the half layout; interleaved
    // they are neighbours: for VEC = 4 (a0 a1)(a2 a3)(b0 b1)(b2 b3).
    __device__ __forceinline__ void rotate(Share<VEC, UPL> &s, const float (&c)[UPL][VEC],
                                           const float (&n)[UPL][VEC]) const {
#pragma unroll
        for (int j = 0; j < UPL; ++j) {
            if (!rot[j]) continue;
            if (VEC == 1 || !inter) {
#pragma unroll
                for (int i = 0; i < VEC; ++i) {
                    const float a = s.a[j][i], b = s.b[j][i];
                    s.a[j][i] = a * c[j][i] - b * n[j][i];
                    s.b[j][i] = b * c[j][i] + a * n[j][i];
                }
            } else {
#pragma unroll
                for (int i = 0; i + 1 < VEC; i += 2) {
                    const float a = s.a[j][i], b = s.a[j][i + 1];
                    s.a[j][i] = a * c[j][i / 2] - b * n[j][i / 2];
                    s.a[j][i + 1] = b * c[j][i / 2] + a * n[j][i / 2];
                    const float d = s.b[j][i], e = s.b[j][i + 1];
                    s.b[j][i] = d * c[j][VEC / 2 + i / 2] - e * n[j][VEC / 2 + i / 2];
                    s.b[j][i + 1] = e * c[j][VEC / 2 + i / 2] + d * n[j][VEC / 2 + i / 2];
                }
            }
        }
    }
    // Position p's cos and sin of this lane's pairs (pairs VEC u .. VEC u + VEC - 1
    // in both layouts); 1 and 0 where nothing turns.
    __device__ __forceinline__ void angles(const RopeArgs &g, int64_t p, int u0, float (&c)[UPL][VEC],
                                           float (&n)[UPL][VEC], bool back) const {
        const bool good = p >= 0 && p < g.pos_n;
        if (g.R > 0 && !good && (threadIdx.x & 31) == 0) set_status(g.status, DPB_DEV_BAD_LENGTH);
#pragma unroll
        for (int j = 0; j < UPL; ++j) {
            const bool on = good && rot[j];
            const int64_t at = p * (g.R / 2) + VEC * (u0 + 32 * j);
#pragma unroll
            for (int i = 0; i < VEC; ++i) c[j][i] = 1.f, n[j][i] = 0.f;
            if (on) {
                using R = typename RawVec<float, VEC>::type;
                unpack<VEC>(__ldg(reinterpret_cast<const R *>(g.cos_tab + at)), c[j]);
                unpack<VEC>(__ldg(reinterpret_cast<const R *>(g.sin_tab + at)), n[j]);
                if (back)
#pragma unroll
                    for (int i = 0; i < VEC; ++i) n[j][i] = -n[j][i];
            }
        }
    }
    __device__ __forceinline__ void weights(const void *w, Share<VEC, UPL> &s) const {
#pragma unroll
        for (int j = 0; j < UPL; ++j)
#pragma unroll
            for (int i = 0; i < VEC; ++i) s.a[j][i] = s.b[j][i] = 1.f;
        if (!w) return;
        RawShare<T, VEC, UPL> r;
        load(static_cast<const T *>(w), true, r);
        values(r, s);
    }
};

template <int VEC, int UPL, typename F>
__device__ __forceinline__ void each(F f) {
#pragma unroll
    for (int j = 0; j < UPL; ++j)
#pragma unroll
        for (int i = 0; i < VEC; ++i) f(j, i);
}

__device__ __forceinline__ float group_sum(float v, int gl) {
    for (int o = gl / 2; o > 0; o >>= 1) v += __shfl_xor_sync(kFull, v, o);
    return v;
}

__device__ __forceinline__ int64_t position(const RopeArgs &g, int64_t t) {
    return g.R > 0 && g.pos && t < g.T ? (int64_t)g.pos[t] : t;
}

// One token's heads of q and k as one list of heads_q + heads_k.
struct Row {
    const Heads &q, &k;
    int64_t t;
    template <typename T>
    __device__ __forceinline__ T *head(int h) const {
        const bool second = h >= q.n;
        const Heads &s = second ? k : q;
        return reinterpret_cast<T *>(s.p) + t * s.ts + (second ? h - q.n : h) * s.hs;
    }
};

template <typename T, int VEC, int UPL>
__global__ void __launch_bounds__(32 * kWarps) norm_rope_kernel(const __grid_constant__ RopeArgs g) {
    const int lane = threadIdx.x & 31, u0 = lane & (g.gl - 1), grp = lane / g.gl, groups = 32 / g.gl;
    const Lane<T, VEC, UPL> ln(g, u0);
    const int nh = g.q.n + g.k.n;
    const float inv_d = 1.f / (float)g.D;
    Share<VEC, UPL> w[2];
    ln.weights(g.wq, w[0]);
    ln.weights(g.wk, w[1]);
    const int64_t step = (int64_t)gridDim.x * kWarps;
    int64_t t = (int64_t)blockIdx.x * kWarps + threadIdx.x / 32;
    int64_t p = position(g, t);
    for (; t < g.T; t += step) {
        const Row in{g.q, g.k, t}, out{g.oq, g.ok, t};
        float c[UPL][VEC], n[UPL][VEC];
        for (int h0 = grp; h0 - grp < nh; h0 += groups * kBatch) {
            RawShare<T, VEC, UPL> raw[kBatch];
#pragma unroll
            for (int e = 0; e < kBatch; ++e) {
                const int h = h0 + e * groups;
                ln.load(in.head<const T>(min(h, nh - 1)), h < nh, raw[e]);
            }
            if (h0 == grp) {  // once a token, behind its first heads' loads
                ln.angles(g, p, u0, c, n, false);
                p = position(g, t + step);
            }
#pragma unroll
            for (int e = 0; e < kBatch; ++e) {
                const int h = h0 + e * groups;
                if (h - grp >= nh) break;  // the whole warp is done
                Share<VEC, UPL> x;
                ln.values(raw[e], x);
                if (g.normalise) {
                    float ss = 0.f;
                    each<VEC, UPL>([&](int j, int i) { ss += x.a[j][i] * x.a[j][i] + x.b[j][i] * x.b[j][i]; });
                    const float r = rsqrtf(group_sum(ss, g.gl) * inv_d + g.eps);
                    const bool second = h >= g.q.n;
                    each<VEC, UPL>([&](int j, int i) {
                        x.a[j][i] *= r * (second ? w[1].a[j][i] : w[0].a[j][i]);
                        x.b[j][i] *= r * (second ? w[1].b[j][i] : w[0].b[j][i]);
                    });
                }
                ln.rotate(x, c, n);
                if (h < nh) ln.store(out.head<T>(h), true, x);
            }
        }
    }
}

template <typename T, int VEC, int UPL>
__global__ void __launch_bounds__(32 * kWarps) norm_rope_grad_kernel(const __grid_constant__ RopeArgs g) {
    __shared__ float part[kWarps][2][kMaxDim];
    const int lane = threadIdx.x & 31, u0 = lane & (g.gl - 1), grp = lane / g.gl, groups = 32 / g.gl;
    const int warp = threadIdx.x / 32;
    const Lane<T, VEC, UPL> ln(g, u0);
    const float inv_d = 1.f / (float)g.D;
    Share<VEC, UPL> w[2], dw[2];
    ln.weights(g.wq, w[0]);
    ln.weights(g.wk, w[1]);
    each<VEC, UPL>([&](int j, int i) { dw[0].a[j][i] = dw[0].b[j][i] = dw[1].a[j][i] = dw[1].b[j][i] = 0.f; });
    const int64_t step = (int64_t)gridDim.x * kWarps;
    int64_t t = (int64_t)blockIdx.x * kWarps + warp;
    int64_t p = position(g, t);
    for (; t < g.T; t += step) {
        float c[UPL][VEC], n[UPL][VEC];
        bool first = true;
        // q's heads, then k's: each kind adds to its own weight gradient
#pragma unroll
        for (int s = 0; s < 2; ++s) {
            const Heads &in = s ? g.k : g.q, &gout = s ? g.gk : g.gq, &out = s ? g.ok : g.oq;
            const T *xs = reinterpret_cast<const T *>(in.p) + t * in.ts;
            const T *ys = reinterpret_cast<const T *>(gout.p) + t * gout.ts;
            T *os = reinterpret_cast<T *>(out.p) + t * out.ts;
            for (int h0 = grp; h0 - grp < in.n; h0 += groups * kBatchGrad) {
                RawShare<T, VEC, UPL> rx[kBatchGrad], ry[kBatchGrad];
#pragma unroll
                for (int e = 0; e < kBatchGrad; ++e) {
                    const int h = h0 + e * groups;
                    ln.load(xs + h * in.hs, g.normalise && h < in.n, rx[e]);
                    ln.load(ys + h * gout.hs, h < in.n, ry[e]);
                }
                if (first) {
                    ln.angles(g, p, u0, c, n, true);
                    p = position(g, t + step);
                    first = false;
                }
#pragma unroll
                for (int e = 0; e < kBatchGrad; ++e) {
                    const int h = h0 + e * groups;
                    if (h - grp >= in.n) break;
                    Share<VEC, UPL> x, y;
                    ln.values(ry[e], y);
                    ln.rotate(y, c, n);
                    if (g.normalise) {
                        ln.values(rx[e], x);
                        float ss = 0.f, sp = 0.f;  // sum of x^2, and of w g x
                        each<VEC, UPL>([&](int j, int i) {
                            const float xa = x.a[j][i], xb = x.b[j][i];
                            ss += xa * xa + xb * xb;
                            sp += w[s].a[j][i] * y.a[j][i] * xa + w[s].b[j][i] * y.b[j][i] * xb;
                        });
                        ss = group_sum(ss, g.gl);
                        sp = group_sum(sp, g.gl);
                        const float r = rsqrtf(ss * inv_d + g.eps);
                        const float f = r * r * r * sp * inv_d;
                        each<VEC, UPL>([&](int j, int i) {
                            const float xa = x.a[j][i], xb = x.b[j][i];
                            dw[s].a[j][i] += y.a[j][i] * xa * r;
                            dw[s].b[j][i] += y.b[j][i] * xb * r;
                            y.a[j][i] = r * w[s].a[j][i] * y.a[j][i] - f * xa;
                            y.b[j][i] = r * w[s].b[j][i] * y.b[j][i] - f * xb;
                        });
                    }
                    if (h < in.n) ln.store(os + h * out.hs, true, y);
                }
            }
        }
    }
    if (!g.part) return;
    // the lanes of the warp's groups that hold the same values, then the
    // block's warps, always in the same order
    for (int o = g.gl; o < 32; o <<= 1)
#pragma unroll
        for (int s = 0; s < 2; ++s)
            each<VEC, UPL>([&](int j, int i) {
                dw[s].a[j][i] += __shfl_xor_sync(kFull, dw[s].a[j][i], o);
                dw[s].b[j][i] += __shfl_xor_sync(kFull, dw[s].b[j][i], o);
            });
    if (grp == 0)
#pragma unroll
        for (int s = 0; s < 2; ++s)
            each<VEC, UPL>([&](int j, int i) {
                if (ln.on[j]) {
                    part[warp][s][ln.oa[j] + i] = dw[s].a[j][i];
                    part[warp][s][ln.ob[j] + i] = dw[s].b[j][i];
                }
            });
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
    DPB_CHECK(need_workspace(ws, ws_bytes, backward ? rope_workspace(c) : kStatusBytes));
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
    a.status = static_cast<int32_t *>(ws);
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
int rope_blocks(K kernel, int64_t T) {
    int dev = 0, sms = 1, occ = 1;
    cudaGetDevice(&dev);
    cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev);
    cudaOccupancyMaxActiveBlocksPerMultiprocessor(&occ, kernel, 32 * kWarps, 0);
    const int64_t most = std::min<int64_t>((int64_t)sms * std::max(occ, 1), kMaxBlocks);
    return (int)std::min<int64_t>((T + kWarps - 1) / kWarps, most);
}

template <typename T, int VEC, int UPL>
cudaError_t launch_forward(const RopeArgs &a, cudaStream_t s) {
    static const int full = rope_blocks(norm_rope_kernel<T, VEC, UPL>, INT64_MAX / 2);
    norm_rope_kernel<T, VEC, UPL><<<(int)std::min<int64_t>((a.T + kWarps - 1) / kWarps, full), 32 * kWarps, 0, s>>>(a);
    return cudaGetLastError();
}

template <typename T, int VEC, int UPL>
cudaError_t launch_backward_rope(const RopeArgs &a, float *dwq, float *dwk, cudaStream_t s) {
    static const int full = rope_blocks(norm_rope_grad_kernel<T, VEC, UPL>, INT64_MAX / 2);
    const int blocks = (int)std::min<int64_t>((a.T + kWarps - 1) / kWarps, full);
    if (blocks > 0) norm_rope_grad_kernel<T, VEC, UPL><<<blocks, 32 * kWarps, 0, s>>>(a);
    if (a.part) weight_grad_kernel<<<(2 * a.D + 31) / 32, 1024, 0, s>>>(a.part, blocks, a.D, dwq, dwk);
    return cudaGetLastError();
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
    const cudaStream_t s = static_cast<cudaStream_t>(stream);
    cudaError_t e;
    if (cfg->dtype == DPB_F32)
        e = call.four ? launch_forward<float, 4, 1>(call.a, s) : launch_forward<float, 1, 4>(call.a, s);
    else
        e = call.four ? launch_forward<__nv_bfloat16, 4, 1>(call.a, s) : launch_forward<__nv_bfloat16, 1, 4>(call.a, s);
    return launch_status(e, "qk_norm_rope");
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
    const cudaStream_t s = static_cast<cudaStream_t>(stream);
    cudaError_t e;
    if (cfg->dtype == DPB_F32)
        e = call.four ? launch_backward_rope<float, 4, 1>(call.a, grad_weight_q, grad_weight_k, s)
                      : launch_backward_rope<float, 1, 4>(call.a, grad_weight_q, grad_weight_k, s);
    else
        e = call.four ? launch_backward_rope<__nv_bfloat16, 4, 1>(call.a, grad_weight_q, grad_weight_k, s)
                      : launch_backward_rope<__nv_bfloat16, 1, 4>(call.a, grad_weight_q, grad_weight_k, s);
    return launch_status(e, "qk_norm_rope_backward");
}

}  // extern "C"
