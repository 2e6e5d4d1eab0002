// dpb_rows.cuh -- access to rows of fp32 or bf16 values in pieces of 16 bytes
// (or, where a row does not allow it, value by value), for the kernels that
// pass over whole rows.
#pragma once

#include <cuda_bf16.h>
#include <cuda_runtime.h>

#include <cstdint>

#include "dpb_internal.h"

namespace dpb {

// N values of a row: 16 bytes of them, or one.
template <typename E, int N>
struct Piece {
    float v[N];
};

__device__ __forceinline__ void load_piece(const float *p, Piece<float, 4> &r) {
    const float4 x = *reinterpret_cast<const float4 *>(p);
    r.v[0] = x.x, r.v[1] = x.y, r.v[2] = x.z, r.v[3] = x.w;
}
__device__ __forceinline__ void load_piece(const __nv_bfloat16 *p, Piece<__nv_bfloat16, 8> &r) {
    const uint4 x = *reinterpret_cast<const uint4 *>(p);
    const uint32_t w[4] = {x.x, x.y, x.z, x.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        r.v[2 * i] = __uint_as_float(w[i] << 16);
        r.v[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
    }
}
__device__ __forceinline__ void load_piece(const float *p, Piece<float, 1> &r) { r.v[0] = *p; }
__device__ __forceinline__ void load_piece(const __nv_bfloat16 *p, Piece<__nv_bfloat16, 1> &r) {
    r.v[0] = __bfloat162float(*p);
}
__device__ __forceinline__ void store_piece(float *p, const Piece<float, 4> &r) {
    *reinterpret_cast<float4 *>(p) = make_float4(r.v[0], r.v[1], r.v[2], r.v[3]);
}
__device__ __forceinline__ uint32_t two_bf16(float a, float b) {
    const __nv_bfloat162 x = __floats2bfloat162_rn(a, b);
    return *reinterpret_cast<const uint32_t *>(&x);
}
__device__ __forceinline__ void store_piece(__nv_bfloat16 *p, const Piece<__nv_bfloat16, 8> &r) {
    *reinterpret_cast<uint4 *>(p) = make_uint4(two_bf16(r.v[0], r.v[1]), two_bf16(r.v[2], r.v[3]),
                                               two_bf16(r.v[4], r.v[5]), two_bf16(r.v[6], r.v[7]));
}
__device__ __forceinline__ void store_piece(float *p, const Piece<float, 1> &r) { *p = r.v[0]; }
__device__ __forceinline__ void store_piece(__nv_bfloat16 *p, const Piece<__nv_bfloat16, 1> &r) {
    *p = __float2bfloat16_rn(r.v[0]);
}

// A piece as it lies in memory: what a thread holds of a row on its way.
template <typename E, int N>
struct Bits {
    uint4 w;
};
template <typename E>
struct Bits<E, 1> {
    E w;
};
template <typename E, int N>
__device__ __forceinline__ void load_bits(const E *p, Bits<E, N> &r) {
    r.w = *reinterpret_cast<const decltype(r.w) *>(p);
}
template <typename E, int N>
__device__ __forceinline__ Piece<E, N> values(const Bits<E, N> &b) {
    Piece<E, N> r;
    load_piece(reinterpret_cast<const E *>(&b.w), r);
    return r;
}

// Whether rows at `p` with this stride can be read in pieces of 16 bytes.
inline bool by_pieces(const void *p, int64_t stride, int64_t rows, int elem) {
    return !p || (reinterpret_cast<uintptr_t>(p) % 16 == 0 && (rows <= 1 || stride * elem % 16 == 0));
}

}  // namespace dpb
