// Device helpers of the attention blocks' kernels (gfx950).
#pragma once

#include "device.h"

namespace mgi {
namespace kern {

// (of a vector as a whole: the cast of one element, __builtin_bit_cast(uint16_t,
// v[i]), gives the first one's bits whatever i is)
__device__ __forceinline__ u16x8 bits8(h8 v) { return __builtin_bit_cast(u16x8, v); }

// An fp32 value as it is: without this the compiler may make one instruction of a
// product or sum and its rounding to fp16 (v_fma_mixlo_f16), which rounds once
// where fp32 and then fp16 rounds twice, in some instances of a kernel and not in
// others, whose results then differ.
__device__ __forceinline__ float pinned(float v) {
    asm("" : "+v"(v));
    return v;
}

// 8 channels of (slice, pixel), rounded once to the output's type
template <typename E>
__device__ __forceinline__ void store8(const TokenOut &o, int slice, int pixel, const float *v) {
    const size_t at = (size_t)slice * o.s + (size_t)pixel * o.p;
    if (o.f32) {
        f4 *d = (f4 *)o.y + 2 * at;
        d[0] = f4{v[0], v[1], v[2], v[3]};
        d[1] = f4{v[4], v[5], v[6], v[7]};
    } else {
        ((h8 *)o.y)[at] = E::pack(v);
    }
}

// the same where the values are of the storage type already: fp32 outputs hold
// what the 16-bit tensor would
template <typename E>
__device__ __forceinline__ void store8(const TokenOut &o, int slice, int pixel, h8 v) {
    const size_t at = (size_t)slice * o.s + (size_t)pixel * o.p;
    if (o.f32) {
        f4 *d = (f4 *)o.y + 2 * at;
        d[0] = f4{E::get(v, 0), E::get(v, 1), E::get(v, 2), E::get(v, 3)};
        d[1] = f4{E::get(v, 4), E::get(v, 5), E::get(v, 6), E::get(v, 7)};
    } else {
        ((h8 *)o.y)[at] = v;
    }
}

// ---- 8-bit tensors
// the magnitude of a finite value, 0 of others
__device__ __forceinline__ float finite(float v) { return fabsf(v) < INFINITY ? fabsf(v) : 0.0f; }
template <typename E>
__device__ __forceinline__ float finite_top(h8 v) {
    float top = 0.0f;
#pragma unroll
    for (int c = 0; c < 8; ++c) top = fmaxf(top, finite(E::get(v, c)));
    return top;
}
// The exponent of a block whose largest finite magnitude is `top`: 448 = 1.75 * 2^8.
__device__ __forceinline__ int block_exponent(float top) {
    const uint32_t b = __float_as_uint(top);
    return max((int)(b >> 23) - 127 - 8 + ((b & 0x7fffff) > 0x600000 ? 1 : 0), -126);
}
__device__ __forceinline__ float power2(int e) { return __uint_as_float((uint32_t)(e + 127) << 23); }
// the codes of 8 values times `down`; NaN's where a value is not finite
__device__ __forceinline__ uint2 codes8(const float *y, float down) {
    float v[8];
#pragma unroll
    for (int c = 0; c < 8; ++c) v[c] = fabsf(y[c]) < INFINITY ? y[c] * down : NAN;
    int q[2];
    q[0] = __builtin_amdgcn_cvt_pk_fp8_f32(v[0], v[1], 0, false);
    q[0] = __builtin_amdgcn_cvt_pk_fp8_f32(v[2], v[3], q[0], true);
    q[1] = __builtin_amdgcn_cvt_pk_fp8_f32(v[4], v[5], 0, false);
    q[1] = __builtin_amdgcn_cvt_pk_fp8_f32(v[6], v[7], q[1], true);
    return uint2{(unsigned)q[0], (unsigned)q[1]};
}
template <typename E>
__device__ __forceinline__ uint2 codes8(h8 x, float down) {
    float v[8];
#pragma unroll
    for (int c = 0; c < 8; ++c) v[c] = E::get(x, c);
    return codes8(v, down);
}
// the values of 8 codes times `up`
__device__ __forceinline__ void values8(uint2 q, float up, float *v) {
#pragma unroll
    for (int c = 0; c < 8; c += 4) {
        const int w = (int)(c ? q.y : q.x);
        const auto lo = __builtin_amdgcn_cvt_pk_f32_fp8(w, false), hi = __builtin_amdgcn_cvt_pk_f32_fp8(w, true);
        v[c] = lo[0] * up; v[c + 1] = lo[1] * up; v[c + 2] = hi[0] * up; v[c + 3] = hi[1] * up;
    }
}

// A wave's place in a (pixel, slice) plane: 8 pixels x 8 slices, the pixel
// fastest, so that sliced tensors and NHWC ones both move 128 bytes at a time.
__device__ __forceinline__ bool plane_place(int M, int S, int &m, int &s) {
    const int lane = threadIdx.x & 63;
    const unsigned wave = blockIdx.x * (blockDim.x >> 6) + (threadIdx.x >> 6), sg = (S + 7) / 8;
    m = (int)(wave / sg) * 8 + (lane & 7);
    s = (int)(wave % sg) * 8 + (lane >> 3);
    // (waves past the last have a pixel past the last)
    return m < M && s < S;
}
inline unsigned plane_blocks(int M, int S) { return (unsigned)((((size_t)M + 7) / 8 * (((size_t)S + 7) / 8) + 3) / 4); }

}  // namespace kern
}  // namespace mgi
