// Device helpers of the attention blocks' kernels (gfx950).
#pragma once

#include "device.h"

namespace mgi {
namespace kern {

// (of a vector as a whole: the cast of one element, __builtin_bit_cast(uint16_t,
// v[i]), gives the first one's bits whatever i is)
__device__ __forceinline__ u16x8 bits8(h8 v) { return __builtin_bit_cast(u16x8, v); }

// act_apply that leaves NaN a NaN
__device__ __forceinline__ float act_keep(float v, int act) {
    if (act == MGI_ACT_NONE) return v;
    v = v < 0.0f ? 0.0f : v;
    return act == MGI_ACT_RELU6 && v > 6.0f ? 6.0f : v;
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

// A wave's place in a (pixel, slice) plane: 8 pixels x 8 slices, the pixel
// fastest, so that sliced tensors and NHWC ones both move 128 bytes at a time.
__device__ __forceinline__ bool plane_place(int M, int S, int &m, int &s) {
    const int lane = threadIdx.x & 63;
    const unsigned wave = blockIdx.x * (blockDim.x >> 6) + (threadIdx.x >> 6), sg = (S + 7) / 8;
    m = (int)(wave / sg) * 8 + (lane & 7);
    s = (int)(wave % sg) * 8 + (lane >> 3);
    return m < M && s < S;
}
inline unsigned plane_blocks(int M, int S) { return (unsigned)((((size_t)M + 7) / 8 * (((size_t)S + 7) / 8) + 3) / 4); }

}  // namespace kern
}  // namespace mgi
