// Pointwise layer in 8-bit floating point (e4m3).
//
//   y[m][o] = act(b[o] + sum_kb sw[o / 128][kb] 2^e[m][kb] sum_{i in kb} cw[o][i] q[m][i])
//
// One matrix instruction multiplies a block of 128 inputs; its operand for the
// pixels' exponents takes the powers of two, which scales exactly, and the
// blocks' sums go into the fp32 result times the weights' scale.  The instruction
// adds eight products at a time with their bits below 2^-13 of the largest's
// leading one cut off, and those sums in fp32 (measured; the unscaled 8-bit
// instructions do the same).  That is 2^-16 of a result of normal values, under
// the 16-bit output's step; products in 16 bits, which would be exact, run at half
// the rate and need the codes converted.
#include "tokens.h"

namespace mgi {
namespace kern {

namespace {

typedef int i8v __attribute__((ext_vector_type(8)));

__device__ __forceinline__ i8v join(uint4 a, uint4 b) {
    return i8v{(int)a.x, (int)a.y, (int)a.z, (int)a.w, (int)b.x, (int)b.y, (int)b.z, (int)b.w};
}

// 16 channels x 16 pixels of a block of 128 inputs: lane l has inputs 16 (l / 16)
// .. + 15 and the same + 64 of channel (or pixel) l % 16; `e`: the pixel's
// exponents of four blocks
template <int Q>
__device__ __forceinline__ f4 mma8(i8v w, i8v x, uint32_t e) {
    return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(w, x, f4{}, 0, 0, 0, 0x7f7f7f7f, Q, (int)e);
}
__device__ __forceinline__ f4 mma8(i8v w, i8v x, uint32_t e, int q) {
    switch (q & 3) {
        case 0: return mma8<0>(w, x, e);
        case 1: return mma8<1>(w, x, e);
        case 2: return mma8<2>(w, x, e);
        default: return mma8<3>(w, x, e);
    }
}

// A wave: 16 channels x 64 pixels
template <typename E>
__global__ __launch_bounds__(256) void pwfp8_kernel(PwFp8Params p) {
    __shared__ float stage[4][64][17];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, col = lane & 15, quad = lane >> 4;
    const unsigned cg = (p.nb16 + 3) / 4;
    const int nb = (int)(blockIdx.x % cg) * 4 + wave, m0 = (int)(blockIdx.x / cg) * 64;
    if (nb < p.nb16) {
        f4 acc[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) acc[j] = *(const f4 *)(p.bias + nb * 16 + quad * 4);
        for (int kb = 0; kb < p.kb; ++kb) {
            const uint4 *wp = (const uint4 *)p.w + ((size_t)nb * p.kb + kb) * 128 + lane;
            const i8v w = join(wp[0], wp[64]);
            const float sw = p.scales[(nb >> 3) * p.kb + kb];
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const int m = min(m0 + j * 16 + col, p.M - 1);
                const uint4 *xp = (const uint4 *)p.x.codes + (size_t)(kb * 8 + quad) * p.M + m;
                const i8v x = join(xp[0], xp[(size_t)4 * p.M]);
                const f4 part = mma8(w, x, p.x.exps[(size_t)(kb >> 2) * p.M + m], kb);
#pragma unroll
                for (int r = 0; r < 4; ++r) acc[j][r] = fmaf(part[r], sw, acc[j][r]);
            }
        }
#pragma unroll
        for (int j = 0; j < 4; ++j)
#pragma unroll
            for (int r = 0; r < 4; ++r) stage[wave][j * 16 + col][quad * 4 + r] = act_keep(acc[j][r], p.act);
    }
    __syncthreads();
    if (nb >= p.nb16) return;
#pragma unroll
    for (int k = 0; k < 2; ++k) {
        const int m = m0 + lane, s = nb * 2 + k;
        float v[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = stage[wave][lane][k * 8 + i];
        if (m < p.M && s < p.ns) store8<E>(p.y, s, m, E::pack(v));
    }
}

}  // namespace

PwFp8Geom pwfp8_geom(size_t, int, int) { return PwFp8Geom{0}; }

hipError_t launch_pwfp8(const PwFp8Params &p, const PwFp8Geom &, hipStream_t st) {
    if (p.M <= 0) return hipSuccess;
    const dim3 grid((unsigned)(((size_t)p.M + 63) / 64 * ((p.nb16 + 3) / 4)));
    if (p.bf16) launch(pwfp8_kernel<BF16>, grid, dim3(256), 0, st, p);
    else launch(pwfp8_kernel<F16>, grid, dim3(256), 0, st, p);
    return hipGetLastError();
}

}  // namespace kern
}  // namespace mgi
