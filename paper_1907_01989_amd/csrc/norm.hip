// Root-mean-square norm, alone or of a sum, and 8-bit tensors.
//
//   h = act(a + b) rounded to 16 bits (or a);  y = h w / sqrt(mean h^2 + eps) (or h)
//   8-bit: e the smallest with max |y| <= 448 2^e over 128 channels, code = e4m3(y 2^-e)
//
// One pass: a pixel's channels stay in registers (as the 16-bit values they
// are) between the sum of squares and the output, so that each operand is read
// once.  Scaling by a power of two is exact, so a code differs from the
// definition's only where the fp32 norm rounds across a border between codes.
#include "tokens.h"

namespace mgi {
namespace kern {

namespace {

// P pixels to a wave, 64 / P slices at a time.  P = 8: a wave's lanes cover 8
// pixels x 8 slices, 128 bytes of either layout, twice to a block of 128
// channels; P = 1: four blocks of one pixel.  R: times that a wave comes round.
template <typename E, int P, int R, bool NORM, bool TO8>
__global__ __launch_bounds__(1024) void norm_kernel(NormParams p) {
    constexpr int SUBS = 64 / P, NS = P == 8 ? 2 : 1, CH = SUBS * NS;   // slices of a wave's chunk
    __shared__ float part[16][P];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, W = blockDim.x >> 6;
    const int sub = lane / P, m = blockIdx.x * P + lane % P, mc = min(m, p.M - 1);
    h8 h[R][NS], b[R][NS];
#pragma unroll
    for (int r = 0; r < R; ++r)
#pragma unroll
        for (int j = 0; j < NS; ++j) {
            const int s = min((wave + W * r) * CH + j * SUBS + sub, p.S - 1);
            h[r][j] = p.a.x[(size_t)s * p.a.s + (size_t)mc * p.a.p];
            if (p.b.x) b[r][j] = p.b.x[(size_t)s * p.b.s + (size_t)mc * p.b.p];
        }
    float squares = 0.0f;
#pragma unroll
    for (int r = 0; r < R; ++r)
#pragma unroll
        for (int j = 0; j < NS; ++j) {
            const int s = (wave + W * r) * CH + j * SUBS + sub;
            if (p.b.x) {
                float v[8];
#pragma unroll
                for (int c = 0; c < 8; ++c) v[c] = act_apply(E::get(h[r][j], c) + E::get(b[r][j], c), p.act);
                h[r][j] = E::pack(v);
                if (p.sum.y && s < p.S && m < p.M) store8<E>(p.sum, s, m, h[r][j]);
            }
            if (s >= p.S) h[r][j] = zero_h8();
            if constexpr (NORM) {
#pragma unroll
                for (int c = 0; c < 8; ++c) squares = fmaf(E::get(h[r][j], c), E::get(h[r][j], c), squares);
            }
        }
    float scale = 1.0f;
    if constexpr (NORM) {
#pragma unroll
        for (int d = P; d < 64; d *= 2) squares += __shfl_xor(squares, d, 64);
        if (W > 1) {
            if (sub == 0) part[wave][lane % P] = squares;
            __syncthreads();
            squares = 0.0f;
            for (int w = 0; w < W; ++w) squares += part[w][lane % P];
        }
        scale = 1.0f / sqrtf(fmaf(squares, p.inv_c, p.eps));
    }
#pragma unroll
    for (int r = 0; r < R; ++r) {
        float y[NS][8], top = 0.0f;
#pragma unroll
        for (int j = 0; j < NS; ++j) {
            const int s = (wave + W * r) * CH + j * SUBS + sub;
            if constexpr (NORM) {
                const f4 *wp = (const f4 *)p.w + 2 * min(s, p.KB * 16 - 1);
                const f4 lo = wp[0], hi = wp[1];
#pragma unroll
                for (int c = 0; c < 8; ++c) y[j][c] = E::get(h[r][j], c) * scale * (c < 4 ? lo[c & 3] : hi[c & 3]);
            } else {
#pragma unroll
                for (int c = 0; c < 8; ++c) y[j][c] = E::get(h[r][j], c);
            }
            // (slices past the last hold zeros, which a scale of infinity would turn into NaN)
            if (NORM && s >= p.S) {
#pragma unroll
                for (int c = 0; c < 8; ++c) y[j][c] = 0.0f;
            }
            if constexpr (TO8) {
#pragma unroll
                for (int c = 0; c < 8; ++c) top = fmaxf(top, finite(y[j][c]));
            }
            if (!TO8 && s < p.S && m < p.M) store8<E>(p.out, s, m, E::pack(y[j]));
        }
        if constexpr (TO8) {
#pragma unroll
            for (int d = P; d < 16 / NS * P; d *= 2) top = fmaxf(top, __shfl_xor(top, d, 64));
            const int e = block_exponent(top);
            const float up = power2(e), down = power2(-e);
#pragma unroll
            for (int j = 0; j < NS; ++j) {
                const int s = (wave + W * r) * CH + j * SUBS + sub;
                const uint2 q = codes8(y[j], down);
                if (m >= p.M) continue;
                if (p.q.codes) {
                    if (s < p.KB * 16) {
                        *(uint2 *)(p.q.codes + ((size_t)(s >> 1) * p.M + m) * 16 + (s & 1) * 8) = q;
                        if (s % 16 == 0) ((uint8_t *)(p.q.exps + (size_t)(s >> 6) * p.M + m))[s >> 4 & 3] = (uint8_t)(e + 127);
                    }
                } else if (s < p.S) {
                    float v[8];
                    values8(q, up, v);
                    store8<E>(p.out, s, m, v);
                }
            }
        }
    }
}

template <typename E, int P, int R>
void launch_norm_r(const NormParams &p, dim3 grid, dim3 block, hipStream_t st) {
    if (p.w && p.to8) launch(norm_kernel<E, P, R, true, true>, grid, block, 0, st, p);
    else if (p.w) launch(norm_kernel<E, P, R, true, false>, grid, block, 0, st, p);
    else launch(norm_kernel<E, P, R, false, true>, grid, block, 0, st, p);
}

template <typename E, int P>
hipError_t launch_norm_p(const NormParams &p, hipStream_t st) {
    constexpr int CH = P == 8 ? 16 : 64;
    const int chunks = (p.KB * 16 + CH - 1) / CH;
    int waves = 1, r = 1;
    while (waves < 16 && waves * 4 < chunks) waves *= 2;
    while (waves * r < chunks) r *= 2;
    const dim3 grid(((unsigned)p.M + P - 1) / P), block(64 * waves);
    switch (r) {
        case 1: launch_norm_r<E, P, 1>(p, grid, block, st); break;
        case 2: launch_norm_r<E, P, 2>(p, grid, block, st); break;
        case 4: launch_norm_r<E, P, 4>(p, grid, block, st); break;
        case 8: launch_norm_r<E, P, 8>(p, grid, block, st); break;
        default: return hipErrorInvalidValue;
    }
    return hipGetLastError();
}

__global__ __launch_bounds__(256) void export16_kernel(const h8 *x, uint16_t *y, int M, int C, int S) {
    int m, s;
    if (!plane_place(M, S, m, s)) return;
    const h8 v = x[(size_t)s * M + m];
    uint16_t *d = y + (size_t)m * C + s * 8;
    if (C % 8 == 0 && ((uintptr_t)y & 15) == 0) {
        *(h8 *)d = v;
        return;
    }
#pragma unroll
    for (int c = 0; c < 8; ++c)
        if (s * 8 + c < C) d[c] = bits8(v)[c];
}

__global__ __launch_bounds__(256) void ingest16_kernel(const uint16_t *x, h8 *y, int M, int C, int S) {
    int m, s;
    if (!plane_place(M, S, m, s)) return;
    const uint16_t *d = x + (size_t)m * C + s * 8;
    h8 v = zero_h8();
    if (C % 8 == 0 && ((uintptr_t)x & 15) == 0) {
        v = *(const h8 *)d;
    } else {
#pragma unroll
        for (int c = 0; c < 8; ++c)
            if (s * 8 + c < C) v[c] = __builtin_bit_cast(_Float16, d[c]);
    }
    y[(size_t)s * M + m] = v;
}

template <typename E>
__global__ __launch_bounds__(256) void export8_kernel(Tensor8 x, void *y, int f32, int M, int C, int S) {
    int m, s;
    if (!plane_place(M, S, m, s)) return;
    const uint2 q = *(const uint2 *)(x.codes + ((size_t)(s >> 1) * M + m) * 16 + (s & 1) * 8);
    const float up = power2((int)(x.exps[(size_t)(s >> 6) * M + m] >> (8 * (s >> 4 & 3)) & 255) - 127);
    float v[8];
    values8(q, up, v);
    const h8 r = E::pack(v);
#pragma unroll
    for (int c = 0; c < 8; ++c) {
        if (s * 8 + c >= C) break;
        const size_t at = (size_t)m * C + s * 8 + c;
        if (f32) ((float *)y)[at] = v[c];
        else ((uint16_t *)y)[at] = bits8(r)[c];
    }
}

}  // namespace

hipError_t launch_norm(const NormParams &p, hipStream_t st) {
    if (p.M <= 0) return hipSuccess;
    // one pixel to a wave where there are few; eight else
    if (p.M < 64) return p.bf16 ? launch_norm_p<BF16, 1>(p, st) : launch_norm_p<F16, 1>(p, st);
    return p.bf16 ? launch_norm_p<BF16, 8>(p, st) : launch_norm_p<F16, 8>(p, st);
}

hipError_t launch_export16(const h8 *x, void *y, int M, int C, hipStream_t st) {
    const int S = (C + 7) / 8;
    launch(export16_kernel, dim3(plane_blocks(M, S)), dim3(256), 0, st, x, (uint16_t *)y, M, C, S);
    return hipGetLastError();
}

hipError_t launch_ingest16(const void *x, h8 *y, int M, int C, hipStream_t st) {
    const int S = (C + 7) / 8;
    launch(ingest16_kernel, dim3(plane_blocks(M, S)), dim3(256), 0, st, (const uint16_t *)x, y, M, C, S);
    return hipGetLastError();
}

hipError_t launch_export8(const Tensor8 &x, void *y, bool f32, int M, int C, bool bf16, hipStream_t st) {
    const int S = (C + 7) / 8;
    if (bf16) launch(export8_kernel<BF16>, dim3(plane_blocks(M, S)), dim3(256), 0, st, x, y, (int)f32, M, C, S);
    else launch(export8_kernel<F16>, dim3(plane_blocks(M, S)), dim3(256), 0, st, x, y, (int)f32, M, C, S);
    return hipGetLastError();
}

}  // namespace kern
}  // namespace mgi
