// Root-mean-square norm, alone or of a sum, and 8-bit tensors.
//
//   h = act(a + b) rounded to 16 bits (or a);  y = h w / sqrt(mean h^2 + eps) (or h)
//   8-bit: e the smallest with max |y| <= 448 2^e over 128 channels, code = e4m3(y 2^-e)
//
// The squares are summed in 64 bits, which no 16-bit value overflows and which
// leaves the root's own and the two products with it and the weight as the only fp32
// roundings; for codes what the products round off is kept, and one is left (both
// hide behind the loads: 16384 x 2048 takes 53.1 us with and 52.7 without).
//
// One pass: a pixel's channels stay in registers (as the 16-bit values they
// are) between the sum of squares and the output, so that each operand is read
// once.  Scaling by a power of two is exact, so a code differs from the
// definition's only where the one rounding to fp32 crosses a border between codes.
//
// Bound by memory: 16384 x 2048 bf16 rows, two operands in, their sum and the values of
// the 8-bit norm out, 268 MB in 53.1 us, 5.0 TB/s, what a copy of 1 GiB reaches.  A few rows
// are bound by the host's call (1 x 4096: the kernel 2.9 us).
#include "tokens.h"

namespace mgi {
namespace kern {

namespace {

// x (scale + rest) w, rounded once: with what the two products leave behind, so that
// a code of 8 bits is the neighbour's only where that one rounding crosses a border.
// (Not finite where a product is not, which the codes do not tell apart.)
__device__ __forceinline__ float scaled(float x, float scale, float rest, float w) {
    const float p = pinned(x * scale), q = pinned(p * w);
    const float behind = fmaf(x, rest, fmaf(x, scale, -p));
    return pinned(q + fmaf(behind, w, fmaf(p, w, -q)));
}

// P pixels to a wave, 64 / P slices at a time.  P = 8: a wave's lanes cover 8
// pixels x 8 slices, 128 bytes of either layout, twice to a block of 128
// channels; P = 4, 2, 1: one, two, four blocks of each.  R: times that a wave comes round.
template <typename E, int P, int R, bool NORM, bool TO8>
__global__ __launch_bounds__(1024) void norm_kernel(NormParams p) {
    constexpr int SUBS = 64 / P, NS = P == 8 ? 2 : 1, CH = SUBS * NS;   // slices of a wave's chunk
    __shared__ double part[16][P];
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
    double squares = 0.0;
#pragma unroll
    for (int r = 0; r < R; ++r)
#pragma unroll
        for (int j = 0; j < NS; ++j) {
            const int s = (wave + W * r) * CH + j * SUBS + sub;
            if (p.b.x) {
                float v[8];
#pragma unroll
                for (int c = 0; c < 8; ++c) v[c] = pinned(act_keep(E::get(h[r][j], c) + E::get(b[r][j], c), p.act));
                h[r][j] = E::pack(v);
                if (p.sum.y && s < p.S && m < p.M) store8<E>(p.sum, s, m, h[r][j]);
            }
            if (s >= p.S) h[r][j] = zero_h8();
            if constexpr (NORM) {
#pragma unroll
                for (int c = 0; c < 8; ++c) squares = fma((double)E::get(h[r][j], c), (double)E::get(h[r][j], c), squares);
            }
        }
    float scale = 1.0f, rest = 0.0f;
    int power = 0;
    if constexpr (NORM) {
#pragma unroll
        for (int d = P; d < 64; d *= 2) squares += __shfl_xor(squares, d, 64);
        if (W > 1) {
            if (sub == 0) part[wave][lane % P] = squares;
            __syncthreads();
            squares = 0.0;
            for (int w = 0; w < W; ++w) squares += part[w][lane % P];
        }
        // the factor in two: an exact power of two, and 1/2 to 1 (infinite, zero and NaN
        // factors as they are): of rows of the least and the largest bf16 values it is no
        // normal fp32 value
        const double factor = 1.0 / sqrt(squares * p.inv_c + p.eps);
        scale = (float)__builtin_amdgcn_frexp_mant(factor);
        if constexpr (TO8) rest = (float)(__builtin_amdgcn_frexp_mant(factor) - scale);
        power = __builtin_amdgcn_frexp_exp(factor);
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
                for (int c = 0; c < 8; ++c) {
                    const float x = ldexpf(E::get(h[r][j], c), power), w = c < 4 ? lo[c & 3] : hi[c & 3];
                    if constexpr (TO8) y[j][c] = scaled(x, scale, rest, w);
                    else y[j][c] = pinned(x * scale * w);
                }
            } else {
#pragma unroll
                for (int c = 0; c < 8; ++c) y[j][c] = E::get(h[r][j], c);
            }
            // (channels past the last hold zeros, which a factor of infinity or NaN would turn into NaN)
            if (NORM && s * 8 + 8 > p.C) {
#pragma unroll
                for (int c = 0; c < 8; ++c) y[j][c] = s * 8 + c < p.C ? y[j][c] : 0.0f;
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
    constexpr int CH = P == 8 ? 16 : 64 / P;
    const int chunks = (p.KB * 16 + CH - 1) / CH;
    // at most four rounds of loads to a wave, fewer until the card has four waves to a
    // SIMD
    const int groups = (p.M + P - 1) / P;
    int waves = 1, r = 1;
    while (waves < 16 && (waves * 4 < chunks || (waves < chunks && (size_t)groups * waves < 4096))) waves *= 2;
    while (waves * r < chunks) r *= 2;
    const dim3 grid((unsigned)groups), block(64 * waves);
    switch (r) {
        case 1: launch_norm_r<E, P, 1>(p, grid, block, st); break;
        case 2: launch_norm_r<E, P, 2>(p, grid, block, st); break;
        case 4: launch_norm_r<E, P, 4>(p, grid, block, st); break;
        case 8: launch_norm_r<E, P, 8>(p, grid, block, st); break;
        default: return hipErrorInvalidValue;
    }
    return hipGetLastError();
}

// Whether rows of C values of `size` bytes are whole 16-byte units from y on.
__device__ __forceinline__ bool whole_rows(const void *y, int C) { return C % 8 == 0 && ((uintptr_t)y & 15) == 0; }

// A wave's 8 pixels x 64 channels through LDS, so that memory sees a pixel's
// channels side by side also where they are no whole 16-byte units (2115 x 6290:
// 31 us by single stores from the sliced order).
template <typename T>
__device__ __forceinline__ void store_rows(T *tile, const T *v, T *y, int M, int C, int m, int s) {
    const int lane = threadIdx.x & 63;
#pragma unroll
    for (int c = 0; c < 8; ++c) tile[(lane & 7) * 66 + (lane >> 3) * 8 + c] = v[c];
    __builtin_amdgcn_wave_barrier();
    asm volatile("" ::: "memory");                   // (a wave's LDS accesses are in order as they are written)
    const int m0 = m - (lane & 7), c = (s - (lane >> 3)) * 8 + lane;
#pragma unroll
    for (int i = 0; i < 8; ++i)
        if (m0 + i < M && c < C) y[(size_t)(m0 + i) * C + c] = tile[i * 66 + lane];
}

__global__ __launch_bounds__(256) void export16_kernel(const h8 *x, uint16_t *y, int M, int C, int S) {
    __shared__ uint16_t tile[4][8 * 66];
    int m, s;
    const bool in = plane_place(M, S, m, s);
    const h8 v = x[(size_t)min(s, S - 1) * M + min(m, M - 1)];
    if (whole_rows(y, C)) {
        if (in) *(h8 *)(y + (size_t)m * C + s * 8) = v;
        return;
    }
    uint16_t b[8];
#pragma unroll
    for (int c = 0; c < 8; ++c) b[c] = bits8(v)[c];
    store_rows(tile[threadIdx.x >> 6], b, y, M, C, m, s);
}

__global__ __launch_bounds__(256) void ingest16_kernel(const uint16_t *x, h8 *y, int M, int C, int S) {
    __shared__ uint16_t tiles[4][8 * 66];
    int m, s;
    const bool in = plane_place(M, S, m, s);
    h8 v = zero_h8();
    if (whole_rows(x, C)) {
        if (in) v = *(const h8 *)(x + (size_t)m * C + s * 8);
    } else {
        // (the other way round; zeros past the last channel)
        uint16_t *tile = tiles[threadIdx.x >> 6];
        const int lane = threadIdx.x & 63, m0 = m - (lane & 7), c = (s - (lane >> 3)) * 8 + lane;
        uint16_t row[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) row[i] = m0 + i < M && c < C ? x[(size_t)(m0 + i) * C + c] : 0;
#pragma unroll
        for (int i = 0; i < 8; ++i) tile[i * 66 + lane] = row[i];
        __builtin_amdgcn_wave_barrier();
        asm volatile("" ::: "memory");
        u16x8 b;
#pragma unroll
        for (int i = 0; i < 8; ++i) b[i] = tile[(lane & 7) * 66 + (lane >> 3) * 8 + i];
        v = __builtin_bit_cast(h8, b);
    }
    if (in) y[(size_t)s * M + m] = v;
}

template <typename E>
__global__ __launch_bounds__(256) void export8_kernel(Tensor8 x, void *y, int f32, int M, int C, int S) {
    __shared__ float tile[4][8 * 66];
    int m, s;
    plane_place(M, S, m, s);
    const int mc = min(m, M - 1), sc = min(s, S - 1);
    const uint2 q = *(const uint2 *)(x.codes + ((size_t)(sc >> 1) * M + mc) * 16 + (sc & 1) * 8);
    const float up = power2((int)(x.exps[(size_t)(sc >> 6) * M + mc] >> (8 * (sc >> 4 & 3)) & 255) - 127);
    float v[8];
    values8(q, up, v);
    if (f32) {
        store_rows(tile[threadIdx.x >> 6], v, (float *)y, M, C, m, s);
    } else {
        uint16_t b[8];
        const u16x8 r = bits8(E::pack(v));
#pragma unroll
        for (int c = 0; c < 8; ++c) b[c] = r[c];
        store_rows((uint16_t *)tile[threadIdx.x >> 6], b, (uint16_t *)y, M, C, m, s);
    }
}

// an array's 16-bit values as fp32
template <typename E>
__global__ __launch_bounds__(256) void widen16_kernel(const uint16_t *x, float *y, size_t n) {
    const size_t i = (size_t)blockIdx.x * 256 + threadIdx.x;
    if (i >= n) return;
    u16x8 b{};
    b[0] = x[i];
    y[i] = E::get(__builtin_bit_cast(h8, b), 0);
}

}  // namespace

hipError_t launch_norm(const NormParams &p, hipStream_t st) {
    if (p.M <= 0) return hipSuccess;
    // Sliced tensors want many pixels to a wave, for whole lines of a slice (2048 x 2048
    // sliced to sliced, 1 / 2 / 4 / 8: 16.8, 9.8, 6.8, 5.2 us), few pixels many waves (300
    // x 2048: 6.2, 4.6, 4.0, 4.6).  NHWC ones are lines by themselves: enough pixels to
    // give all lanes channels (100000 x 64: 27.6, 15.6, 10.0, 8.4; 8192 x 1000: 7.8, 7.6,
    // 7.8, 7.7).  Codes alone, 16 bytes of a pixel, are between (norm 197 x 4096: 3.9, 4.5,
    // 5.8, 7.6; 5000 x 4096: 23.5, 18.1, 17.6, 20.3; without the norm 8192 x 4096: 49.5,
    // 39.2, 28.9, 25).
    const bool nhwc = p.a.s == 1 && (!p.b.x || p.b.s == 1) && (!p.sum.y || p.sum.s == 1) && (p.q.codes || p.out.s == 1);
    int P;
    if (p.M < 64) P = 1;
    else if (!nhwc) P = p.M < 256 ? 2 : p.M < 1024 ? 4 : 8;
    else if (p.q.codes) P = p.M < 300 ? 1 : p.M < 2048 ? 2 : p.w ? 4 : 8;
    else P = p.KB == 1 ? 8 : p.KB == 2 ? 4 : 2;
    switch (P) {
        case 1: return p.bf16 ? launch_norm_p<BF16, 1>(p, st) : launch_norm_p<F16, 1>(p, st);
        case 2: return p.bf16 ? launch_norm_p<BF16, 2>(p, st) : launch_norm_p<F16, 2>(p, st);
        case 4: return p.bf16 ? launch_norm_p<BF16, 4>(p, st) : launch_norm_p<F16, 4>(p, st);
        default: return p.bf16 ? launch_norm_p<BF16, 8>(p, st) : launch_norm_p<F16, 8>(p, st);
    }
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

hipError_t launch_widen16(const void *x, float *y, size_t n, bool bf16, hipStream_t st) {
    const dim3 grid((unsigned)((n + 255) / 256));
    if (bf16) launch(widen16_kernel<BF16>, grid, dim3(256), 0, st, (const uint16_t *)x, y, n);
    else launch(widen16_kernel<F16>, grid, dim3(256), 0, st, (const uint16_t *)x, y, n);
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
