// Pointwise layer in 8-bit floating point (e4m3).
//
//   y[m][o] = act(b[o] + sum_kb sw[o / 128][kb] 2^e[m][kb] sum_{i in kb} cw[o][i] q[m][i])
//
// One matrix instruction multiplies a block of 128 inputs; its operands for
// exponents take the pixels' powers of two and the weight scale's, which scales
// exactly, and the blocks' sums go into the fp32 result times the rest of the scale,
// 1 to 2: no sum leaves fp32's range whose share of the result does not.  The instruction
// adds eight products at a time with their bits below 2^-13 of the largest's
// leading one cut off, and those sums in fp32 (measured; the unscaled 8-bit
// instructions do the same).  That is 2^-16 of a result of normal values, under
// the 16-bit output's step; products in 16 bits, which would be exact, run at half
// the rate and need the codes converted.
#include <type_traits>

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
// exponents of four blocks, `k`: the weights' exponent
template <int Q>
__device__ __forceinline__ f4 mma8(i8v w, i8v x, uint32_t k, uint32_t e) {
    return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(w, x, f4{}, 0, 0, 0, (int)k, Q, (int)e);
}

// a scale is 2^(k - 127) times what is left in s, 1 to 2 (less where it is subnormal or zero)
__device__ __forceinline__ uint32_t split_scale(float &s) {
    const uint32_t bits = __float_as_uint(s), k = bits >> 23 & 255;
    s = k ? __uint_as_float((bits & 0x807fffffu) | 0x3f800000u) : s * 0x1p126f;
    return max(k, 1u);
}

// A block of a pixel's inputs, 32 of them to each of the lanes l, l ^ 16, l ^ 32,
// l ^ 48, in 8 bits: the codes in the operand's order and the exponent's byte.
// Magnitudes are compared as 16-bit integers, and pairs are scaled and converted by
// one instruction; blocks with infinities or NaN take the quantize kernel's way.
template <typename E>
__device__ __forceinline__ uint32_t to_8_bits(const uint4 (&raw)[4], i8v &codes) {
    typedef uint16_t u16x2 __attribute__((ext_vector_type(2)));
    const uint32_t *words = (const uint32_t *)raw;
    u16x2 most{};
#pragma unroll
    for (int i = 0; i < 16; ++i) most = __builtin_elementwise_max(most, __builtin_bit_cast(u16x2, words[i] & 0x7fff7fffu));
    uint32_t top = max(most[0], most[1]);
    top = max(top, (uint32_t)__shfl_xor((int)top, 16, 64));
    top = max(top, (uint32_t)__shfl_xor((int)top, 32, 64));
    if (__any(top >= (E::bf ? 0x7f80u : 0x7c00u))) {
        float t = 0.0f;
#pragma unroll
        for (int h = 0; h < 4; ++h) t = fmaxf(t, finite_top<E>(__builtin_bit_cast(h8, raw[h])));
        t = fmaxf(t, __shfl_xor(t, 16, 64));
        t = fmaxf(t, __shfl_xor(t, 32, 64));
        const int e = block_exponent(t);
#pragma unroll
        for (int h = 0; h < 4; ++h) {
            const uint2 q = codes8<E>(__builtin_bit_cast(h8, raw[h]), power2(-e));
            codes[2 * h] = (int)q.x;
            codes[2 * h + 1] = (int)q.y;
        }
        return (uint32_t)(e + 127);
    }
    h8 one = zero_h8();
    {
        u16x8 b = bits8(one);
        b[0] = (uint16_t)top;
        one = __builtin_bit_cast(h8, b);
    }
    const int e = block_exponent(E::get(one, 0));
    const float up = power2(e);
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        typedef short s2 __attribute__((ext_vector_type(2)));
        s2 q{};
        if constexpr (E::bf) {
            typedef __bf16 b2 __attribute__((ext_vector_type(2)));
            q = __builtin_amdgcn_cvt_scalef32_pk_fp8_bf16(q, __builtin_bit_cast(b2, words[2 * i]), up, false);
            q = __builtin_amdgcn_cvt_scalef32_pk_fp8_bf16(q, __builtin_bit_cast(b2, words[2 * i + 1]), up, true);
        } else {
            typedef _Float16 f2 __attribute__((ext_vector_type(2)));
            q = __builtin_amdgcn_cvt_scalef32_pk_fp8_f16(q, __builtin_bit_cast(f2, words[2 * i]), up, false);
            q = __builtin_amdgcn_cvt_scalef32_pk_fp8_f16(q, __builtin_bit_cast(f2, words[2 * i + 1]), up, true);
        }
        codes[i] = __builtin_bit_cast(int, q);
    }
    return (uint32_t)(e + 127);
}

// f for each of up to four blocks, those of a word of exponents
template <typename F>
__device__ __forceinline__ void four_blocks(int n, F f) {
    f(std::integral_constant<int, 0>{});
    if (n > 1) f(std::integral_constant<int, 1>{});
    if (n > 2) f(std::integral_constant<int, 2>{});
    if (n > 3) f(std::integral_constant<int, 3>{});
}

// A slice of a pixel's results, one of those up to channel `end`.  Channels past the
// last hold zeros, which the zero weights there do not give for a pixel with NaN.
template <typename E>
__device__ __forceinline__ void store_slice(const PwFp8Params &p, int end, int s, int m, float *v) {
    if (m >= p.M || s >= p.ns) return;
    if (end > p.cout) {
#pragma unroll
        for (int c = 0; c < 8; ++c) v[c] = s * 8 + c < p.cout ? v[c] : 0.0f;
    }
    store8<E>(p.y, s, m, E::pack(v));
}

// Of two neighbouring blocks of 16 channels (a, b; channels 4 quad .. + 3 of a
// pixel to a lane) each lane completes one slice: of the first where its quad is
// even, of the second where it is odd.
template <typename E>
__device__ __forceinline__ void store_pair(const PwFp8Params &p, f4 a, f4 b, int nb, int m, int quad) {
    float v[8];
    const bool odd = quad & 1;
#pragma unroll
    for (int r = 0; r < 4; ++r) {
        a[r] = pinned(act_keep(a[r], p.act));
        b[r] = pinned(act_keep(b[r], p.act));
        const float other = __shfl_xor(odd ? a[r] : b[r], 16, 64);
        v[r] = odd ? other : a[r];
        v[4 + r] = odd ? b[r] : other;
    }
    const int s = (nb + odd) * 2 + (quad >> 1);
    store_slice<E>(p, nb * 16 + 32, s, m, v);
}

// Few pixels: bound by the weights' bytes and latency.  A workgroup has 16 channels
// and 16 * FM pixels; its eight waves take the blocks of inputs in turn, four at a
// time with all loads in flight, and their sums are added in the order of the waves.
// RAW: the pixels are 16-bit and are brought into 8 bits here, as the quantize
// kernel does, which saves its launch (1 x 4096 x 4096: 6.7 us a call, 7.6 from the
// kernel's start to its end; the host's part takes 5.2 to 5.5).
template <typename E, int FM, bool RAW>
__global__ __launch_bounds__(512) void pwfp8_few_kernel(PwFp8Params p) {
    __shared__ f4 red[8][FM][64];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), col = lane & 15, quad = lane >> 4;
    const int nb = blockIdx.x % p.nb16, m0 = blockIdx.x / p.nb16 * (16 * FM);
    const uint4 *wp = (const uint4 *)p.w + (size_t)nb * p.kb * 128 + lane;
    const float *sp = p.scales + (nb >> 3) * p.kb;
    f4 acc[FM];
    int m[FM];
#pragma unroll
    for (int j = 0; j < FM; ++j) {
        acc[j] = f4{};
        m[j] = min(m0 + j * 16 + col, p.M - 1);
    }
    for (int k0 = wave * 4; k0 < p.kb; k0 += 32) {
        uint4 w[4][2], x[FM][4][RAW ? 4 : 2];
        uint32_t e[FM];
#pragma unroll
        for (int u = 0; u < 4; ++u) {
            const int kb = min(k0 + u, p.kb - 1);
            w[u][0] = wp[(size_t)kb * 128];
            w[u][1] = wp[(size_t)kb * 128 + 64];
        }
#pragma unroll
        for (int j = 0; j < FM; ++j) {
            if constexpr (!RAW) e[j] = p.x.exps[(size_t)(k0 >> 2) * p.M + m[j]];
#pragma unroll
            for (int u = 0; u < 4; ++u) {
                const int kb = min(k0 + u, p.kb - 1);
                if constexpr (RAW) {
#pragma unroll
                    for (int h = 0; h < 4; ++h) {
                        const int s = kb * 16 + (h >> 1) * 8 + quad * 2 + (h & 1);
                        const h8 v = p.raw.x[(size_t)min(s, p.raw_s - 1) * p.raw.s + (size_t)m[j] * p.raw.p];
                        x[j][u][h] = __builtin_bit_cast(uint4, s < p.raw_s ? v : zero_h8());
                    }
                } else {
#pragma unroll
                    for (int h = 0; h < 2; ++h)
                        x[j][u][h] = *((const uint4 *)p.x.codes + (size_t)(kb * 8 + h * 4 + quad) * p.M + m[j]);
                }
            }
        }
        four_blocks(p.kb - k0, [&](auto q) {
            constexpr int u = decltype(q)::value;
            float sw = sp[k0 + u];
            const uint32_t k = split_scale(sw);
#pragma unroll
            for (int j = 0; j < FM; ++j) {
                i8v xv;
                uint32_t ev;
                if constexpr (RAW) {
                    ev = to_8_bits<E>(x[j][u], xv) << (8 * u);
                } else {
                    xv = join(x[j][u][0], x[j][u][1]);
                    ev = e[j];
                }
                const f4 part = mma8<u>(join(w[u][0], w[u][1]), xv, k, ev);
#pragma unroll
                for (int r = 0; r < 4; ++r) acc[j][r] = fmaf(part[r], sw, acc[j][r]);
            }
        });
    }
#pragma unroll
    for (int j = 0; j < FM; ++j) red[wave][j][lane] = acc[j];
    __syncthreads();
    for (int j = wave; j < FM; j += 8) {
        f4 v = *(const f4 *)(p.bias + nb * 16 + quad * 4);
#pragma unroll
        for (int w = 0; w < 8; ++w) v += red[w][j][lane];
        // (the quads' halves of a slice meet)
        const int at = m0 + j * 16 + col, s = nb * 2 + (quad >> 1);
        float y[8];
#pragma unroll
        for (int r = 0; r < 4; ++r) {
            v[r] = pinned(act_keep(v[r], p.act));
            const float other = __shfl_xor(v[r], 16, 64);
            y[r] = quad & 1 ? other : v[r];
            y[4 + r] = quad & 1 ? v[r] : other;
        }
        if ((quad & 1) == 0) store_slice<E>(p, nb * 16 + 16, s, at, y);
    }
}

// Many pixels: PX x CO tiles, a ring of NST stages of one block of 128 inputs each.  Both
// operands come by direct loads in the order of the matrix operands, so that LDS is
// written and read in whole KiB.  A wave has WPX x WCO of the tile.  Steps are without
// branches, four to a round (with them, and with addresses in vector registers: 197 x
// 4096 x 4096 15.5 us, now 13.6; 4096 x 4096 x 4096 68.4, now 66.3).
//
// What bounds it: 8192 x 4096 x 4096 takes 130 us (2.1 PFLOP/s), 61% of them with
// matrix instructions in a tile's steps, and the starts and stores of two rounds of
// tiles about 25.  With the weights' LDS reads taken out it takes 98, without the loads
// to LDS 113, without the inputs' reads 129.  Reading the inputs a block ahead or the
// weights two blocks of channels ahead, and a wave's priority, made no difference.
template <int PX, int CO, int NPX, int NCO>
struct PwTile {
    static constexpr int WAVES = NPX * NCO, FM = PX / NPX / 16, FN = CO / NCO / 16;
    static constexpr int XE = PX * 8, WE = CO * 8;                // 16-byte elements of a stage
    static constexpr int LOADS = (XE + WE) / 64 / WAVES;
    static_assert((XE / 64) % WAVES == 0 && (WE / 64) % WAVES == 0 && FN % 2 == 0, "whole loads to a wave, pairs of channel blocks");
};

template <typename E, int PX, int CO, int NPX, int NCO, int NST>
__global__ __launch_bounds__(64 * NPX * NCO, PX == 128 ? 4 : 2) void pwfp8_tile_kernel(PwFp8Params p) {
    using T = PwTile<PX, CO, NPX, NCO>;
    constexpr int FM = T::FM, FN = T::FN, XL = T::XE / 64 / T::WAVES, WL = T::WE / 64 / T::WAVES;
    static_assert(NST == 2 || NST == 4, "a step's stage is known when it is compiled");
    __shared__ h8 ring[NST][T::XE + T::WE];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), col = lane & 15, quad = lane >> 4;
    // an XCD's tiles are neighbours: of all pixels where those are fewer tiles, so that
    // its weights are read into its L2 once, else of all channels
    const int ct = (p.nb16 * 16 + CO - 1) / CO, mt = (p.M + PX - 1) / PX, tile = xcd_tile(blockIdx.x, gridDim.x);
    const int m0 = (mt < ct ? tile % mt : tile / ct) * PX, n0 = (mt < ct ? tile / mt : tile % ct) * (CO / 16);
    const int wm = wave % NPX * FM, wn = wave / NPX * FN;         // the wave's first pixel and channel block

    // the wave's loads: 64 pixels of a slice of 16 channels; half a block of 16 channels.
    // `more`: another block follows; the last one is loaded again where there is none,
    // so that steps have no branches
    const h8 *xp[XL], *wp[WL];
    uint32_t xo[XL];
#pragma unroll
    for (int i = 0; i < XL; ++i) {
        const int e = wave * XL + i, s = e / (PX / 64), px = e % (PX / 64) * 64 + lane;
        xp[i] = (const h8 *)p.x.codes + (size_t)s * p.M;
        xo[i] = (uint32_t)min(m0 + px, p.M - 1) * 16;
    }
#pragma unroll
    for (int i = 0; i < WL; ++i) {
        const int e = wave * WL + i, nb = min(n0 + e / 2, p.nb16 - 1);
        wp[i] = (const h8 *)p.w + (size_t)nb * p.kb * 128 + (e & 1) * 64;
    }
    const size_t xstep = (size_t)8 * p.M;
    auto issue = [&](bool more, h8 *st) {
#pragma unroll
        for (int i = 0; i < XL; ++i) {
            load_lds16(xp[i], xo[i], st + (wave * XL + i) * 64);
            xp[i] += more ? xstep : 0;
        }
#pragma unroll
        for (int i = 0; i < WL; ++i) {
            load_lds16(wp[i], (uint32_t)lane * 16, st + T::XE + (wave * WL + i) * 64);
            wp[i] += more ? 128 : 0;
        }
    };
    f4 acc[FN][FM];
#pragma unroll
    for (int i = 0; i < FN; ++i)
#pragma unroll
        for (int j = 0; j < FM; ++j) acc[i][j] = f4{};
    const uint32_t *ep[FM];
    uint32_t e[FM], next[FM];
#pragma unroll
    for (int j = 0; j < FM; ++j) {
        ep[j] = p.x.exps + min(m0 + (wm + j) * 16 + col, p.M - 1);
        e[j] = *ep[j];
    }
    // the blocks' scales, one to a lane (read as a scalar in the loop they would wait
    // for the ring's loads)
    static_assert(FN <= 8 && kMaxNormChannels <= 128 * 128, "a wave's channels share a scale; two registers of scales");
    const float *sp = p.scales + (size_t)((n0 + wn) >> 3) * p.kb;
    float s0 = sp[min(lane, p.kb - 1)], s1 = sp[min(64 + lane, p.kb - 1)];
    const uint32_t k0 = split_scale(s0), k1 = split_scale(s1);
#pragma unroll
    for (int i = 0; i < NST - 1; ++i)
        issue(i + 1 < p.kb, ring[i]);
    auto step = [&](auto q, int kb) {
        constexpr int u = decltype(q)::value;
        h8 *st = ring[u % NST];
        wait_vm_lds<(NST - 2) * T::LOADS>();                         // (stages issued after this one stay in flight)
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");
        if (u == 0) {
            const int more = kb + 4 < p.kb ? p.M : 0;
#pragma unroll
            for (int j = 0; j < FM; ++j) next[j] = *(ep[j] += more);
        }
        issue(kb + NST < p.kb, ring[(u + NST - 1) % NST]);
        const float sw = __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(kb < 64 ? s0 : s1), kb & 63));
        const uint32_t k = __builtin_amdgcn_readlane(kb < 64 ? k0 : k1, kb & 63);
        auto weights = [&](int i) {
            const h8 *at = st + T::XE + (wn + i) * 128 + lane;
            return join(__builtin_bit_cast(uint4, at[0]), __builtin_bit_cast(uint4, at[64]));
        };
        i8v x[FM], w = weights(0);
#pragma unroll
        for (int j = 0; j < FM; ++j) {
            const h8 *at = st + quad * PX + (wm + j) * 16 + col;
            x[j] = join(__builtin_bit_cast(uint4, at[0]), __builtin_bit_cast(uint4, at[4 * PX]));
        }
        // the products of a block of channels run while those of the one before are
        // scaled and added, and the next one's weights are read
        f4 part[FM];
#pragma unroll
        for (int i = 0; i <= FN; ++i) {
            i8v wn_;
            if (i + 1 < FN) wn_ = weights(i + 1);
            __builtin_amdgcn_sched_barrier(0);
#pragma unroll
            for (int j = 0; j < FM; ++j) {
                if (i > 0) {
#pragma unroll
                    for (int r = 0; r < 4; ++r) acc[i - 1][j][r] = fmaf(part[j][r], sw, acc[i - 1][j][r]);
                }
                __builtin_amdgcn_sched_barrier(0);
                if (i < FN) part[j] = mma8<u>(w, x[j], k, e[j]);
                __builtin_amdgcn_sched_barrier(0);
            }
            w = wn_;
        }
    };
    int kb = 0;
    for (; kb + 4 <= p.kb; kb += 4) {
        step(std::integral_constant<int, 0>{}, kb);
        step(std::integral_constant<int, 1>{}, kb + 1);
        step(std::integral_constant<int, 2>{}, kb + 2);
        step(std::integral_constant<int, 3>{}, kb + 3);
#pragma unroll
        for (int j = 0; j < FM; ++j) e[j] = next[j];
    }
    if (kb < p.kb) four_blocks(p.kb - kb, [&](auto q) { step(q, kb + decltype(q)::value); });
    wait_vm_lds<0>();                                                 // (no load to LDS outlives the workgroup)
#pragma unroll
    for (int i = 0; i < FN; i += 2) {
        const int nb = n0 + wn + i;
        if (nb >= p.nb16) break;
        const f4 b0 = *(const f4 *)(p.bias + nb * 16 + quad * 4), b1 = *(const f4 *)(p.bias + nb * 16 + 16 + quad * 4);
#pragma unroll
        for (int j = 0; j < FM; ++j) store_pair<E>(p, acc[i][j] + b0, acc[i + 1][j] + b1, nb, m0 + (wm + j) * 16 + col, quad);
    }
}

template <typename E, int PX, int CO, int NPX, int NCO, int NST>
void launch_tile(const PwFp8Params &p, hipStream_t st) {
    const size_t tiles = ((size_t)p.M + PX - 1) / PX * ((p.nb16 * 16 + CO - 1) / CO);
    launch(pwfp8_tile_kernel<E, PX, CO, NPX, NCO, NST>, dim3((unsigned)tiles), dim3(64 * NPX * NCO), 0, st, p);
}

template <typename E, int FM>
void launch_few(const PwFp8Params &p, hipStream_t st) {
    const dim3 grid((unsigned)(((size_t)p.M + 16 * FM - 1) / (16 * FM) * p.nb16));
    launch(pwfp8_few_kernel<E, FM, false>, grid, dim3(512), 0, st, p);
}

template <typename E>
hipError_t launch_pwfp8_t(const PwFp8Params &p, const PwFp8Geom &g, hipStream_t st) {
    switch (g.variant) {
        case 0:
            if (p.raw.x) launch(pwfp8_few_kernel<E, 1, true>, dim3((unsigned)((p.M + 15) / 16 * p.nb16)), dim3(512), 0, st, p);
            else if (p.M <= 16) launch_few<E, 1>(p, st);
            else if (p.M <= 32) launch_few<E, 2>(p, st);
            else launch_few<E, 4>(p, st);
            break;
        case 1: launch_tile<E, 64, 64, 2, 2, 4>(p, st); break;
        case 2: launch_tile<E, 64, 128, 2, 2, 2>(p, st); break;
        case 3: launch_tile<E, 128, 128, 2, 4, 2>(p, st); break;
        case 4: launch_tile<E, 256, 256, 4, 2, 2>(p, st); break;
        default: return hipErrorInvalidValue;
    }
    return hipGetLastError();
}

}  // namespace

// The largest tile that fills the card: of 256 x 256 one to a compute unit, of
// 128 x 128 two, of 64 x 128 one (315 x 1960 x 12032: 16.7 us, by 128 x 128 20.1, by
// 64 x 64 24.0; 2115 x 96 x 6290: 13.4 by 128 x 128, 14.9 by 64 x 128).  Few tiles and many inputs: the kernel of few pixels, which
// shares the inputs out.
PwFp8Geom pwfp8_geom(size_t M, int nb16, int kb) {
    if (M <= 64) return {0};
    auto tiles = [&](size_t px, size_t co) { return (M + px - 1) / px * ((nb16 * 16 + co - 1) / co); };
    if (tiles(256, 256) >= 256) return {4};
    if (tiles(128, 128) >= 512) return {3};
    if (tiles(64, 128) >= 256) return {2};
    if (tiles(64, 64) < 128 && kb >= 16) return {0};
    return {1};
}

hipError_t launch_pwfp8(const PwFp8Params &p, const PwFp8Geom &g, hipStream_t st) {
    if (p.M <= 0) return hipSuccess;
    return p.bf16 ? launch_pwfp8_t<BF16>(p, g, st) : launch_pwfp8_t<F16>(p, g, st);
}

}  // namespace kern
}  // namespace mgi
