// Fully connected layer with 4-bit weights and a scale per group of inputs:
//     y[m][o] = act(b[o] + sum_g s[o][g] sum_{i in g} (code[o][i] - z[o][g]) x[m][i]).
//
// The differences code - z are whole numbers of at most 15, exact in either
// 16-bit type, so the inner sums run on the matrix cores with no rounding but
// that of the fp32 accumulator, and the scale multiplies the group's sum, not
// the weights.  A wave owns 16 FN output channels for up to 16 FM rows and a
// range of K; it streams codes and activations from global memory straight to
// registers in the operands' own order.
//
// At few rows the codes' bytes bound it, at many rows the products.
#include "device.h"

namespace mgi {
namespace kern {

namespace {

typedef uint32_t u4v __attribute__((ext_vector_type(4)));
typedef _Float16 h2 __attribute__((ext_vector_type(2)));

// Eight codes of a word minus the zero point as an MFMA fragment.
template <typename E>
struct Codes;

// fp16: 0x6400 | q is the value 1024 + q; subtracting 1024 + z is exact
template <>
struct Codes<F16> {
    h2 off;
    __device__ __forceinline__ explicit Codes(uint32_t z) {
        const uint32_t b = 0xE400u | z;                    // -(1024 + z)
        off = __builtin_bit_cast(h2, b | b << 16);
    }
    __device__ __forceinline__ h8 frag(uint32_t w) const {
        u4x r;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const uint32_t q = (w >> (4 * i) & 0x000F000Fu) | 0x64006400u;
            r[i] = __builtin_bit_cast(uint32_t, __builtin_bit_cast(h2, q) + off);
        }
        return __builtin_bit_cast(h8, r);
    }
};

// bf16: through fp32, whose upper halves are the (exact) bf16 values
template <>
struct Codes<BF16> {
    float z;
    __device__ __forceinline__ explicit Codes(uint32_t z_) : z((float)z_) {}
    __device__ __forceinline__ h8 frag(uint32_t w) const {
        const uint32_t even = w & 0x0F0F0F0Fu, odd = w >> 4 & 0x0F0F0F0Fu;   // pairs 0, 2 and 1, 3
        u4x r;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const uint32_t q = (i & 1 ? odd : even) >> (i & 2 ? 8 : 0);
            const float lo = (float)(q & 0xFFu) - z, hi = (float)(q >> 16 & 0xFFu) - z;
            r[i] = __builtin_amdgcn_perm(__float_as_uint(hi), __float_as_uint(lo), 0x07060302u);
        }
        return __builtin_bit_cast(h8, r);
    }
};

template <typename E>
__device__ __forceinline__ float scale_of(uint16_t b) {
    return E::bf ? __uint_as_float((uint32_t)b << 16) : (float)__builtin_bit_cast(_Float16, b);
}

// One block of 128 inputs in flight: codes, scales, zero points, activations.
template <int FM, int FN, int GS, bool ZP>
struct Stage {
    static constexpr int SG = 4 / GS;      // scales per channel and block
    u4v w[FN];
    uint32_t s[FN][2 * SG], z[FN];
    h8 x[4][FM];
};

template <typename E, int FM, int FN, int GS, bool ZP>
__global__ __launch_bounds__(512) void fcint4_kernel(FcInt4Params p, int splits) {
    constexpr int F = FM * FN, PF = 2;
    typedef Stage<FM, FN, GS, ZP> St;
    constexpr int SG = St::SG;
    extern __shared__ f4 red[];            // [waves][F][64]
    __shared__ int last;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, waves = blockDim.x >> 6;
    // row tiles of the same weights are neighbours, which xcd_tile puts on one XCD
    const int t = xcd_tile(blockIdx.x, gridDim.x);
    const int mt = t % p.mtiles, r = t / p.mtiles, split = r % splits, nt = r / splits;
    const int m0 = mt * 16 * FM, nb0 = nt * FN;
    const int parts = waves * splits, part = split * waves + wave;
    const int b0 = (int)((long)p.kb * part / parts), b1 = (int)((long)p.kb * (part + 1) / parts);
    const h8 *xl[FM];
#pragma unroll
    for (int j = 0; j < FM; ++j) xl[j] = p.x + (size_t)min(m0 + j * 16 + (lane & 15), p.M - 1) * p.xp;
    f4 acc[FN][FM];
#pragma unroll
    for (int i = 0; i < FN; ++i)
#pragma unroll
        for (int j = 0; j < FM; ++j) acc[i][j] = f4{0.f, 0.f, 0.f, 0.f};

    auto load = [&](int b, St &st) {
#pragma unroll
        for (int i = 0; i < FN; ++i) {
            const size_t at = (size_t)min(nb0 + i, p.nb16 - 1) * p.kb + b;
            st.w[i] = ((const u4v *)p.w)[at * 64 + lane];
            __builtin_memcpy(st.s[i], p.scales + (at * 16 + 4 * (lane >> 4)) * SG, 8 * SG);
            if (ZP) {
                const uint8_t *z = p.zp + (at * 16 + (lane & 15)) * SG;
                st.z[i] = SG == 4 ? *(const uint32_t *)z : SG == 2 ? *(const uint16_t *)z : *z;
            }
        }
        const bool edge = b * 16 + 16 > p.ksl;
#pragma unroll
        for (int s = 0; s < 4; ++s) {
            const int ks = b * 16 + s * 4 + (lane >> 4);
#pragma unroll
            for (int j = 0; j < FM; ++j)
                st.x[s][j] = *(edge && ks >= p.ksl ? p.zero : xl[j] + (size_t)ks * p.xs);
        }
    };
    auto compute = [&](const St &st) {
#pragma unroll
        for (int q = 0; q < SG; ++q)
#pragma unroll
            for (int i = 0; i < FN; ++i) {
                const Codes<E> code(ZP ? st.z[i] >> (8 * q) & 15 : 8);
                f4 g[FM];
#pragma unroll
                for (int j = 0; j < FM; ++j) g[j] = f4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int s = 0; s < GS; ++s) {
                    const h8 w = code.frag(st.w[i][q * GS + s]);
#pragma unroll
                    for (int j = 0; j < FM; ++j) g[j] = E::mma(w, st.x[q * GS + s][j], g[j]);
                }
#pragma unroll
                for (int c = 0; c < 4; ++c) {
                    const float sc = scale_of<E>((uint16_t)(st.s[i][(c * SG + q) >> 1] >> (16 * ((c * SG + q) & 1))));
#pragma unroll
                    for (int j = 0; j < FM; ++j) acc[i][j][c] = fmaf(sc, g[j][c], acc[i][j][c]);
                }
            }
    };
    if (b0 < b1) {
        St st[PF];
#pragma unroll
        for (int u = 0; u < PF; ++u) load(min(b0 + u, b1 - 1), st[u]);
        for (int b = b0; b < b1; b += PF) {
#pragma unroll
            for (int u = 0; u < PF; ++u) {
                if (b + u < b1) compute(st[u]);
                if (b + u + PF < b1) load(b + u + PF, st[u]);
            }
        }
    }
#pragma unroll
    for (int i = 0; i < FN; ++i)
#pragma unroll
        for (int j = 0; j < FM; ++j) red[(wave * F + i * FM + j) * 64 + lane] = acc[i][j];
    __syncthreads();
    // the waves' sums, in a fixed order; of several workgroups that share K
    // each leaves its sum, and the last to arrive adds them, again in order
    f4 *mine = splits > 1 ? (f4 *)p.part + ((size_t)(nt * p.mtiles + mt) * splits + split) * F * 64 : nullptr;
    for (int f = wave; f < F; f += waves) {
        f4 v = red[f * 64 + lane];
        for (int w = 1; w < waves; ++w) v += red[(w * F + f) * 64 + lane];
        if (splits > 1) {
            typedef unsigned long long u64;
            u64 *to = (u64 *)(mine + f * 64 + lane);
            put(to, (u64)__float_as_uint(v[1]) << 32 | __float_as_uint(v[0]));
            put(to + 1, (u64)__float_as_uint(v[3]) << 32 | __float_as_uint(v[2]));
        } else {
            red[f * 64 + lane] = v;
        }
    }
    if (splits > 1) {
        if (!arrive_last(p.cnt + nt * p.mtiles + mt, splits, &last)) return;
        const f4 *first = mine - (size_t)split * F * 64;
        for (int f = wave; f < F; f += waves) {
            f4 v = first[f * 64 + lane];
            for (int q = 1; q < splits; ++q) v += first[((size_t)q * F + f) * 64 + lane];
            red[f * 64 + lane] = v;
        }
    }
    const bool vec = p.cout % 4 == 0 && ((uintptr_t)p.y & 15) == 0;
    for (int f = wave; f < F; f += waves) {
        const f4 v = red[f * 64 + lane];       // (written by this wave)
        const int nb = nb0 + f / FM, m = m0 + (f % FM) * 16 + (lane & 15), n = nb * 16 + 4 * (lane >> 4);
        if (nb >= p.nb16 || m >= p.M) continue;
        const f4 mul = *(const f4 *)(p.mul + n), bias = *(const f4 *)(p.bias + n);
        f4 o;
#pragma unroll
        for (int c = 0; c < 4; ++c) {          // (comparisons keep a NaN, a clamp would not)
            const float u = fmaf(v[c], mul[c], bias[c]);
            o[c] = p.act != MGI_ACT_NONE && u < 0.0f ? 0.0f : p.act == MGI_ACT_RELU6 && u > 6.0f ? 6.0f : u;
        }
        float *y = p.y + (size_t)m * p.cout + n;
        if (vec) {
            if (n < p.cout) *(f4 *)y = o;
        } else {
#pragma unroll
            for (int c = 0; c < 4; ++c)
                if (n + c < p.cout) y[c] = o[c];
        }
    }
}

template <typename E, int FM, int FN, int GS>
hipError_t launch_z(const FcInt4Params &p, const FcInt4Geom &g, hipStream_t st) {
    const size_t lds = (size_t)g.waves * FM * FN * 1024;
    const dim3 grid((unsigned)(g.tiles(p.M, p.nb16) * g.splits)), block(64 * g.waves);
    if (p.zp) launch(fcint4_kernel<E, FM, FN, GS, true>, grid, block, lds, st, p, g.splits);
    else launch(fcint4_kernel<E, FM, FN, GS, false>, grid, block, lds, st, p, g.splits);
    return hipGetLastError();
}

template <typename E>
hipError_t launch_e(const FcInt4Params &p, const FcInt4Geom &g, hipStream_t st) {
#define MGI_FCINT4(FM_, FN_)                                                     \
    if (g.fm == FM_ && g.fn == FN_) {                                             \
        if (g.gs == 1) return launch_z<E, FM_, FN_, 1>(p, g, st);                 \
        if (g.gs == 2) return launch_z<E, FM_, FN_, 2>(p, g, st);                 \
        if (g.gs == 4) return launch_z<E, FM_, FN_, 4>(p, g, st);                 \
    }
    MGI_FCINT4(1, 1) MGI_FCINT4(1, 2) MGI_FCINT4(2, 2)
#undef MGI_FCINT4
    return hipErrorInvalidValue;
}

}  // namespace

FcInt4Geom fcint4_geom(int M, int nb16, int kb, int group) {
    FcInt4Geom g{};
    g.gs = group % 128 == 0 ? 4 : group % 64 == 0 ? 2 : 1;
    g.fm = M <= 16 ? 1 : 2;
    g.fn = g.fm == 1 && nb16 < 512 ? 1 : 2;
    g.waves = std::max(1, std::min(4, kb));
    g.splits = 1;
    return g;
}

hipError_t launch_fcint4(const FcInt4Params &p0, const FcInt4Geom &g, hipStream_t st) {
    FcInt4Params p = p0;
    if (p.M <= 0) return hipSuccess;
    p.mtiles = (p.M + 16 * g.fm - 1) / (16 * g.fm);
    p.ntiles = (p.nb16 + g.fn - 1) / g.fn;
    if (g.waves < 1 || g.waves > 8 || g.splits < 1 || (g.splits > 1 && (!p.part || !p.cnt)) ||
        (size_t)p.mtiles * p.ntiles * g.splits > 0x7fffffffu || p.kb * 16 < p.ksl)
        return hipErrorInvalidValue;
    return p.bf16 ? launch_e<BF16>(p, g, st) : launch_e<F16>(p, g, st);
}

}  // namespace kern
}  // namespace mgi
