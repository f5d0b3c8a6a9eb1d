// Fully connected layer with 4-bit weights and a scale per group of inputs:
//     y[m][o] = act(b[o] + sum_g s[o][g] sum_{i in g} (code[o][i] - z[o][g]) x[m][i]).
//
// The differences code - z are whole numbers of at most 15, exact in either
// 16-bit type, so the inner sums run on the matrix cores with no rounding but
// that of the fp32 accumulator, and the scale multiplies the group's sum, not
// the weights.  Weights come as blocks of 16 output channels x 128 inputs (see
// pack_fc_int4), in the MFMA operand's own order.
//
// At few rows the bytes of the weights bound it, at more the vector work of
// taking codes apart (bf16: 19 instructions for eight codes, fp16: 11) beside
// the products.
#include <type_traits>

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
    // byte q of the word z holds the zero point
    __device__ __forceinline__ Codes(uint32_t z, int q) {
        const uint32_t b = __builtin_amdgcn_perm(z, z, 0x0c000c00u + 0x00010001u * q) | 0xE400E400u;   // -(1024 + z)
        off = __builtin_bit_cast(h2, b);
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

// bf16: code - z of four codes at once as signed bytes (128 + code - z carries
// into no neighbour), then through fp32, whose upper halves are the (exact)
// bf16 values
__device__ __forceinline__ float byte_f32(uint32_t v, int i) { return (float)(int8_t)(v >> (8 * i)); }
template <>
struct Codes<BF16> {
    uint32_t off;
    __device__ __forceinline__ Codes(uint32_t z, int q) : off(0x80808080u - __builtin_amdgcn_perm(z, z, 0x01010101u * q)) {}
    __device__ __forceinline__ h8 frag(uint32_t w) const {
        // pairs 0, 2 and 1, 3
        const uint32_t even = ((w & 0x0F0F0F0Fu) + off) ^ 0x80808080u, odd = ((w >> 4 & 0x0F0F0F0Fu) + off) ^ 0x80808080u;
        u4x r;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const float lo = byte_f32(i & 1 ? odd : even, i >> 1), hi = byte_f32(i & 1 ? odd : even, 2 + (i >> 1));
            r[i] = __builtin_amdgcn_perm(__float_as_uint(hi), __float_as_uint(lo), 0x07060302u);
        }
        return __builtin_bit_cast(h8, r);
    }
};

// scale i of a row of them
template <typename E>
__device__ __forceinline__ float scale_of(const uint32_t *s, int i) {
    const uint32_t v = s[i >> 1];
    if (E::bf) return __uint_as_float(i & 1 ? v & 0xFFFF0000u : v << 16);
    return (float)__builtin_bit_cast(_Float16, (uint16_t)(i & 1 ? v >> 16 : v));
}

// Channels k .. k + 7 of a row of a graph input that is read as it is: fp32, or
// fp16 in rows that are not whole slices or for a bf16 plan.  cin >= 8: near the
// end of a row the load is of its last eight, shifted when they are used.
template <typename T>
struct Raw {
    typedef T v8 __attribute__((ext_vector_type(8)));
    typedef v8 v8u __attribute__((aligned(sizeof(T))));   // (rows start anywhere)
    v8 v;
    __device__ __forceinline__ void load(const T *row, int k, int cin) { v = *(const v8u *)(row + min(k, cin - 8)); }
    // in the plan's type; edge: some row's eight may be past its end (zeros)
    template <typename E>
    __device__ __forceinline__ h8 stored(int k, int cin, bool edge) const {
        v8 u = v;
        if (edge) {
            const int past = k + 8 - cin;
            const v8 zero = (v8)(T)0.0f;
            if (past > 0) {
                if (past & 1) u = __builtin_shufflevector(u, zero, 1, 2, 3, 4, 5, 6, 7, 8);
                if (past & 2) u = __builtin_shufflevector(u, zero, 2, 3, 4, 5, 6, 7, 8, 9);
                if (past & 4) u = __builtin_shufflevector(u, zero, 4, 5, 6, 7, 8, 9, 10, 11);
                if (past >= 8) u = zero;
            }
        }
        if constexpr (sizeof(T) == 2 && !E::bf) {
            return u;
        } else {
            float f[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) f[i] = (float)u[i];
            return E::pack(f);
        }
    }
};

// One block of 128 inputs in flight: codes, scales, zero points, activations
// (T: of a graph input read as it is, or void).
template <int GS, typename T>
struct Stage {
    static constexpr int SG = 4 / GS;      // scales per channel and block
    u4v w;
    uint32_t s[2 * SG], z;
    Raw<T> x[4];
};
template <int GS>
struct Stage<GS, void> {
    static constexpr int SG = 4 / GS;
    u4v w;
    uint32_t s[2 * SG], z;
    h8 x[4];
};

// A 16 x 16 tile of sums to the logits: the scales' power of two, bias, activation.
__device__ __forceinline__ void store_tile(const FcInt4Params &p, const f4 &v, int nb, int m0, int lane) {
    const int m = m0 + (lane & 15), n = nb * 16 + 4 * (lane >> 4);
    if (nb >= p.nb16 || m >= p.M) return;
    const f4 mul = *(const f4 *)(p.mul + n), bias = *(const f4 *)(p.bias + n);
    f4 o;
#pragma unroll
    for (int c = 0; c < 4; ++c) {          // (comparisons keep a NaN, a clamp would not)
        const float u = fmaf(v[c], mul[c], bias[c]);
        o[c] = p.act != MGI_ACT_NONE && u < 0.0f ? 0.0f : p.act == MGI_ACT_RELU6 && u > 6.0f ? 6.0f : u;
    }
    float *y = p.y + (size_t)m * p.cout + n;
    if (p.cout % 4 == 0 && ((uintptr_t)p.y & 15) == 0) {
        if (n < p.cout) *(f4 *)y = o;
    } else {
#pragma unroll
        for (int c = 0; c < 4; ++c)
            if (n + c < p.cout) y[c] = o[c];
    }
}

// Up to 16 rows, few output channels: a workgroup takes 16 channels, its waves
// share K.  Each streams codes and activations from memory to registers, one
// block ahead; the waves' sums are added in a fixed order.
template <typename E, int GS, bool ZP, typename T>
__global__ __launch_bounds__(512) void fcint4_kernel(FcInt4Params p) {
    constexpr int PF = 2;
    constexpr bool RAW = !std::is_void<T>::value;
    typedef Stage<GS, T> St;
    constexpr int SG = St::SG;
    __shared__ f4 red[8][64];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), waves = blockDim.x >> 6;
    // row tiles of the same weights are neighbours, which xcd_tile puts on one XCD
    const int t = xcd_tile(blockIdx.x, gridDim.x);
    const int nb = t / p.mtiles, m0 = (t - nb * p.mtiles) * 16;
    const int b0 = (int)((long)p.kb * wave / waves), b1 = (int)((long)p.kb * (wave + 1) / waves);
    // Addresses are uniform bases plus 32-bit lane offsets that stay the same
    // from block to block, so that a load needs no vector arithmetic.
    const int kg = lane >> 4;
    const h8 *xbase = p.x + (size_t)m0 * p.xp;
    const uint32_t xrow = 16u * (uint32_t)(min(lane & 15, p.M - 1 - m0) * p.xp);
    f4 acc = f4{0.f, 0.f, 0.f, 0.f};

    auto load = [&](int b, St &st) {
        const char *w = (const char *)p.w + ((size_t)nb * p.kb + b) * fcint4_block_bytes(GS, ZP);
        st.w = *(const u4v *)(w + 16u * (uint32_t)lane);
        __builtin_memcpy(st.s, w + 1024u + (uint32_t)(8 * SG * kg), 8 * SG);
        if (ZP) {
            const char *z = w + (1024u + 32 * SG) + (uint32_t)(SG * (lane & 15));
            st.z = SG == 4 ? *(const uint32_t *)z : SG == 2 ? *(const uint16_t *)z : *(const uint8_t *)z;
        }
        if constexpr (RAW) {
            const T *row = (const T *)p.xin + (size_t)(m0 + min(lane & 15, p.M - 1 - m0)) * p.cin;
#pragma unroll
            for (int s = 0; s < 4; ++s) st.x[s].load(row, b * 128 + s * 32 + kg * 8, p.cin);
            return;
        } else {
        // slices past the last are read as the last (and cleared before use)
        const bool edge = b * 16 + 16 > p.ksl;
        uint32_t off[4];
#pragma unroll
        for (int s = 0; s < 4; ++s) off[s] = 16u * (uint32_t)(kg * p.xs);
        if (edge) {
#pragma unroll
            for (int s = 0; s < 4; ++s) {
                const int k0 = min(b * 16 + s * 4, max(p.ksl - 4, 0));
                off[s] = 16u * (uint32_t)((min(b * 16 + s * 4 + kg, p.ksl - 1) - k0) * p.xs);
            }
        }
#pragma unroll
        for (int s = 0; s < 4; ++s) {
            const int k0 = min(b * 16 + s * 4, max(p.ksl - 4, 0));
            st.x[s] = *(const h8 *)((const char *)(xbase + (size_t)k0 * p.xs) + (off[s] + xrow));
        }
        }
    };
    auto compute = [&](int b, St &st) {
        h8 x[4];
#pragma unroll
        for (int s = 0; s < 4; ++s) {
            if constexpr (RAW) x[s] = st.x[s].template stored<E>(b * 128 + s * 32 + kg * 8, p.cin, b * 128 + 128 > p.cin);
            else x[s] = st.x[s];
        }
        if (!RAW && b * 16 + 16 > p.ksl) {
#pragma unroll
            for (int s = 0; s < 4; ++s)
                if (b * 16 + s * 4 + kg >= p.ksl) x[s] = zero_h8();
        }
#pragma unroll
        for (int q = 0; q < SG; ++q) {
            const Codes<E> code(ZP ? st.z : 0x08080808u, q);
            f4 g = f4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int s = q * GS; s < (q + 1) * GS; ++s) g = E::mma(code.frag(st.w[s]), x[s], g);
#pragma unroll
            for (int c = 0; c < 4; ++c) acc[c] = fmaf(scale_of<E>(st.s, c * SG + q), g[c], acc[c]);
        }
    };
    if (b0 < b1) {
        St st[PF];
#pragma unroll
        for (int u = 0; u < PF; ++u) load(min(b0 + u, b1 - 1), st[u]);
        // (a load under a condition would make every wait behind it one for all
        // loads: the last blocks have their own copy of the loop's body)
        int b = b0;
        for (; b + 2 * PF <= b1; b += PF) {
#pragma unroll
            for (int u = 0; u < PF; ++u) {
                compute(b + u, st[u]);
                load(b + u + PF, st[u]);
            }
        }
#pragma unroll
        for (int u = 0; u < PF; ++u) {
            if (b + u < b1) compute(b + u, st[u]);
            if (u + 1 < PF) load(min(b + u + PF, b1 - 1), st[u]);
        }
#pragma unroll
        for (int u = 0; u + 1 < PF; ++u)
            if (b + PF + u < b1) compute(b + PF + u, st[u]);
    }
    red[wave][lane] = acc;
    __syncthreads();
    if (wave > 0) return;
    for (int w = 1; w < waves; ++w) acc += red[w][lane];
    store_tile(p, acc, nb, m0, lane);
}

// More rows or more output channels: a group of NW waves takes 16 channels each
// for the same 16 FM rows, and a wave of its own fetches for it, block after
// block, the rows' activations and the waves' codes into a ring of three stages
// in LDS.  The waves that compute then read activations once per row tile and
// spend no instructions on loads (16 x 8192 x 8192: 13.4 us where every wave
// fetches for itself, 10.3 so).  kgroups such groups share K.
template <int FM, int NW>
struct TileLds {
    static constexpr int X = FM * 4096, W = 1280, STAGE = X + NW * W, STAGES = 3;
};

// A barrier that no access of LDS is moved across (and no wait: each wave has
// waited for what the others are to see).
__device__ __forceinline__ void ring_barrier() {
    asm volatile("" ::: "memory");
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
}
__device__ __forceinline__ void wait_lds() { asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory"); }

// A block of activations, 16 FM rows x 16 slices of 16 bytes, to LDS by one
// wave.  NHWC: a load is four rows of 256 bytes, slices swapped by the row so
// that the reads meet no bank twice; sliced: slice after slice.  Addresses are
// uniform bases plus lane offsets that do not change.
template <int FM, bool NHWC>
struct RowFetch {
    static constexpr int XL = FM * 4;      // loads of a block
    uint32_t ofs[XL];
    int slice[XL];
    const h8 *base;
    __device__ __forceinline__ RowFetch(const FcInt4Params &p, int m0, int lane) {
        const int rows = min(16 * FM, p.M - m0);
#pragma unroll
        for (int q = 0; q < XL; ++q) {
            const int slot = q * 64 + lane;
            const int row = NHWC ? slot >> 4 : slot % (16 * FM);
            slice[q] = NHWC ? (slot & 15) ^ (row & 15) : slot / (16 * FM);
            ofs[q] = 16u * (uint32_t)(min(row, rows - 1) * p.xp + slice[q] * p.xs);
        }
        base = p.x + (size_t)m0 * p.xp;
    }
    __device__ __forceinline__ void issue(const FcInt4Params &p, int b, char *st) const {
        const h8 *x = base + (size_t)(b * 16) * p.xs;
        if (b * 16 + 16 <= p.ksl) {
#pragma unroll
            for (int q = 0; q < XL; ++q) load_lds16(x, ofs[q], (const h8 *)(st + q * 1024));
        } else {                           // slices past the last: zeros
#pragma unroll
            for (int q = 0; q < XL; ++q)
                load_lds16(b * 16 + slice[q] < p.ksl ? (const h8 *)((const char *)x + ofs[q]) : p.zero,
                           (const h8 *)(st + q * 1024));
        }
    }
};

// The wave that fetches a raw graph input for a group of one row tile: through
// registers, a block ahead of the ring, since the values are converted on the
// way; laid out as kNhwc.
template <typename E, typename T, int NW>
__device__ __forceinline__ void fetch_raw(const FcInt4Params &p, int kgroups, int kq, int m0, int steps, char *ring) {
    typedef TileLds<1, NW> L;
    constexpr int XL = 4, AHEAD = L::STAGES - 1;
    const int lane = threadIdx.x & 63, rows = min(16, p.M - m0);
    const int b0 = (int)((long)p.kb * kq / kgroups), b1 = (int)((long)p.kb * (kq + 1) / kgroups);
    const T *row[XL];
    int slice[XL];
#pragma unroll
    for (int q = 0; q < XL; ++q) {
        const int r = q * 4 + (lane >> 4);
        slice[q] = (lane & 15) ^ (r & 15);
        row[q] = (const T *)p.xin + (size_t)(m0 + min(r, rows - 1)) * p.cin;
    }
    Raw<T> x[XL];
    auto block = [&](int i) { return min(b0 + i, b1 - 1); };   // (past the range: its last again)
    auto load = [&](int i) {
#pragma unroll
        for (int q = 0; q < XL; ++q)                           // (what rows past the last hold is not stored)
            if (q * 4 < rows) x[q].load(row[q], block(i) * 128 + slice[q] * 8, p.cin);
    };
    auto write = [&](int i, char *st) {
        const int b = block(i);
#pragma unroll
        for (int q = 0; q < XL; ++q)
            if (q * 4 < rows)
                *(h8 *)(st + (q * 64 + lane) * 16) = x[q].template stored<E>(b * 128 + slice[q] * 8, p.cin, b * 128 + 128 > p.cin);
    };
#pragma unroll
    for (int i = 0; i < AHEAD; ++i) {
        load(i);
        write(i, ring + i * L::STAGE);
    }
    load(AHEAD);
    char *const end = ring + L::STAGES * L::STAGE;
    char *fill = ring + AHEAD * L::STAGE;
    for (int i = 0; i < steps; ++i) {
        wait_lds();                                            // (the writes are done)
        ring_barrier();
        write(i + AHEAD, fill);
        load(i + AHEAD + 1);
        fill = fill + L::STAGE == end ? ring : fill + L::STAGE;
    }
    wait_lds();
    ring_barrier();
}

// (MODE: how the activations are stored, see FcInt4Params)
constexpr int kSliced = 0, kNhwc = 1, kRaw = 2;
template <typename E, int FM, int NW, int GS, bool ZP, int MODE>
__global__ __launch_bounds__(MODE == kRaw ? 1024 : 768) void fcint4_tile_kernel(FcInt4Params p, int kgroups) {
    typedef TileLds<FM, NW> L;
    constexpr bool NHWC = MODE != kSliced;
    constexpr int SG = 4 / GS, BLOCK = fcint4_block_bytes(GS, ZP);
    extern __shared__ f4 red[];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int t = xcd_tile(blockIdx.x, gridDim.x);
    const int nt = t / p.mtiles, m0 = (t - nt * p.mtiles) * 16 * FM;
    const int steps = (p.kb + kgroups - 1) / kgroups;

    if constexpr (MODE == kRaw)
    if (wave >= (NW + 1) * kgroups) {
        const int kq = wave - (NW + 1) * kgroups;
        char *ring = (char *)red + (size_t)kq * L::STAGES * L::STAGE;
        if (p.fp16_in) fetch_raw<E, _Float16, NW>(p, kgroups, kq, m0, steps, ring);
        else fetch_raw<E, float, NW>(p, kgroups, kq, m0, steps, ring);
        if (kgroups > 1) __syncthreads();
        return;
    }
    if (wave >= NW * kgroups) {                       // fetch for group kq
        const int kq = wave - NW * kgroups;
        const int b0 = (int)((long)p.kb * kq / kgroups), b1 = (int)((long)p.kb * (kq + 1) / kgroups);
        char *ring = (char *)red + (size_t)kq * L::STAGES * L::STAGE;
        constexpr int XL = MODE == kRaw ? 0 : FM * 4;
        const RowFetch<FM, NHWC> rows(p, m0, lane);
        const char *wbase[NW];
#pragma unroll
        for (int i = 0; i < NW; ++i)
            wbase[i] = (const char *)p.w + (size_t)__builtin_amdgcn_readfirstlane(min(nt * NW + i, p.nb16 - 1)) * p.kb * BLOCK;
        auto issue = [&](int i, char *st) {           // (past the range: its last block again)
            const int b = __builtin_amdgcn_readfirstlane(min(min(b0 + i, b1 - 1), p.kb - 1));
            if constexpr (MODE != kRaw) rows.issue(p, b, st);
#pragma unroll
            for (int n = 0; n < NW; ++n)
                load_lds16((const h8 *)(wbase[n] + (size_t)b * BLOCK), 16u * (uint32_t)lane, (const h8 *)(st + L::X + n * L::W));
            if (lane < (BLOCK - 1024) / 16) {
#pragma unroll
                for (int n = 0; n < NW; ++n)
                    load_lds16((const h8 *)(wbase[n] + (size_t)b * BLOCK), 1024u + 16u * (uint32_t)lane,
                               (const h8 *)(st + L::X + n * L::W + 1024));
            }
        };
        char *const end = ring + L::STAGES * L::STAGE;
        char *fill = ring + (L::STAGES - 1) * L::STAGE;
#pragma unroll
        for (int i = 0; i < L::STAGES - 1; ++i) issue(i, ring + i * L::STAGE);
        for (int i = 0; i < steps; ++i) {
            // a stage is whole once only the loads of later ones are in flight;
            // behind the barrier all waves are done with the one before it
            wait_vm_lds<(L::STAGES - 2) * (XL + 2 * NW)>();
            ring_barrier();
            issue(i + L::STAGES - 1, fill);
            fill = fill + L::STAGE == end ? ring : fill + L::STAGE;
        }
        wait_vm_lds<0>();
        ring_barrier();
        if (kgroups > 1) __syncthreads();
        return;
    }

    const int ng = wave % NW, kq = wave / NW, kg = lane >> 4, nb = nt * NW + ng;
    const int blocks = (int)((long)p.kb * (kq + 1) / kgroups) - (int)((long)p.kb * kq / kgroups);
    int xoff[4];
#pragma unroll
    for (int s = 0; s < 4; ++s)
        xoff[s] = NHWC ? (lane & 15) * 256 + ((s * 4 + kg) ^ (lane & 15)) * 16 : ((s * 4 + kg) * 16 * FM + (lane & 15)) * 16;
    f4 acc[FM];
#pragma unroll
    for (int j = 0; j < FM; ++j) acc[j] = f4{0.f, 0.f, 0.f, 0.f};
    auto compute = [&](const char *st) {
        const char *w = st + L::X + ng * L::W;
        const u4v codes = *(const u4v *)(w + lane * 16);
        uint32_t sc[2 * SG], z = 0x08080808u;
        __builtin_memcpy(sc, w + 1024 + kg * 8 * SG, 8 * SG);
        if (ZP) {
            const char *zp = w + 1024 + 32 * SG + (lane & 15) * SG;
            z = SG == 4 ? *(const uint32_t *)zp : SG == 2 ? *(const uint16_t *)zp : *(const uint8_t *)zp;
        }
        h8 x[4][FM];
#pragma unroll
        for (int s = 0; s < 4; ++s)
#pragma unroll
            for (int j = 0; j < FM; ++j) x[s][j] = *(const h8 *)(st + xoff[s] + j * (NHWC ? 4096 : 256));
#pragma unroll
        for (int q = 0; q < SG; ++q) {
            const Codes<E> code(z, q);
            f4 g[FM];
#pragma unroll
            for (int j = 0; j < FM; ++j) g[j] = f4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int s = q * GS; s < (q + 1) * GS; ++s) {
                const h8 a = code.frag(codes[s]);
#pragma unroll
                for (int j = 0; j < FM; ++j) g[j] = E::mma(a, x[s][j], g[j]);
            }
#pragma unroll
            for (int c = 0; c < 4; ++c) {
                const float f = scale_of<E>(sc, c * SG + q);
#pragma unroll
                for (int j = 0; j < FM; ++j) acc[j][c] = fmaf(f, g[j][c], acc[j][c]);
            }
        }
    };
    const char *const ring = (const char *)red + (size_t)kq * L::STAGES * L::STAGE, *const end = ring + L::STAGES * L::STAGE;
    const char *cur = ring;
    for (int i = 0; i < steps; ++i) {
        wait_lds();                     // (this wave's reads of the stage before)
        ring_barrier();
        if (i < blocks) compute(cur);
        cur = cur + L::STAGE == end ? ring : cur + L::STAGE;
    }
    wait_lds();
    ring_barrier();
    if (kgroups > 1) {                  // the groups' sums, in a fixed order
#pragma unroll
        for (int j = 0; j < FM; ++j) red[(wave * FM + j) * 64 + lane] = acc[j];
        __syncthreads();
        if (kq > 0) return;
#pragma unroll
        for (int j = 0; j < FM; ++j)
            for (int q = 1; q < kgroups; ++q) acc[j] += red[((q * NW + ng) * FM + j) * 64 + lane];
    }
#pragma unroll
    for (int j = 0; j < FM; ++j) store_tile(p, acc[j], nb, m0 + j * 16, lane);
}

// The differences code - z of a lane's 32 inputs, as 6-bit floats (sign, two bits
// of exponent, three of mantissa; the patterns 0 .. 15 are 0 .. 15 eighths, so
// all are exact), as four MFMA fragments: one instruction.
typedef uint32_t u6v __attribute__((ext_vector_type(6)));
struct Frags {
    h8 a[4];
};
template <typename E>
__device__ __forceinline__ Frags six_bit(u6v w) {
    if constexpr (E::bf) return __builtin_bit_cast(Frags, __builtin_amdgcn_cvt_scalef32_pk32_bf16_fp6(w, 8.0f));
    else return __builtin_bit_cast(Frags, __builtin_amdgcn_cvt_scalef32_pk32_f16_fp6(w, 8.0f));
}

// Many rows: 64 rows x 64 channels, K shared by four groups of two waves, each
// with 32 channels of all rows, and a wave that fetches the group's activations
// into a ring of two stages.  A fragment read from LDS feeds two products, the
// next step's are read before a step's products, and codes, which no other wave
// reads, go to registers, a block ahead.  Taking 4-bit codes apart would take
// longer than the products, so the layer is kept as 6-bit differences for this
// kernel (256 x 4096 x 4096 bf16 19.5 us with 16 channels to a wave, 18.3 with 32,
// 16.2 so).  What bounds it is the traffic from the L2 caches: 0.7 MB to a compute
// unit there.
constexpr int kWideGroups = 4, kWideX = 64 * 256, kWideLds = kWideGroups * 2 * kWideX;
template <typename E, int GS, bool NHWC>
__global__ __launch_bounds__(768) void fcint4_wide_kernel(FcInt4Params p) {
    constexpr int FM = 4, NB = 2, SG = 4 / GS, BLOCK = 1536 + 32 * SG;
    extern __shared__ f4 red[];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int t = xcd_tile(blockIdx.x, gridDim.x);
    const int nt = t / p.mtiles, m0 = (t - nt * p.mtiles) * 16 * FM;
    const int steps = (p.kb + kWideGroups - 1) / kWideGroups;
    const bool fetches = wave >= 2 * kWideGroups;
    const int kq = fetches ? wave - 2 * kWideGroups : wave >> 1;
    const int b0 = (int)((long)p.kb * kq / kWideGroups), b1 = (int)((long)p.kb * (kq + 1) / kWideGroups);
    char *const ring = (char *)red + kq * 2 * kWideX;

    if (fetches) {
        const RowFetch<FM, NHWC> rows(p, m0, lane);
        rows.issue(p, b0, ring);
        for (int i = 0; i < steps; ++i) {
            // block i is whole; behind the barrier all waves are done with block i - 1
            wait_vm_lds<0>();
            ring_barrier();
            rows.issue(p, min(b0 + i + 1, b1 - 1), ring + ((i + 1) & 1) * kWideX);   // (past the range: its last again)
        }
        wait_vm_lds<0>();
        ring_barrier();
        __syncthreads();
        return;
    }

    struct Weights {
        u4v lo;
        uint2 hi;
        uint32_t s[2 * SG];
    };
    const int ng = wave & 1, kg = lane >> 4, nb = nt * 4 + ng * NB;
    const char *wbase[NB];
#pragma unroll
    for (int n = 0; n < NB; ++n) wbase[n] = (const char *)p.w + (size_t)min(nb + n, p.nb16 - 1) * p.kb * BLOCK;
    auto load = [&](int b, Weights *v) {
#pragma unroll
        for (int n = 0; n < NB; ++n) {
            const char *w = wbase[n] + (size_t)b * BLOCK;
            v[n].lo = *(const u4v *)(w + 16u * (uint32_t)lane);
            v[n].hi = *(const uint2 *)(w + 1024u + 8u * (uint32_t)lane);
            __builtin_memcpy(v[n].s, w + 1536u + (uint32_t)(8 * SG * kg), 8 * SG);
        }
    };
    int xoff[4];
#pragma unroll
    for (int s = 0; s < 4; ++s)
        xoff[s] = NHWC ? (lane & 15) * 256 + ((s * 4 + kg) ^ (lane & 15)) * 16 : ((s * 4 + kg) * 16 * FM + (lane & 15)) * 16;
    f4 acc[NB][FM];
#pragma unroll
    for (int n = 0; n < NB; ++n)
#pragma unroll
        for (int j = 0; j < FM; ++j) acc[n][j] = f4{0.f, 0.f, 0.f, 0.f};
    auto compute = [&](const char *st, const Frags *w, const uint32_t (*sc)[2 * SG]) {
        h8 x[2][FM];
        auto read = [&](int s) {
#pragma unroll
            for (int j = 0; j < FM; ++j) x[s & 1][j] = *(const h8 *)(st + xoff[s] + j * (NHWC ? 4096 : 256));
        };
        read(0);
        f4 g[NB][FM];
#pragma unroll
        for (int s = 0; s < 4; ++s) {
            if (s < 3) read(s + 1);
            __builtin_amdgcn_sched_barrier(0);
#pragma unroll
            for (int n = 0; n < NB; ++n)
#pragma unroll
                for (int j = 0; j < FM; ++j)
                    g[n][j] = E::mma(w[n].a[s], x[s & 1][j], s % GS == 0 ? f4{0.f, 0.f, 0.f, 0.f} : g[n][j]);
            if (s % GS != GS - 1) continue;
#pragma unroll
            for (int n = 0; n < NB; ++n)
#pragma unroll
                for (int c = 0; c < 4; ++c) {
                    const float f = scale_of<E>(sc[n], c * SG + s / GS);
#pragma unroll
                    for (int j = 0; j < FM; ++j) acc[n][j][c] = fmaf(f, g[n][j][c], acc[n][j][c]);
                }
        }
    };
    Weights next[NB];
    load(b0, next);
    for (int i = 0; i < steps; ++i) {
        Frags w[NB];
        uint32_t sc[NB][2 * SG];
#pragma unroll
        for (int n = 0; n < NB; ++n) {
            const u4v lo = next[n].lo;
            w[n] = six_bit<E>(u6v{lo[0], lo[1], lo[2], lo[3], next[n].hi.x, next[n].hi.y});
            __builtin_memcpy(sc[n], next[n].s, 8 * SG);
        }
        wait_lds();                     // (this wave's reads of the block before)
        ring_barrier();
        load(min(b0 + i + 1, b1 - 1), next);
        if (b0 + i < b1) compute(ring + (i & 1) * kWideX, w, sc);
    }
    wait_lds();
    ring_barrier();
    // the groups' sums, in a fixed order
#pragma unroll
    for (int n = 0; n < NB; ++n)
#pragma unroll
        for (int j = 0; j < FM; ++j) red[((wave * NB + n) * FM + j) * 64 + lane] = acc[n][j];
    __syncthreads();
    // wave w stores row tile w % 4 of channel blocks w / 4 and 2 + w / 4
#pragma unroll
    for (int u = 0; u < 2; ++u) {
        const int n = u * 2 + (wave >> 2), j = wave & 3;    // (block n is wave n / 2's n % 2)
        f4 v = red[(n * FM + j) * 64 + lane];
#pragma unroll
        for (int q = 1; q < kWideGroups; ++q) v += red[((q * 4 + n) * FM + j) * 64 + lane];
        store_tile(p, v, nt * 4 + n, m0 + j * 16, lane);
    }
}

template <typename E, int GS, bool NHWC>
hipError_t launch_wide(const FcInt4Params &p, hipStream_t st) {
    static_assert(kWideLds >= 2 * kWideGroups * 2 * 4 * 1024, "the groups' sums fit into the ring");
    const dim3 grid((unsigned)p.mtiles * ((p.nb16 + 3) / 4)), block(64 * 3 * kWideGroups);
    launch(fcint4_wide_kernel<E, GS, NHWC>, grid, block, kWideLds, st, p);
    return hipGetLastError();
}

template <typename E, int GS, typename T>
hipError_t launch_stream(const FcInt4Params &p, const FcInt4Geom &g, hipStream_t st) {
    const dim3 grid((unsigned)p.mtiles * p.nb16), block(64 * g.waves);
    if (p.zp) launch(fcint4_kernel<E, GS, true, T>, grid, block, 0, st, p);
    else launch(fcint4_kernel<E, GS, false, T>, grid, block, 0, st, p);
    return hipGetLastError();
}

template <typename E, int FM, int NW, int GS, int MODE>
hipError_t launch_tile(const FcInt4Params &p, const FcInt4Geom &g, hipStream_t st) {
    typedef TileLds<FM, NW> L;
    static_assert(L::STAGES * L::STAGE >= NW * FM * 1024, "the groups' sums fit into the ring");
    const size_t lds = (size_t)g.kgroups * L::STAGES * L::STAGE;
    const dim3 grid((unsigned)p.mtiles * ((p.nb16 + NW - 1) / NW)), block(64 * (NW + (MODE == kRaw ? 2 : 1)) * g.kgroups);
    if (lds > 160 * 1024 || block.x > (MODE == kRaw ? 1024 : 768)) return hipErrorInvalidValue;
    if (p.zp) launch(fcint4_tile_kernel<E, FM, NW, GS, true, MODE>, grid, block, lds, st, p, g.kgroups);
    else launch(fcint4_tile_kernel<E, FM, NW, GS, false, MODE>, grid, block, lds, st, p, g.kgroups);
    return hipGetLastError();
}

template <typename E, int FM, int NW, int GS>
hipError_t launch_mode(const FcInt4Params &p, const FcInt4Geom &g, hipStream_t st) {
    if constexpr (FM == 1)
        if (p.xin) return launch_tile<E, FM, NW, GS, kRaw>(p, g, st);
    if (p.xin) return hipErrorInvalidValue;
    if (p.xp == 1) return launch_tile<E, FM, NW, GS, kSliced>(p, g, st);
    if constexpr (!E::bf) return launch_tile<E, FM, NW, GS, kNhwc>(p, g, st);   // (graph inputs are fp16)
    return hipErrorInvalidValue;
}

template <typename E, int GS>
hipError_t launch_e(const FcInt4Params &p, const FcInt4Geom &g, hipStream_t st) {
    if (g.kgroups == 0 && p.xin && p.fp16_in) return launch_stream<E, GS, _Float16>(p, g, st);
    if (g.kgroups == 0 && p.xin) return launch_stream<E, GS, float>(p, g, st);
    if (g.kgroups == 0) return launch_stream<E, GS, void>(p, g, st);
    if (g.fm == 1 && g.waves == 2) return launch_mode<E, 1, 2, GS>(p, g, st);
    if (g.fm == 1 && g.waves == 4) return launch_mode<E, 1, 4, GS>(p, g, st);
    if (g.fm == 2 && g.waves == 2) return launch_mode<E, 2, 2, GS>(p, g, st);
    if (g.six_bit()) {
        if (p.xin) return hipErrorInvalidValue;
        if (p.xp == 1) return launch_wide<E, GS, false>(p, st);
        if constexpr (!E::bf) return launch_wide<E, GS, true>(p, st);
    }
    return hipErrorInvalidValue;
}

}  // namespace

// (Times are of inputs in the storage type.)  Up to 16 rows: the streaming kernel
// while each compute unit gets at most one block of 16 channels (1 x 4096 x 4096
// 4.8 us, the tile kernel 6.0; 5 x 6816 x 1424 6.8 and 10.0), with up to eight
// waves of at least two blocks of K each; else tiles of 32 channels with four groups along K (7 x 2001 x 5003 5.1 us,
// streaming 5.8; 16 x 8192 x 8192 10.3 and 13.4), or, for more than 16384
// channels, of 64 with two (1 x 4096 x 32000 bf16 18.0 us, 19.8).
// More: tiles of 64 rows x 64 channels where half of them is used, every compute
// unit gets one and each group two blocks of K (256 x 4096 x 4096 bf16 16.2 us,
// 32 x 32 tiles 20.4; 256 x 1024 x 8192 13.0 and 21.0; but 25 x 3545 x 32821 bf16
// 48.3 and 32.1), else of 32 x 32, with up to four groups along K where a compute
// unit gets no second tile (64 x 4096 x 1000 7.8 us, two groups 9.4).
FcInt4Geom fcint4_geom(int M, int nb16, int kb, int group) {
    FcInt4Geom g{};
    g.gs = group % 128 == 0 ? 4 : group % 64 == 0 ? 2 : 1;
    g.fm = 1;
    if (M <= 16 && nb16 <= 256) {
        g.waves = std::max(1, std::min(8, kb / 2));
        return g;
    }
    if (M <= 16) {
        g.waves = nb16 > 1024 ? 4 : 2;
        g.kgroups = std::max(1, std::min(nb16 > 1024 ? 2 : 4, kb / 2));
    } else {
        const bool large = M > 32 && (size_t)((M + 63) / 64) * ((nb16 + 3) / 4) >= 256 && kb >= 8;
        g.fm = large ? 4 : 2;
        g.waves = 2;
        const bool few = (size_t)((M + 31) / 32) * ((nb16 + 1) / 2) <= 256;
        g.kgroups = large ? kWideGroups : kb >= 16 && few ? 4 : kb >= 8 ? 2 : 1;
    }
    return g;
}

hipError_t launch_fcint4(const FcInt4Params &p0, const FcInt4Geom &g, hipStream_t st) {
    FcInt4Params p = p0;
    if (p.M <= 0) return hipSuccess;
    p.mtiles = (p.M + 16 * g.fm - 1) / (16 * g.fm);
    if (g.waves < 1 || g.waves > 8 || g.kgroups < 0 || (size_t)p.mtiles * p.nb16 > 0x7fffffffu || p.kb * 16 < p.ksl ||
        (p.kb - 1) * 16 >= p.ksl)
        return hipErrorInvalidValue;
    if (g.gs == 1) return p.bf16 ? launch_e<BF16, 1>(p, g, st) : launch_e<F16, 1>(p, g, st);
    if (g.gs == 2) return p.bf16 ? launch_e<BF16, 2>(p, g, st) : launch_e<F16, 2>(p, g, st);
    if (g.gs == 4) return p.bf16 ? launch_e<BF16, 4>(p, g, st) : launch_e<F16, 4>(p, g, st);
    return hipErrorInvalidValue;
}

}  // namespace kern
}  // namespace mgi
