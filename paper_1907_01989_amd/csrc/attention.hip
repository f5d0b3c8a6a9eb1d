// Attention over images or packed sequences.
//
//   y_i = sum_j p_ij v_j / sum_j p_ij,  p_ij = exp(scale q_i.k_j - m_i)
//
// One pass over the keys with the running maximum m and sum of each row.  Rows
// of a tile are (query, head of the group that shares a head of keys), the head
// fastest, so that one reading of keys and values serves the group.  The scores
// are computed transposed, S^T = K Q^T: a lane has one row's scores of half the
// keys, the other half is in lane ^ 32, and as they come out of the matrix
// instruction they are the operand of O^T = V^T P^T, so P never leaves the
// registers.  m, the sums, the scores and O are fp32; P is rounded to 16 bits
// for the product (an error of half a step relative to each weight, which the
// sum over keys averages; in fp16 half of 2^-31 of the base where that is more),
// its sum is taken before.
//
// What bounds it (MI355X).  Long sequences, 8192 causal tokens, 32 heads of 128 on 8 of
// keys, bf16: 503 to 548 us a call on different cards, 1.0 to 1.09 PFLOP/s, where a
// library's product of 8192 x 8192 x 8192 reaches 1.21.  A wave's step has 1024 cycles of matrix instructions and about
// as many of maxima, exponentials and sums, of which two waves on a SIMD hide little of
// each other's (matrix instructions 58% of a compute unit's busy cycles, vector ones 57%).  Taking half
// of the LDS reads of V out, or the exponentials, changed the time by 7% at most;
// scores of the next tile computed between the weights of this one took 663 us against
// 625 on the same card, a wave's priority made no difference.  Packed short sequences
// (5003 tokens in 13 of them, 16 heads of 80: 42 us): vector instructions 58%, matrix ones
// 34% of the busy cycles, of three waves on a SIMD, and the compute units that hold the
// longest sequence's tiles end last.  One query on 32768 keys: bytes in flight, 134 MB in
// 29 us, 4.6 TB/s with the start.
#include <algorithm>
#include <type_traits>

#include "tokens.h"

namespace mgi {
namespace kern {

namespace {

typedef float f16v __attribute__((ext_vector_type(16)));

constexpr int kBN = 64;              // keys of a tile that waves share
constexpr int kPrivate = 32;         // ... and of a wave's own
constexpr float kSlack = 8.0f;       // log2 of how far weights may pass 1 before the base is moved
// log2 of a factor of all of a row's weights, which its division takes out again: fp16
// ends at 65504 and its last step is 2^-24, so that with weights of up to 2^15 only those
// below 2^-32 of the base are lost, not those of 2^-25, of which a row may have tens of
// thousands
template <typename E>
constexpr float kLift = E::bf ? 0.0f : 7.0f;

// Rows of a tile: 32 to a wave; WR waves along the rows, the others of the four
// along the keys.
__host__ __device__ constexpr int tile_rows(int wr) { return 32 * wr; }

template <typename E>
__device__ __forceinline__ f16v mma32(h8 a, h8 b, f16v c) {
    if constexpr (E::bf)
        return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bh8, a), __builtin_bit_cast(bh8, b), c, 0, 0, 0);
    else
        return __builtin_amdgcn_mfma_f32_32x32x16_f16(a, b, c, 0, 0, 0);
}

// the larger of a lane's value and lane ^ 32's, without a way through LDS (8192 causal
// tokens: 589 -> 580 us)
__device__ __forceinline__ float larger_half(float v) {
    const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}

// A tile of query rows: the sequence's queries and keys, and the tile's number
// among the sequence's.
struct Tile {
    int q0, nq, k0, nk, tile;
    bool none;
};

// Over the lanes of a wave: sums and maxima up to each lane (values of at least 0),
// the left neighbour's value
template <typename F>
__device__ __forceinline__ int scan(int v, F join) {
    v = join(v, __builtin_amdgcn_update_dpp(0, v, 0x111, 0xf, 0xf, false));   // shifts within rows of 16
    v = join(v, __builtin_amdgcn_update_dpp(0, v, 0x112, 0xf, 0xf, false));
    v = join(v, __builtin_amdgcn_update_dpp(0, v, 0x114, 0xf, 0xf, false));
    v = join(v, __builtin_amdgcn_update_dpp(0, v, 0x118, 0xf, 0xf, false));
    v = join(v, __builtin_amdgcn_update_dpp(0, v, 0x142, 0xa, 0xf, false));   // a row's last lane to the next row
    return join(v, __builtin_amdgcn_update_dpp(0, v, 0x143, 0xc, 0xf, false));   // ... to the upper half
}
__device__ __forceinline__ int scan_add(int v) { return scan(v, [](int a, int b) { return a + b; }); }
__device__ __forceinline__ int scan_max(int v) { return scan(v, [](int a, int b) { return max(a, b); }); }
__device__ __forceinline__ int from_left(int v, int first) { return __builtin_amdgcn_update_dpp(first, v, 0x138, 0xf, 0xf, false); }

// Finds tile `t` among the tiles of all sequences.  Bounds are read up to the
// token count and not below their predecessors.  Two more sequences without
// keys take the queries before the first bound and behind the last.  Every workgroup
// goes through the bounds before its own, 64 at a time, which thousands of short
// sequences pay for (16384 of 16 tokens, 8 heads of 64: 22.2 ms, as images 1.2).
template <int BM>
__device__ __forceinline__ Tile find_tile(const AttentionParams &p, int t) {
    Tile r;
    r.none = false;
    if (!p.bq) {
        const int per = (p.tq * p.group + BM - 1) / BM, image = t / per;
        r.q0 = image * p.tq;
        r.nq = p.tq;
        r.k0 = image * p.tk;
        r.nk = p.tk;
        r.tile = per - 1 - (t - image * per);   // (causal: the longest first)
        return r;
    }
    const int lane = threadIdx.x & 63;
    int qmax = 0, kmax = 0, before = 0;
    for (int base = 0; base < p.nseq + 2; base += 64) {
        const int i = base + lane, at = min(i, p.nseq);
        const int qv = p.bq[at], kv = p.bk ? p.bk[at] : qv;
        const int qe = max(scan_max(i <= p.nseq ? min(max(qv, 0), p.tq) : p.tq), qmax);
        const int ke = max(scan_max(i <= p.nseq ? min(max(kv, 0), p.tk) : p.tk), kmax);
        const int qs = from_left(qe, qmax), ks = from_left(ke, kmax);
        const int upto = before + scan_add(i < p.nseq + 2 ? ((qe - qs) * p.group + BM - 1) / BM : 0);
        const uint64_t has = __ballot(upto > t);
        if (has) {
            const int src = __builtin_ctzll(has);
            const bool keys = base + src != 0 && base + src != p.nseq + 1;
            r.q0 = __builtin_amdgcn_readlane(qs, src);
            r.nq = __builtin_amdgcn_readlane(qe, src) - r.q0;
            r.k0 = __builtin_amdgcn_readlane(ks, src);
            r.nk = keys ? __builtin_amdgcn_readlane(ke, src) - r.k0 : 0;
            r.tile = __builtin_amdgcn_readlane(upto, src) - 1 - t;
            return r;
        }
        before = __builtin_amdgcn_readlane(upto, 63);
        qmax = __builtin_amdgcn_readlane(qe, 63);
        kmax = __builtin_amdgcn_readlane(ke, 63);
    }
    r.none = true;
    return r;
}

// Where a 16-byte element (key k of 16, slice s of 4) of a block is, in elements:
// the lane whose load brings it.  A wave loads a block, 1 KiB, at once, so that
// memory is read in pieces of 64 bytes (NHWC: four slices of a key) or 256 (sliced:
// 16 keys of a slice), and the exclusive ors spread what the matrix instructions'
// operands take at a time, 8 keys of a slice or 4 keys of 4 slices, over all banks.
template <bool NHWC>
__device__ __forceinline__ int at_of(int k, int s) { return NHWC ? k * 4 + (s ^ (k >> 1 & 3)) : s * 16 + (k ^ (s & 1) << 2); }
template <bool NHWC>
__device__ __forceinline__ void of_lane(int lane, int &k, int &s) {
    if (NHWC) {
        k = lane >> 2;
        s = (lane & 3) ^ (k >> 1 & 3);
    } else {
        s = lane >> 4;
        k = (lane & 15) ^ (s & 1) << 2;
    }
}

typedef short s4 __attribute__((ext_vector_type(4)));

// A column of V: 4 keys of a channel to each lane, out of 16 lanes' 4 keys x 16 channels
__device__ __forceinline__ s4 read_column(const h8 *base, int bytes) {
    return __builtin_amdgcn_ds_read_tr16_b64_v4i16(
        (__attribute__((address_space(3))) s4 *)((__attribute__((address_space(3))) char *)(size_t)(unsigned)(size_t)(
                                                     __attribute__((address_space(3))) const void *)base + bytes));
}

// Infinite and NaN values that a row sees.  A channel in which one of its keys has
// such a value is that (NaN of infinities of both signs), however small the key's
// weight: the products have NaN of weights that are zero in 16 bits, and so has a sum
// that was scaled by zero since.  Where a sum ended infinite or NaN, what there is of
// these values is added up by itself.
__device__ __forceinline__ bool ended_odd(const float *v) {
    float top = 0.0f;
#pragma unroll
    for (int i = 0; i < 8; i += 2)
        top = __builtin_elementwise_maximum(__builtin_elementwise_maximum(fabsf(v[i]), fabsf(v[i + 1])), top);
    return !(top < INFINITY);
}
__device__ __forceinline__ void add_odd(const float *x, float *odd) {
#pragma unroll
    for (int i = 0; i < 8; ++i) odd[i] += fabsf(x[i]) < INFINITY ? 0.0f : x[i];
}
__device__ __forceinline__ void take_odd(const float *odd, float *v) {
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = odd[i] != 0.0f ? odd[i] : v[i];
}

__device__ __forceinline__ h8 with_zeros_for_odd(h8 v, bool bf) {
    const uint16_t mask = bf ? 0x7f80 : 0x7c00;
    u16x8 b = bits8(v);
#pragma unroll
    for (int i = 0; i < 8; ++i) b[i] = (b[i] & mask) == mask ? 0 : b[i];
    return __builtin_bit_cast(h8, b);
}
__device__ __forceinline__ bool any_odd(h8 v, bool bf) {
    const uint16_t mask = bf ? 0x7f80 : 0x7c00;
    const u16x8 b = bits8(v);
    bool odd = false;
#pragma unroll
    for (int i = 0; i < 8; ++i) odd = odd || (b[i] & mask) == mask;
    return odd;
}

// A workgroup's head of keys, row tile and chunk: the head fastest, so that an XCD
// (every eighth workgroup) has few of them, whose keys then stay in its L2, and the
// long tiles of all heads, which come first, are spread over all XCDs (8 heads on one
// of keys, 3141 tokens of 96 channels: contiguous tiles to each XCD 62 us).
__device__ __forceinline__ void place(const AttentionGeom &geo, int kv_heads, int block, int &kvh, int &tile, int &chunk) {
    const int item = block / kv_heads;
    kvh = block - item * kv_heads;
    tile = item / geo.chunks;
    chunk = item - tile * geo.chunks;
}

// ND: the head's channels in steps of 32.  WR = 4: four waves of 32 rows share
// tiles of 64 keys; WR = 1: four waves have the same 32 rows and 32 keys each, by
// themselves.  Two stages of LDS: the next tile's loads are in flight while a tile
// is worked on.
template <typename E, int ND, int WR, bool NHWC>
__global__ __launch_bounds__(256, WR == 1 ? 1 : ND == 3 ? 3 : 2) void attention_kernel(AttentionParams p, AttentionGeom geo) {
    constexpr int BM = tile_rows(WR), NK = WR == 4 ? 2 : 1;          // blocks of 32 keys of a wave's tile
    constexpr int KEYS = 32 * NK, STEP = WR == 4 ? KEYS : 4 * KEYS;  // keys of a wave's tile, from one to the next
    constexpr int PART = NK * 2 * ND * 64, STAGE = 2 * PART;         // elements of K (or V), of both
    constexpr int OWN = WR == 4 ? 1 : 4;
    __shared__ h8 lds[2 * OWN * STAGE];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), half = lane >> 5;
    int kvh, number, chunk;
    place(geo, p.kv_heads, blockIdx.x, kvh, number, chunk);
    const Tile t = find_tile<BM>(p, number);
    if (t.none) return;
    const int rows = t.nq * p.group, first = t.tile * BM, r0 = first + (WR == 4 ? wave * 32 : 0);
    const int row = r0 + (lane & 31), rc = min(row, rows - 1);
    const int token = rc / p.group, head = kvh * p.group + rc - token * p.group;
    // keys that a row sees
    auto seen = [&](int r) {
        const int tok = min(r, rows - 1) / p.group;
        return p.causal ? min(max(tok + 1 + t.nk - t.nq, 0), t.nk) : t.nk;
    };
    const int from = chunk * geo.chunk;
    const int whole = seen(first + BM - 1), most = __builtin_amdgcn_readfirstlane(min(whole, geo.chunks > 1 ? from + geo.chunk : t.nk));
    if (chunk > 0 && from >= most) return;                           // (the first chunk writes rows that see nothing)
    const bool split = __builtin_amdgcn_readfirstlane(geo.chunks > 1 && whole > geo.chunk);
    // the fewest that a row of the tile sees, the most that one of the wave does
    const int least = __builtin_amdgcn_readfirstlane(seen(first)), mine = __builtin_amdgcn_readfirstlane(min(seen(r0 + 31), most));
    const int lim = seen(rc);
    const bool works = r0 < rows;

    h8 q[ND * 2];
#pragma unroll
    for (int s = 0; s < ND * 2; ++s) {
        const int sl = 2 * s + half;
        q[s] = sl < p.d8 ? p.q.x[(size_t)(head * p.d8 + sl) * p.q.s + (size_t)(t.q0 + token) * p.q.p] : zero_h8();
        if (p.scale < 0.0f) q[s] = -q[s];
    }
    const float c = fabsf(p.scale);
    f16v o[ND];
#pragma unroll
    for (int d = 0; d < ND; ++d) o[d] = f16v{};
    float m = -INFINITY, l = 0.0f;

    // this lane's element of the blocks that the wave loads; slices past the head's
    // last come from a block of zeros
    int lk, ls;
    of_lane<NHWC>(lane, lk, ls);
    const h8 *kp = p.k.x + (size_t)(kvh * p.d8 + ls) * p.k.s, *vp = p.v.x + (size_t)(kvh * p.d8 + ls) * p.v.s;
    constexpr int BLOCKS = WR == 4 ? 1 : 2, LOADS = BLOCKS * ND;     // blocks of 16 keys that a wave loads, loads of K (or V)
    // one of the 2 LOADS loads of a tile: K's blocks and slices, then V's
    auto issue = [&](int j0, int stage, int piece) {
        const bool values = piece >= LOADS;
        const int u = piece % LOADS / ND, g = piece % ND, b = WR == 4 ? wave : u;
        h8 *to = lds + (stage * OWN + (WR == 4 ? 0 : wave)) * STAGE + (values ? PART : 0);
        const TokenIn &x = values ? p.v : p.k;
        const h8 *at = (values ? vp : kp) + (size_t)(t.k0 + min(j0 + b * 16 + lk, t.nk - 1)) * x.p;
        load_lds16(g == ND - 1 && ls + 4 * g >= p.d8 ? p.zero : at + (size_t)(4 * g) * x.s, to + (b * ND + g) * 64);
    };
    auto issue_all = [&](int j0, int stage) {
#pragma unroll
        for (int i = 0; i < 2 * LOADS; ++i) issue(j0, stage, i);
    };
    // the lane's places in a stage, in elements (K: of even and odd steps of 16
    // channels) and bytes
    const int key = lane & 15, kblock = (lane >> 4 & 1) * ND * 64;
    const int ka[2] = {kblock + at_of<NHWC>(key, half), kblock + at_of<NHWC>(key, 2 + half)};
    const int va = at_of<NHWC>(4 * half + (key >> 2), (lane >> 4 & 1) * 2 + (key >> 1 & 1)) * 16 + (key & 1) * 8;
    constexpr int EIGHT = NHWC ? 512 : 128;                          // bytes from a key to the eighth after it

    // The next tile's loads are issued between the products: all at once they wait for
    // one another, 700 of a step's 3600 cycles (8192 causal tokens, heads of 128: 614 us,
    // now 593).  Heads of 96 channels, whose waves have 168 registers, have none to spare
    // for that (103 us against 47, the packed sequences above); waves by themselves
    // wait for their own loads either way.
    constexpr bool SPREAD = WR == 4 && ND != 3;
    auto scores = [&](auto load, int j0, int to, const h8 *kt, f16v (&s)[NK]) {
        auto read = [&](int k, int b) { return kt[ka[k & 1] + (b * 2 * ND + k / 2) * 64]; };
#pragma unroll
        for (int b = 0; b < NK; ++b) s[b] = f16v{};
        if constexpr (!decltype(load)::value) {
#pragma unroll
            for (int k = 0; k < ND * 2 - 1; ++k)
#pragma unroll
                for (int b = 0; b < NK; ++b) s[b] = mma32<E>(read(k, b), q[k], s[b]);
            // (16 channels of zeros are left out: heads of 80, the packed sequences above 46.5 -> 45.0 us)
            if (p.d8 > ND * 4 - 2) {
#pragma unroll
                for (int b = 0; b < NK; ++b) s[b] = mma32<E>(read(ND * 2 - 1, b), q[ND * 2 - 1], s[b]);
            }
        } else {
            h8 a[3][NK];                                                 // (read two steps ahead)
#pragma unroll
            for (int k = 0; k < 2; ++k)
#pragma unroll
                for (int b = 0; b < NK; ++b) a[k][b] = read(k, b);
#pragma unroll
            for (int k = 0; k < ND * 2; ++k) {
                if (k + 2 < ND * 2) {
#pragma unroll
                    for (int b = 0; b < NK; ++b) a[(k + 2) % 3][b] = read(k + 2, b);
                }
#pragma unroll
                for (int i = 0; i < LOADS / ND; ++i) issue(j0, to, k * (LOADS / ND) + i);
                __builtin_amdgcn_sched_barrier(0);
#pragma unroll
                for (int b = 0; b < NK; ++b) s[b] = mma32<E>(a[k % 3][b], q[k], s[b]);
                __builtin_amdgcn_sched_barrier(0);
            }
        }
    };
    // Hidden keys have no score; values that are infinite or NaN are taken out of the
    // tile (0 times them is NaN) and added to the rows that see them.
    auto hide = [&](int j0, h8 *vt, f16v (&s)[NK]) {
        bool odd = false;
        const int me = WR == 4 ? tid : lane, all = WR == 4 ? 256 : 64;
        for (int e = me; e < PART; e += all) odd = odd || any_odd(vt[e], E::bf);
        const bool found = WR == 4 ? __syncthreads_or(odd) : __any(odd);
        if (found) {
            for (int k = 0; k < KEYS; ++k)
#pragma unroll
                for (int d = 0; d < ND; ++d)
#pragma unroll
                    for (int g = 0; g < 4; ++g) {
                        const h8 v = vt[(k / 16 * ND + d) * 64 + at_of<NHWC>(k % 16, g)];
#pragma unroll
                        for (int i = 0; i < 4; ++i) {
                            const float x = half ? E::get(v, 4 + i) : E::get(v, i);
                            if (j0 + k < lim && !(fabsf(x) < INFINITY)) o[d][g * 4 + i] += x;
                        }
                    }
            if constexpr (WR == 4) __syncthreads();
            else __builtin_amdgcn_wave_barrier();
            asm volatile("" ::: "memory");
            for (int e = me; e < PART; e += all) vt[e] = with_zeros_for_odd(vt[e], E::bf);
            if constexpr (WR == 4) __syncthreads();
            else __builtin_amdgcn_wave_barrier();
            asm volatile("" ::: "memory");
        }
#pragma unroll
        for (int b = 0; b < NK; ++b)
#pragma unroll
            for (int i = 0; i < 16; ++i)
                if (j0 + b * 32 + i / 4 * 8 + half * 4 + i % 4 >= lim) s[b][i] = -INFINITY;
    };
    // The rows' maxima: the weights' base moves only when a score passes it by 2^kSlack.
    auto rebase = [&](const f16v (&s)[NK]) {
        float top = s[0][0];
#pragma unroll
        for (int b = 0; b < NK; ++b)
#pragma unroll
            for (int i = 0; i < 16; ++i) top = fmaxf(top, s[b][i]);
        top = larger_half(top);
        const bool move = fmaf(top, c, m == -INFINITY ? INFINITY : -m * c) > kSlack;
        if (__any(move)) {
            // (before the first weights there is nothing to scale but infinities)
            const float to = move ? top : m, keep = move && m != -INFINITY ? __builtin_amdgcn_exp2f((m - to) * c) : 1.0f;
            m = to;
            l *= keep;
#pragma unroll
            for (int d = 0; d < ND; ++d) o[d] *= keep;
        }
        return m == -INFINITY ? 0.0f : m * c - kLift<E>;
    };
    auto weights = [&](const f16v (&s)[NK], float base, h8 (&pr)[2 * NK]) {
        float sum = 0.0f;
#pragma unroll
        for (int k = 0; k < 2 * NK; ++k) {
            float w[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                w[i] = __builtin_amdgcn_exp2f(fmaf(s[k / 2][(k & 1) * 8 + i], c, -base));
                sum += w[i];
            }
            pr[k] = E::pack(w);
        }
        l += sum;
    };
    auto values = [&](const h8 *vt, const h8 (&pr)[2 * NK]) {
        auto read = [&](int i) {
            const int off = va + i * 1024;
            const s4 a = read_column(vt, off), b = read_column(vt, off + EIGHT);
            return __builtin_bit_cast(h8, __builtin_shufflevector(a, b, 0, 1, 2, 3, 4, 5, 6, 7));
        };
        constexpr int N = 2 * NK * ND;
        if constexpr (WR == 4 && ND < 4) {
            // (read ahead, which the compiler does not do by itself here: the packed
            // sequences above 44.7 -> 42.3 us; heads of 128 channels do not gain)
            constexpr int D = 2;                                         // (heads of 96 keep two registers in memory for it)
            h8 v[D + 1];
#pragma unroll
            for (int i = 0; i < D; ++i) v[i] = read(i);
#pragma unroll
            for (int i = 0; i < N; ++i) {
                if (i + D < N) v[(i + D) % (D + 1)] = read(i + D);
                __builtin_amdgcn_sched_barrier(0);
                o[i % ND] = mma32<E>(v[i % (D + 1)], pr[i / ND], o[i % ND]);
                __builtin_amdgcn_sched_barrier(0);
            }
        } else {
#pragma unroll
            for (int i = 0; i < N; ++i) o[i % ND] = mma32<E>(read(i), pr[i / ND], o[i % ND]);
        }
    };

    const int start = from + (WR == 4 ? 0 : wave * KEYS);
    int stage = 0;
    if (start < most) {
        issue_all(start, 0);
    }
    for (int j0 = start; j0 < most; j0 += STEP, stage ^= 1) {
        wait_vm_lds<0>();
        if constexpr (WR == 4) __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");                           // (no LDS access moves over the wait)
        const bool more = j0 + STEP < most;
        h8 *kt = lds + (stage * OWN + (WR == 4 ? 0 : wave)) * STAGE, *vt = kt + PART;
        f16v s[NK];
        const bool mute = !works || j0 >= mine;
        if (more && (mute || !SPREAD)) issue_all(j0 + STEP, stage ^ 1);
        if (!mute) {
            if (SPREAD && more) scores(std::true_type{}, j0 + STEP, stage ^ 1, kt, s);
            else scores(std::false_type{}, 0, 0, kt, s);
        }
        if (j0 + KEYS > least) hide(j0, vt, s);
        if (mute) continue;
        const float base = rebase(s);
        h8 pr[2 * NK];
        weights(s, base, pr);
        values(vt, pr);
    }
    l += __shfl_xor(l, 32, 64);
    const int d32 = ND * 32;
    const size_t slot = ((size_t)(kvh * geo.tiles + number) * geo.chunks + chunk) * BM;    // this chunk's rows among all partial ones
    if constexpr (WR == 4) {
        if (!works) return;
        float ended = 0.0f;
#pragma unroll
        for (int d = 0; d < ND; ++d)
#pragma unroll
            for (int i = 0; i < 16; i += 2)
                ended = __builtin_elementwise_maximum(__builtin_elementwise_maximum(fabsf(o[d][i]), fabsf(o[d][i + 1])), ended);
        if (__any(!(ended < INFINITY) && l == l)) {                  // (the scores' NaN are the whole row's)
#pragma unroll
            for (int d = 0; d < ND; ++d) {
                f16v odd = f16v{};
                for (int j = from; j < most; ++j)
#pragma unroll
                    for (int g = 0; g < 4; ++g) {
                        if (d * 4 + g >= p.d8) continue;
                        const h8 v = p.v.x[(size_t)(kvh * p.d8 + d * 4 + g) * p.v.s + (size_t)(t.k0 + j) * p.v.p];
#pragma unroll
                        for (int i = 0; i < 4; ++i) {
                            const float x = half ? E::get(v, 4 + i) : E::get(v, i);
                            if (j < lim && !(fabsf(x) < INFINITY)) odd[g * 4 + i] += x;
                        }
                    }
#pragma unroll
                for (int i = 0; i < 16; ++i) o[d][i] = odd[i] != 0.0f ? odd[i] : o[d][i];
            }
        }
        if (split) {
            if (row < rows) {
                float *part = p.part + (slot + row - first) * (d32 + 2);
#pragma unroll
                for (int d = 0; d < ND; ++d)
#pragma unroll
                    for (int g = 0; g < 4; ++g)
#pragma unroll
                        for (int i = 0; i < 4; i += 2)
                            *(float2 *)(part + d * 32 + g * 8 + half * 4 + i) = float2{o[d][g * 4 + i], o[d][g * 4 + i + 1]};
                if (half == 0) *(float2 *)(part + d32) = float2{m, l};
            }
            return;
        }
        const float inv = l == 0.0f ? 1.0f : 1.0f / l;               // (no weights: o is zero, infinite or NaN)
        // a lane has 4 of a slice's 8 channels, lane ^ 32 the others: of two slices
        // each completes one
#pragma unroll
        for (int d = 0; d < ND; ++d)
#pragma unroll
            for (int g = 0; g < 4; g += 2) {
                float v[8];
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const float a = pinned(o[d][g * 4 + i] * inv), b = pinned(o[d][g * 4 + 4 + i] * inv);
                    const float other = __shfl_xor(half ? a : b, 32, 64);
                    v[i] = half ? other : a;
                    v[4 + i] = half ? b : other;
                }
                const int sl = d * 4 + g + half;
                if (row < rows && sl < p.d8) store8<E>(p.y, head * p.d8 + sl, t.q0 + token, E::pack(v));
            }
    } else {
        // the four waves' parts of the rows, in turn in the order of the waves
        constexpr int LINE = ND * 32 + 4;
        float *sums = (float *)lds;                                  // [wave][row][LINE]
        __shared__ float2 ml[4][32];
        __syncthreads();                                             // (all have read their last tile)
        if (half == 0) ml[wave][lane] = float2{m, l};
        float *mine_ = sums + (wave * 32 + (lane & 31)) * LINE;
#pragma unroll
        for (int d = 0; d < ND; ++d)
#pragma unroll
            for (int g = 0; g < 4; ++g)
                *(f4 *)(mine_ + d * 32 + g * 8 + half * 4) = f4{o[d][g * 4], o[d][g * 4 + 1], o[d][g * 4 + 2], o[d][g * 4 + 3]};
        __syncthreads();
        for (int e = tid; e < 32 * ND * 4; e += 256) {
            const int r = e & 31, sl = e >> 5;
            if (first + r >= rows || sl >= p.d8) continue;
            float top = -INFINITY, total = 0.0f, v[8] = {};
#pragma unroll
            for (int w = 0; w < 4; ++w) top = fmaxf(top, ml[w][r].x);
#pragma unroll
            for (int w = 0; w < 4; ++w) {
                const float f = ml[w][r].x == -INFINITY ? 0.0f : __builtin_amdgcn_exp2f((ml[w][r].x - top) * c);
                total = fmaf(ml[w][r].y, f, total);
                const f4 *from_ = (const f4 *)(sums + (w * 32 + r) * LINE + sl * 8);
                const f4 lo = from_[0], hi = from_[1];
#pragma unroll
                for (int i = 0; i < 8; ++i) v[i] = fmaf(i < 4 ? lo[i & 3] : hi[i & 3], f, v[i]);
            }
            if (ended_odd(v) && total == total) {
                float odd[8] = {};
                const int end = min(seen(first + r), most);
                for (int j = from; j < end; ++j) {
                    const h8 x = p.v.x[(size_t)(kvh * p.d8 + sl) * p.v.s + (size_t)(t.k0 + j) * p.v.p];
                    float w[8];
#pragma unroll
                    for (int i = 0; i < 8; ++i) w[i] = E::get(x, i);
                    add_odd(w, odd);
                }
                take_odd(odd, v);
            }
            if (split) {
                float *part = p.part + (slot + r) * (d32 + 2);
#pragma unroll
                for (int i = 0; i < 8; i += 2) *(float2 *)(part + sl * 8 + i) = float2{v[i], v[i + 1]};
                if (sl == 0) *(float2 *)(part + d32) = float2{top, total};
            } else {
                const float inv = total == 0.0f ? 1.0f : 1.0f / total;
#pragma unroll
                for (int i = 0; i < 8; ++i) v[i] = pinned(v[i] * inv);
                const int tok = (first + r) / p.group, hd = kvh * p.group + first + r - tok * p.group;
                store8<E>(p.y, hd * p.d8 + sl, t.q0 + tok, E::pack(v));
            }
        }
    }
}

// Joins the chunks of the rows that have several, in a launch of its own (by the
// workgroup that is done last, as other kernels here do: its stores past the L2 and
// its acquire take longer than the launch, 13 packed sequences 62 us against 41, one
// query on 32768 keys 37 either way, before this kernel took 4.5 us there).  A thread has 8 channels of every
// CG-th chunk of a row, then what CG threads found is joined in order.
template <typename E, int BM, int CG>
__global__ __launch_bounds__(256) void attention_join_kernel(AttentionParams p, AttentionGeom geo, int d32) {
    constexpr int ROWS = 16 / CG;                                    // of a workgroup
    __shared__ float found[CG > 1 ? CG : 1][16][8];
    __shared__ float2 ml[CG > 1 ? CG : 1][16];
    const int pair = blockIdx.x / (BM / ROWS), kvh = pair / geo.tiles;
    const int sl = threadIdx.x & 15, g = CG > 1 ? threadIdx.x >> 4 : 0, r = (blockIdx.x - pair * (BM / ROWS)) * ROWS + (CG > 1 ? 0 : threadIdx.x >> 4);
    const Tile t = find_tile<BM>(p, pair - kvh * geo.tiles);
    const int rows = t.nq * p.group, first = t.tile * BM, row = first + r;
    if (t.none || first >= rows) return;
    const int last = min(first + BM - 1, rows - 1) / p.group;
    const int most = p.causal ? min(max(last + 1 + t.nk - t.nq, 0), t.nk) : t.nk;
    const int n = min((most + geo.chunk - 1) / geo.chunk, geo.chunks);
    if (n < 2) return;
    const float c = fabsf(p.scale);
    const float *part = p.part + ((size_t)pair * geo.chunks * BM + r) * (d32 + 2);
    const size_t step = (size_t)BM * (d32 + 2);
    float top = -INFINITY, total = 0.0f, v[8] = {};
    auto add = [&](float m, float l, const float *x) {
        const float to = fmaxf(top, m), keep = top == -INFINITY ? 0.0f : __builtin_amdgcn_exp2f((top - to) * c);
        const float f = m == -INFINITY ? 0.0f : __builtin_amdgcn_exp2f((m - to) * c);
        top = to;
        total = fmaf(total, keep, l * f);
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = fmaf(x[i], f, v[i] * keep);
    };
    if (sl < p.d8 && row < rows) {
        float x[8];
        auto read = [&](int k) {
            const float *at = part + k * step + sl * 8;
#pragma unroll
            for (int i = 0; i < 8; i += 2) *(float2 *)(x + i) = *(const float2 *)(at + i);
        };
        for (int k = g; k < n; k += CG) {
            const float2 w = *(const float2 *)(part + k * step + d32);
            read(k);
            add(w.x, w.y, x);
        }
        if (ended_odd(v)) {
            float odd[8] = {};
            for (int k = g; k < n; k += CG) {
                read(k);
                add_odd(x, odd);
            }
            take_odd(odd, v);
        }
    }
    if constexpr (CG > 1) {
#pragma unroll
        for (int i = 0; i < 8; ++i) found[g][sl][i] = v[i];
        ml[g][sl] = float2{top, total};
        __syncthreads();
        if (g > 0) return;
        for (int k = 1; k < min(n, CG); ++k) add(ml[k][sl].x, ml[k][sl].y, found[k][sl]);
        if (ended_odd(v)) {
            float odd[8] = {};
            for (int k = 0; k < min(n, CG); ++k) add_odd(found[k][sl], odd);
            take_odd(odd, v);
        }
    }
    if (row >= rows || sl >= p.d8) return;
    const float inv = total == 0.0f ? 1.0f : 1.0f / total;
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = pinned(v[i] * inv);
    const int tok = row / p.group, hd = kvh * p.group + row - tok * p.group;
    store8<E>(p.y, hd * p.d8 + sl, t.q0 + tok, E::pack(v));
}

template <typename E, int ND, int WR>
void launch_attention_w(const AttentionParams &p, const AttentionGeom &g, hipStream_t st) {
    const dim3 grid((unsigned)g.tiles * p.kv_heads * g.chunks);
    // (a timed run stamps the first kernel's start and the last one's end)
    LaunchEvents &ev = launch_events();
    const LaunchEvents saved = ev;
    if (g.chunks > 1) ev.stop = nullptr;
    if (p.k.s == 1 && p.v.s == 1) launch(attention_kernel<E, ND, WR, true>, grid, dim3(256), 0, st, p, g);
    else launch(attention_kernel<E, ND, WR, false>, grid, dim3(256), 0, st, p, g);
    ev = saved;
    if (g.chunks == 1) return;
    constexpr int CG = WR == 1 ? 16 : 1;                             // (many chunks of few rows, few of many)
    const dim3 join((unsigned)g.tiles * p.kv_heads * (tile_rows(WR) * CG / 16));
    ev.start = nullptr;
    launch(attention_join_kernel<E, tile_rows(WR), CG>, join, dim3(256), 0, st, p, g, ND * 32);
    ev = saved;
}

template <typename E, int ND>
void launch_attention_n(const AttentionParams &p, const AttentionGeom &g, hipStream_t st) {
    if (g.wr == 4) launch_attention_w<E, ND, 4>(p, g, st);
    else launch_attention_w<E, ND, 1>(p, g, st);
}

template <typename E>
hipError_t launch_attention_t(const AttentionParams &p, const AttentionGeom &g, hipStream_t st) {
    switch ((p.d8 + 3) / 4) {
        case 1: launch_attention_n<E, 1>(p, g, st); break;
        case 2: launch_attention_n<E, 2>(p, g, st); break;
        case 3: launch_attention_n<E, 3>(p, g, st); break;
        case 4: launch_attention_n<E, 4>(p, g, st); break;
        default: return hipErrorInvalidValue;
    }
    return hipGetLastError();
}

}  // namespace

AttentionGeom attention_geom(int q_tokens, int k_tokens, int n, int nseq, int group, int kv_heads, int d8) {
    AttentionGeom g{};
    const long rows = (long)q_tokens * group, sequences = nseq ? nseq : n;
    // few rows to a sequence: the waves share the keys out instead
    g.wr = rows <= 32 * sequences ? 1 : 4;
    const int bm = tile_rows(g.wr);
    g.tiles = (int)(nseq ? rows / bm + nseq + 2 : n * ((rows / n + bm - 1) / bm));
    // The keys are split where workgroups are few: below what the card holds of tiles
    // that waves share (two to a compute unit) or of the others (one).  Packed sequences, whose lengths the host does not know, may have one that
    // is much longer than the others and ends alone, so they are split further, unless
    // that would be into halves (the joining launch costs 3 us where nothing is split).
    const long keys = nseq ? k_tokens : k_tokens / n, items = (long)g.tiles * kv_heads;
    const long want = g.wr == 1 ? 256 : nseq ? 2048 : 512;
    const int step = g.wr == 4 ? kBN : 4 * kPrivate;
    long chunks = items < want ? want / items : 1;
    if (nseq && g.wr == 4 && chunks < 3) chunks = 1;
    chunks = std::min(chunks, (keys + 4 * step - 1) / (4 * step));
    g.chunk = (int)((keys + chunks * step - 1) / (chunks * step)) * step;
    g.chunks = (int)((keys + g.chunk - 1) / g.chunk);
    if (g.chunks > 1) g.part_bytes = (size_t)items * g.chunks * bm * ((d8 + 3) / 4 * 32 + 2) * 4;
    return g;
}

hipError_t launch_attention(const AttentionParams &p, const AttentionGeom &g, hipStream_t st) {
    return p.bf16 ? launch_attention_t<BF16>(p, g, st) : launch_attention_t<F16>(p, g, st);
}

}  // namespace kern
}  // namespace mgi
