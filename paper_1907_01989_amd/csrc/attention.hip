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
// sum over keys averages), its sum is taken before.
#include "tokens.h"

namespace mgi {
namespace kern {

namespace {

typedef float f16v __attribute__((ext_vector_type(16)));

constexpr int kBM = 128, kBN = 64;   // rows and keys of a tile

template <typename E>
__device__ __forceinline__ f16v mma32(h8 a, h8 b, f16v c) {
    if constexpr (E::bf)
        return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bh8, a), __builtin_bit_cast(bh8, b), c, 0, 0, 0);
    else
        return __builtin_amdgcn_mfma_f32_32x32x16_f16(a, b, c, 0, 0, 0);
}

// A tile of query rows: the sequence's queries and keys, and the tile's number
// among the sequence's.
struct Tile {
    int q0, nq, k0, nk, tile;
    bool none;
};

// Finds tile `t` among the tiles of all sequences.  Bounds are read up to the
// token count and not below their predecessors.  Two more sequences without
// keys take the queries before the first bound and behind the last.
__device__ __forceinline__ Tile find_tile(const AttentionParams &p, int t) {
    Tile r;
    r.none = false;
    if (!p.bq) {
        const int per = (p.tq * p.group + kBM - 1) / kBM, image = t / per;
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
        const int i = base + lane;
        int qe = i <= p.nseq ? min(max(p.bq[min(i, p.nseq)], 0), p.tq) : p.tq;
        int ke = i <= p.nseq ? min(max((p.bk ? p.bk : p.bq)[min(i, p.nseq)], 0), p.tk) : p.tk;
#pragma unroll
        for (int d = 1; d < 64; d *= 2) {
            const int a = __shfl_up(qe, d, 64), b = __shfl_up(ke, d, 64);
            if (lane >= d) {
                qe = max(qe, a);
                ke = max(ke, b);
            }
        }
        qe = max(qe, qmax);
        ke = max(ke, kmax);
        int qs = __shfl_up(qe, 1, 64), ks = __shfl_up(ke, 1, 64);
        if (lane == 0) {
            qs = qmax;
            ks = kmax;
        }
        const int n = i < p.nseq + 2 ? ((qe - qs) * p.group + kBM - 1) / kBM : 0;
        int upto = n;
#pragma unroll
        for (int d = 1; d < 64; d *= 2) {
            const int a = __shfl_up(upto, d, 64);
            if (lane >= d) upto += a;
        }
        const uint64_t has = __ballot(before + upto > t);
        if (has) {
            const int src = __builtin_ctzll(has);
            const bool keys = base + src != 0 && base + src != p.nseq + 1;
            r.q0 = __shfl(qs, src, 64);
            r.nq = __shfl(qe, src, 64) - r.q0;
            r.k0 = __shfl(ks, src, 64);
            r.nk = keys ? __shfl(ke, src, 64) - r.k0 : 0;
            r.tile = before + __shfl(upto, src, 64) - 1 - t;
            return r;
        }
        before += __shfl(upto, 63, 64);
        qmax = __shfl(qe, 63, 64);
        kmax = __shfl(ke, 63, 64);
    }
    r.none = true;
    return r;
}

__device__ __forceinline__ bool finite16(uint16_t v, bool bf) { return bf ? (v & 0x7f80) != 0x7f80 : (v & 0x7c00) != 0x7c00; }

// ND: the head's channels in steps of 32
template <typename E, int ND>
__global__ __launch_bounds__(256) void attention_kernel(AttentionParams p, int tiles) {
    __shared__ h8 kt[ND * 4][kBN], vt[ND * 4][kBN];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), half = lane >> 5;
    const int kvh = blockIdx.x / tiles;
    const Tile t = find_tile(p, blockIdx.x - kvh * tiles);
    if (t.none) return;
    const int rows = t.nq * p.group, r0 = t.tile * kBM + wave * 32, row = r0 + (lane & 31), rc = min(row, rows - 1);
    const int token = rc / p.group, head = kvh * p.group + rc - token * p.group;
    // keys that a row sees, and the least and the most of the tile's rows
    auto seen = [&](int r) {
        const int tok = min(r, rows - 1) / p.group;
        return p.causal ? min(max(tok + 1 + t.nk - t.nq, 0), t.nk) : t.nk;
    };
    const int lim = seen(rc), least = seen(t.tile * kBM), most = seen(t.tile * kBM + kBM - 1);
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
    const h8 *kp = p.k.x + (size_t)kvh * p.d8 * p.k.s, *vp = p.v.x + (size_t)kvh * p.d8 * p.v.s;
    for (int j0 = 0; j0 < most; j0 += kBN) {
        for (int e = tid; e < (ND + 1) / 2 * 8 * kBN; e += 256) {
            const int key = (e & 7) | (e >> 6) % 8 << 3, sl = (e >> 3 & 7) | e >> 9 << 3;
            const size_t j = (size_t)(t.k0 + min(j0 + key, t.nk - 1));
            if (sl >= ND * 4) continue;
            kt[sl][key] = sl < p.d8 ? kp[(size_t)sl * p.k.s + j * p.k.p] : zero_h8();
            vt[sl][key] = sl < p.d8 ? vp[(size_t)sl * p.v.s + j * p.v.p] : zero_h8();
        }
        __syncthreads();
        f16v s[2];
        s[0] = s[1] = f16v{};
#pragma unroll
        for (int k = 0; k < ND * 2; ++k)
#pragma unroll
            for (int b = 0; b < 2; ++b) s[b] = mma32<E>(kt[2 * k + half][b * 32 + (lane & 31)], q[k], s[b]);
        const bool masked = j0 + kBN > least;
        if (masked) {
            // hidden keys: no score, and values that are infinite or NaN are
            // taken out of the tile (0 times them is NaN) and added to the rows
            // that see them
            bool odd = false;
            for (int e = tid; e < ND * 4 * kBN; e += 256) {
                const h8 v = vt[e / kBN][e % kBN];
#pragma unroll
                for (int i = 0; i < 8; ++i) odd = odd || !finite16(bits8(v)[i], E::bf);
            }
            if (__syncthreads_or(odd)) {
                for (int key = 0; key < kBN; ++key)
#pragma unroll
                    for (int d = 0; d < ND; ++d)
#pragma unroll
                        for (int i = 0; i < 16; ++i) {
                            const float v = E::get(vt[d * 4 + i / 4][key], half * 4 + i % 4);
                            if (j0 + key < lim && !(fabsf(v) < INFINITY)) o[d][i] += v;
                        }
                __syncthreads();
                for (int e = tid; e < ND * 4 * kBN; e += 256) {
                    h8 v = vt[e / kBN][e % kBN];
#pragma unroll
                    for (int i = 0; i < 8; ++i)
                        if (!finite16(bits8(v)[i], E::bf)) v[i] = (_Float16)0.0f;
                    vt[e / kBN][e % kBN] = v;
                }
                __syncthreads();
            }
#pragma unroll
            for (int b = 0; b < 2; ++b)
#pragma unroll
                for (int i = 0; i < 16; ++i)
                    if (j0 + b * 32 + i / 4 * 8 + half * 4 + i % 4 >= lim) s[b][i] = -INFINITY;
        }
        float top = m;
#pragma unroll
        for (int b = 0; b < 2; ++b)
#pragma unroll
            for (int i = 0; i < 16; ++i) top = fmaxf(top, s[b][i]);
        top = fmaxf(top, __shfl_xor(top, 32, 64));
        const float base = top == -INFINITY ? 0.0f : top * c;
        const float keep = __builtin_amdgcn_exp2f(fmaf(m, c, -base));
        m = top;
        float sum = 0.0f;
        h8 pr[4];
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            float w[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                w[i] = __builtin_amdgcn_exp2f(fmaf(s[k / 2][(k & 1) * 8 + i], c, -base));
                sum += w[i];
            }
            pr[k] = E::pack(w);
        }
        l = fmaf(l, keep, sum);
#pragma unroll
        for (int d = 0; d < ND; ++d) {
            o[d] *= keep;
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                h8 v;
#pragma unroll
                for (int i = 0; i < 8; ++i)
                    v[i] = vt[d * 4 + (lane & 31) / 8][k * 16 + i / 4 * 8 + half * 4 + i % 4][lane & 7];
                o[d] = mma32<E>(v, pr[k], o[d]);
            }
        }
        __syncthreads();
    }
    l += __shfl_xor(l, 32, 64);
    const float inv = l == 0.0f ? 0.0f : 1.0f / l;
    // a lane has 4 of a slice's 8 channels, lane ^ 32 the others: of two slices
    // each completes one
#pragma unroll
    for (int d = 0; d < ND; ++d)
#pragma unroll
        for (int g = 0; g < 4; g += 2) {
            float v[8];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const float a = o[d][g * 4 + i] * inv, b = o[d][g * 4 + 4 + i] * inv;
                const float other = __shfl_xor(half ? a : b, 32, 64);
                v[i] = half ? other : a;
                v[4 + i] = half ? b : other;
            }
            const int sl = d * 4 + g + half;
            if (row < rows && sl < p.d8) store8<E>(p.y, head * p.d8 + sl, t.q0 + token, E::pack(v));
        }
}

template <typename E>
hipError_t launch_attention_t(const AttentionParams &p, const AttentionGeom &g, hipStream_t st) {
    const dim3 grid((unsigned)g.tiles * p.kv_heads);
    switch ((p.d8 + 3) / 4) {
        case 1: launch(attention_kernel<E, 1>, grid, dim3(256), 0, st, p, g.tiles); break;
        case 2: launch(attention_kernel<E, 2>, grid, dim3(256), 0, st, p, g.tiles); break;
        case 3: launch(attention_kernel<E, 3>, grid, dim3(256), 0, st, p, g.tiles); break;
        case 4: launch(attention_kernel<E, 4>, grid, dim3(256), 0, st, p, g.tiles); break;
        default: return hipErrorInvalidValue;
    }
    return hipGetLastError();
}

}  // namespace

AttentionGeom attention_geom(int q_tokens, int k_tokens, int n, int nseq, int group, int kv_heads, int d8) {
    AttentionGeom g{};
    const long rows = (long)q_tokens * group;
    g.tiles = (int)(nseq ? rows / kBM + nseq + 2 : (long)n * ((rows / n + kBM - 1) / kBM));
    g.chunks = 1;
    g.wr = 4;
    return g;
}

hipError_t launch_attention(const AttentionParams &p, const AttentionGeom &g, hipStream_t st) {
    return p.bf16 ? launch_attention_t<BF16>(p, g, st) : launch_attention_t<F16>(p, g, st);
}

}  // namespace kern
}  // namespace mgi
