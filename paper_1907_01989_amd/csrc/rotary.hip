// Rotary positions with several axes.
//
//   (a, b) -> (a cos t - b sin t, a sin t + b cos t),  t = position * frequency
//
// Angles are counted in turns: the frequency is a fraction of a turn in 64-bit
// fixed point, so that the product with a 32-bit position modulo 2^64 is the
// angle's fraction of a turn, without the loss that a float product has at far
// positions; its upper 32 bits go to the hardware's sine and cosine, which take
// turns.  Large tensors are bound by memory, read and written once: 29952 pixels x 32
// heads of 128, 491 MB in 102 us, 4.8 TB/s.  Smaller ones wait for the angles before
// their loads (12544 pixels x 12 heads of 80, 48 MB: 15 us apart, 11 adjacent).
#include "tokens.h"

namespace mgi {
namespace kern {

namespace {

// the pixel's positions along the axes
struct Place {
    const int *pos;
    int at[3];
    __device__ __forceinline__ Place(const RotaryParams &p, int m) {
        pos = p.pos ? p.pos + (size_t)m * p.axes : nullptr;
        if (pos) return;
        int row;
        divmod_fast(m, p.W, p.inv_w, row, at[2]);
        divmod_fast(row, p.H, p.inv_h, at[0], at[1]);
    }
    __device__ __forceinline__ int operator[](int axis) const {
        return pos ? pos[axis] : axis == 0 ? at[0] : axis == 1 ? at[1] : at[2];
    }
};

// sine and cosine of position * frequency
__device__ __forceinline__ void turn(int position, uint64_t freq, float &sn, float &cs) {
    const uint32_t u = (uint32_t)position, lo = (uint32_t)freq, hi = (uint32_t)(freq >> 32);
    const uint32_t f = __umulhi(u, lo) + u * hi - (position < 0 ? lo : 0u);
    const float t = (float)(int)f * 0x1p-32f;
    sn = __builtin_amdgcn_sinf(t);
    cs = __builtin_amdgcn_cosf(t);
}

// A thread has one unit of a head's channels: 8 pairs in slices `pairs / 8`
// apart (apart), 4 adjacent pairs of one slice, or a slice that is copied.  It
// computes its angles once and walks the heads with them.  Lanes: 8 pixels x 8
// units.
template <typename E, bool ADJ>
__global__ __launch_bounds__(256) void rotary_kernel(RotaryParams p, int units, int per) {
    const int m = blockIdx.x * 8 + (threadIdx.x & 7), n = threadIdx.x >> 3;
    const int lanes = 32 / units, u = n % units;          // heads side by side
    const int turned = ADJ ? p.pairs / 4 : p.pairs / 8;   // units that are rotated
    if (m >= p.M || n >= lanes * units) return;
    const Place place(p, m);
    constexpr int NP = ADJ ? 4 : 8;
    float sn[NP], cs[NP];
    const bool rot = u < turned;
    if (rot) {
#pragma unroll
        for (int i = 0; i < NP; ++i) turn(place[p.axis[u * NP + i]], p.freq[u * NP + i], sn[i], cs[i]);
    }
    const int a = ADJ || rot ? u : u + turned, b = a + turned;
    const int end = min(p.heads, (int)(blockIdx.y + 1) * per);
    const h8 *xa = p.x.x + (size_t)a * p.x.s + (size_t)m * p.x.p, *xb = p.x.x + (size_t)b * p.x.s + (size_t)m * p.x.p;
    const bool two = !ADJ && rot;
    // four heads' loads in flight together (29952 x 32 x 128: 110 us by one)
    for (int h0 = blockIdx.y * per + n / units; h0 < end; h0 += 4 * lanes) {
        h8 x[4], y[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const size_t at = (size_t)min(h0 + i * lanes, end - 1) * p.d8 * p.x.s;
            x[i] = xa[at];
            if (two) y[i] = xb[at];
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int h = h0 + i * lanes, s = h * p.d8;
            if (h >= end) break;
            if (!rot) {
                store8<E>(p.y, s + a, m, x[i]);
            } else if constexpr (ADJ) {
                float v[8];
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    const float c = E::get(x[i], 2 * k), d = E::get(x[i], 2 * k + 1);
                    v[2 * k] = pinned(c * cs[k] - d * sn[k]);
                    v[2 * k + 1] = pinned(c * sn[k] + d * cs[k]);
                }
                store8<E>(p.y, s + a, m, E::pack(v));
            } else {
                float v[8], w[8];
#pragma unroll
                for (int k = 0; k < 8; ++k) {
                    const float c = E::get(x[i], k), d = E::get(y[i], k);
                    v[k] = pinned(c * cs[k] - d * sn[k]);
                    w[k] = pinned(c * sn[k] + d * cs[k]);
                }
                store8<E>(p.y, s + a, m, E::pack(v));
                store8<E>(p.y, s + b, m, E::pack(w));
            }
        }
    }
}

// Pairs that do not fill slices: a thread makes the 8 channels of a slice one by one.
template <typename E>
__global__ __launch_bounds__(256) void rotary_any_kernel(RotaryParams p) {
    int m, s;
    if (!plane_place(p.M, p.heads * p.d8, m, s)) return;
    const Place place(p, m);
    const int head = s / p.d8 * p.d8, c0 = (s - head) * 8;
    const h8 x = p.x.x[(size_t)s * p.x.s + (size_t)m * p.x.p];
    float v[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const int c = c0 + i;
        v[i] = E::get(x, i);
        if (c >= 2 * p.pairs) continue;
        const bool first = p.adjacent ? c % 2 == 0 : c < p.pairs;
        const int pair = p.adjacent ? c / 2 : first ? c : c - p.pairs;
        const int o = p.adjacent ? c ^ 1 : first ? c + p.pairs : c - p.pairs;
        const h8 *at = p.x.x + (size_t)(head + o / 8) * p.x.s + (size_t)m * p.x.p;
        h8 other = zero_h8();
        other[0] = ((const _Float16 *)at)[o % 8];
        float sn, cs;
        turn(place[p.axis[pair]], p.freq[pair], sn, cs);
        v[i] = pinned(first ? v[i] * cs - E::get(other, 0) * sn : E::get(other, 0) * sn + v[i] * cs);
    }
    store8<E>(p.y, s, m, E::pack(v));
}

template <typename E>
hipError_t launch_rotary_t(const RotaryParams &p, hipStream_t st) {
    const bool whole = p.pairs % (p.adjacent ? 4 : 8) == 0;
    const int units = p.adjacent ? p.d8 : p.d8 - p.pairs / 8;
    if (!whole || units > 32 || units <= 0) {
        launch(rotary_any_kernel<E>, dim3(plane_blocks(p.M, p.heads * p.d8)), dim3(256), 0, st, p);
        return hipGetLastError();
    }
    const unsigned blocks = ((unsigned)p.M + 7) / 8;
    // heads to a workgroup: all, or fewer where that leaves compute units idle
    const int lanes = 32 / units;
    int parts = 1;
    while (blocks * parts < 1024 && parts < 64 && (p.heads + parts - 1) / parts > lanes) parts *= 2;
    const int per = ((p.heads + parts - 1) / parts + lanes - 1) / lanes * lanes;
    const dim3 grid(blocks, (p.heads + per - 1) / per);
    if (p.adjacent) launch(rotary_kernel<E, true>, grid, dim3(256), 0, st, p, units, per);
    else launch(rotary_kernel<E, false>, grid, dim3(256), 0, st, p, units, per);
    return hipGetLastError();
}

}  // namespace

hipError_t launch_rotary(const RotaryParams &p, hipStream_t st) {
    if (p.M <= 0) return hipSuccess;
    return p.bf16 ? launch_rotary_t<BF16>(p, st) : launch_rotary_t<F16>(p, st);
}

}  // namespace kern
}  // namespace mgi
