// Questions about the channels of each pixel: the k largest, the logarithm of
// the softmax at given channels, the softmax's entropy.
//
// With m the row's maximum, s = sum exp(x - m) and t = sum exp(x - m) (x - m):
//     log softmax(x)_i = (x_i - m) - log s,    entropy = log s - t / s.
// Both terms of the entropy are non-negative, so neither loses digits to the
// other.  Sums are fp32.
//
// One workgroup owns a row, or a segment of one, and holds it in registers, so
// the row is read once whatever is asked: a call about long rows is bound by their
// bytes (4096 x 32000 fp32 5.0 TB/s), one about many short ones by the workgroups'
// starts (513 x 513 x 21 244 us, of which the bytes take 5).
// Where rows are few or long they are split into segments; each leaves its
// (m, s, t) and its own k best, and the workgroup that arrives last joins them.
#include "device.h"

namespace mgi {
namespace kern {

namespace {

constexpr int kCap = 1024;            // candidates a workgroup ranks
constexpr float kLog2e = 1.44269504088896341f;
// Workgroups along x of a grid that has more than one along y: threads along one
// dimension have to stay below 2^32, which 2^26 rows of one wave each reach.
constexpr int kGridBits = 22;

// unsigned integers in the order of the values (-0 as +0)
__device__ __forceinline__ uint32_t order_of(float v) {
    const uint32_t u = __float_as_uint(v + 0.0f);
    return u ^ ((uint32_t)((int)u >> 31) | 0x80000000u);
}
__device__ __forceinline__ float value_of(uint32_t o) {
    return __uint_as_float(o & 0x80000000u ? o ^ 0x80000000u : ~o);
}
// ... and of values, then of descending columns: larger keys come first, and
// no two columns share one; 0 is below every key
__device__ __forceinline__ unsigned long long key_of(float v, int col) {
    return (unsigned long long)order_of(v) << 32 | (uint32_t)~col;
}

// Reductions over a wave by cross-lane moves of the vector unit (lanes 1, 2, 4
// and 8 below, then the last lane of the row and of the half below): lane 63
// has all.  A shuffle through the LDS costs some 100 cycles a step, this 12.
constexpr int kRowShr = 0x110, kRowBcast15 = 0x142, kRowBcast31 = 0x143;
template <int CTRL, int ROWS>
__device__ __forceinline__ int below(int v, int none) {
    return __builtin_amdgcn_update_dpp(none, v, CTRL, ROWS, 0xf, false);
}
template <typename T, typename F>
__device__ __forceinline__ T wave_scan(T v, T none, F join) {   // inclusive
    const int z = __builtin_bit_cast(int, none);
    auto in = [](T a) { return __builtin_bit_cast(int, a); };
    auto out = [](int a) { return __builtin_bit_cast(T, a); };
    v = join(v, out(below<kRowShr + 1, 0xf>(in(v), z)));
    v = join(v, out(below<kRowShr + 2, 0xf>(in(v), z)));
    v = join(v, out(below<kRowShr + 4, 0xf>(in(v), z)));
    v = join(v, out(below<kRowShr + 8, 0xf>(in(v), z)));
    v = join(v, out(below<kRowBcast15, 0xa>(in(v), z)));
    return join(v, out(below<kRowBcast31, 0xc>(in(v), z)));
}
template <typename T, typename F>
__device__ __forceinline__ T wave_all(T v, T none, F join) {
    return __builtin_bit_cast(T, __builtin_amdgcn_readlane(__builtin_bit_cast(int, wave_scan(v, none, join)), 63));
}
__device__ __forceinline__ float wave_max(float v) {
    return wave_all(v, -INFINITY, [](float a, float b) { return fmaxf(a, b); });
}
__device__ __forceinline__ float wave_sum(float v) {
    return wave_all(v, 0.0f, [](float a, float b) { return a + b; });
}

// The r-th largest different value of a wave, which at least r lanes reach, or
// `none`: r rounds of the maximum, those that hold it dropping out.  All lanes
// get the maximum: rotations within rows of 16, then rows and halves swapped.
template <typename T, typename F>
__device__ __forceinline__ T wave_rth(T v, T none, int r, F join) {
    T top = none;
#pragma unroll 1
    for (int i = 0; i < r; ++i) {
        int u = __builtin_bit_cast(int, v);
        auto max2 = [&](int a, int b) { return __builtin_bit_cast(int, join(__builtin_bit_cast(T, a), __builtin_bit_cast(T, b))); };
        u = max2(u, below<0x128, 0xf>(u, 0));   // (row_ror)
        u = max2(u, below<0x124, 0xf>(u, 0));
        u = max2(u, below<0x122, 0xf>(u, 0));
        u = max2(u, below<0x121, 0xf>(u, 0));
        auto rows = __builtin_amdgcn_permlane16_swap((unsigned)u, (unsigned)u, false, false);
        u = max2((int)rows[0], (int)rows[1]);
        auto halves = __builtin_amdgcn_permlane32_swap((unsigned)u, (unsigned)u, false, false);
        top = __builtin_bit_cast(T, max2((int)halves[0], (int)halves[1]));
        if (v == top) v = none;
    }
    return top;
}

// A bound of at most the r-th largest of a wave's keys (order_of) and within
// 2^-7 of it: the key's upper half, two bits at a time from counts of lanes.  As
// long as five rounds of wave_rth, whatever r.  (Where the values are far from
// zero beside their spread most of them pass it and push_exact is called: 512 x
// 32000, k = 50, about zero 19 us, about 1000 +- 1 238.)
__device__ __forceinline__ uint32_t wave_rth_near(uint32_t key, int r) {
    uint32_t top = 0;
#pragma unroll
    for (int b = 30; b >= 16; b -= 2) {
        int n = 0;
#pragma unroll
        for (uint32_t q = 1; q < 4; ++q) n += __popcll(__ballot(key >= (top | q << b))) >= r;
        top |= (uint32_t)n << b;
    }
    return top;
}

__device__ __forceinline__ int lanes_below(unsigned long long mask) {
    return (int)__builtin_amdgcn_mbcnt_hi((uint32_t)(mask >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)mask, 0));
}

// Room for a lane's n candidates behind the other lanes': the first slot, or -1
// for a wave without any.
__device__ __forceinline__ int take_slots(int *count, int n) {
    const int upto = wave_scan(n, 0, [](int a, int b) { return a + b; });
    const int all = __builtin_amdgcn_readlane(upto, 63);
    if (all == 0) return -1;
    int base = 0;
    if ((threadIdx.x & 63) == 0) base = atomicAdd(count, all);
    return __builtin_amdgcn_readfirstlane(base) + upto - n;
}

template <int W>
struct Shared {
    alignas(16) unsigned long long cand[kCap + kMaxTopK + 8];   // zeros behind the candidates
    unsigned long long best[kMaxTopK];
    int rank[W > 1 ? kCap + kMaxTopK : 1];     // (one wave counts in registers)
    float m[W], bound[W], s[W], t[W];
    uint32_t key_bound[W];
    int cnt[W];
    int n, last;
};

// A workgroup's values: element e of vector i of a thread is column at(i) + e
// of the row; vectors that would pass the segment's end are moved back to end
// there, and repeat columns that other threads (or none) own, which do not
// count.  Slots that hold no column hold -inf.
template <typename T, int NT, int PER>
struct Held {
    static constexpr int VEC = 16 / (int)sizeof(T), I = PER / VEC;
    float v[PER];
    int lo, hi;
    __device__ __forceinline__ int own(int i) const { return lo + (i * NT + (int)threadIdx.x) * VEC; }
    __device__ __forceinline__ int at(int i) const {
        const int j = own(i);
        return hi - lo >= VEC ? min(j, hi - VEC) : j;
    }
    __device__ __forceinline__ bool valid(int i, int e) const {
        const int c = at(i) + e;
        return c >= own(i) && c < hi;
    }
    __device__ __forceinline__ void load(const T *x, int lo_, int hi_) {
        typedef T tv __attribute__((ext_vector_type(VEC)));
        typedef tv tvu __attribute__((aligned(sizeof(T))));   // (rows start anywhere)
        lo = lo_;
        hi = hi_;
        if (hi - lo < VEC) {
#pragma unroll
            for (int q = 0; q < PER; ++q) v[q] = (float)x[min(own(q / VEC) + q % VEC, hi - 1)];
        } else {
            tv b[I];
#pragma unroll
            for (int i = 0; i < I; ++i) b[i] = *(const tvu *)(x + at(i));
#pragma unroll
            for (int q = 0; q < PER; ++q) v[q] = (float)b[q / VEC][q % VEC];
        }
#pragma unroll
        for (int i = 0; i < I; ++i)
            if (lo + (i + 1) * NT * VEC > hi) {
#pragma unroll
                for (int e = 0; e < VEC; ++e)
                    if (!valid(i, e)) v[i * VEC + e] = -INFINITY;
            }
    }
};

// Adds the values of at least `th` to the candidates.  Of many a lane marks its
// own and then takes them one after the other, reading them again from memory
// (the cache): few lanes have more than two or three, but among a wave's lanes
// nearly every register has one.
template <int W, typename T, typename H>
__device__ __forceinline__ void push(Shared<W> &sh, const H &h, const T *x, float th) {
    constexpr int PER = H::I * H::VEC;
    uint32_t mark[(PER + 31) / 32] = {};
#pragma unroll
    for (int q = 0; q < PER; ++q) mark[q / 32] |= h.v[q] >= th ? 1u << q % 32 : 0u;
    int n = 0;
#pragma unroll
    for (uint32_t m : mark) n += __popc(m);
    int slot = take_slots(&sh.n, n);
    if (slot < 0) return;
    if constexpr (PER <= 8) {
#pragma unroll
        for (int q = 0; q < PER; ++q)
            if (mark[0] >> q & 1) {
                if (slot < kCap) sh.cand[slot] = key_of(h.v[q], h.at(q / H::VEC) + q % H::VEC);
                ++slot;
            }
        return;
    }
#pragma unroll
    for (int w = 0; w < (PER + 31) / 32; ++w)
#pragma unroll 1
        for (uint32_t m = mark[w]; m; m &= m - 1) {
            const int q = w * 32 + __ffs(m) - 1, c = h.at(q / H::VEC) + q % H::VEC;
            if (slot < kCap) sh.cand[slot] = key_of((float)x[c], c);
            ++slot;
        }
}

// The first k of n candidates, in order, to sh.best: a candidate's place is the
// number of larger ones, and every wave counts among its share of them.
template <int W>
__device__ __forceinline__ void rank(Shared<W> &sh, int n, int k) {
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    n = __builtin_amdgcn_readfirstlane(n);
    const int share = ((n + W - 1) / W + 7) / 8 * 8, q0 = wave * share, q1 = min(q0 + share, n);
    for (int j = lane; j < n && q0 < n; j += 64) {
        const unsigned long long key = sh.cand[j];
        int r = 0;
#pragma unroll 1
        for (int q = q0; q < q1; q += 8) {
#pragma unroll
            for (int u = 0; u < 8; ++u) r += sh.cand[q + u] > key;   // (no key is above itself; zeros are above none)
        }
        if (W > 1) atomicAdd(&sh.rank[j], r);
        else if (r < k) sh.best[r] = key;
    }
    __syncthreads();
    if (W > 1) {
        for (int j = threadIdx.x; j < n; j += 64 * W)
            if (sh.rank[j] < k) sh.best[sh.rank[j]] = sh.cand[j];
        __syncthreads();
    }
}

// Empty candidates and places, which only a call that asks for the top columns
// reads (all threads of the workgroup; none may read the old ones any more).
template <int W>
__device__ __forceinline__ void clear(Shared<W> &sh, int k) {
    if (k == 0) return;
    for (int j = threadIdx.x; j < kCap + kMaxTopK + 8; j += 64 * W) sh.cand[j] = 0;
    for (int j = threadIdx.x; W > 1 && j < kCap + kMaxTopK; j += 64 * W) sh.rank[j] = 0;
    if (threadIdx.x == 0) sh.n = 0;
}

// Called by the whole workgroup where `push` found fewer than k candidates (all
// others are -inf) or more than there is room for (more than that many equal
// values, most often): the exact k-th largest value, what is above it, and of
// its equals the first columns.  Leaves exactly k candidates.  Reads the row
// again: a call that keeps the values in registers takes them from the usual
// case's second workgroup of a compute unit.
template <typename T, int NT>
__device__ __noinline__ void push_exact(Shared<NT / 64> &sh, const T *x, int lo, int hi, int k) {
    constexpr int W = NT / 64;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    auto value = [&](int c) { return fmaxf((float)x[min(c, hi - 1)], -INFINITY); };   // NaN: -inf
    // the sum over the workgroup of a wave's count, before: of the waves before this one
    auto total = [&](int n, int &before) {
        __syncthreads();
        if (lane == 0) sh.cnt[wave] = n;
        __syncthreads();
        n = before = 0;
        for (int w = 0; w < W; ++w) {
            if (w < wave) before += sh.cnt[w];
            n += sh.cnt[w];
        }
        return n;
    };
    const int found = sh.n;
    int have = found, before;
    uint32_t kth = order_of(-INFINITY);
    if (found > kCap) {
        // two bits at a time: the largest key that at least k reach
        kth = 0;
        for (int b = 30; b >= 0; b -= 2) {
            int n[3] = {0, 0, 0};
            for (int c0 = lo; c0 < hi; c0 += 4 * NT) {
                uint32_t o[4];
#pragma unroll
                for (int u = 0; u < 4; ++u) {
                    const int c = c0 + u * NT + (int)threadIdx.x;
                    const float v = value(c);
                    o[u] = c < hi ? order_of(v) : 0;
                }
#pragma unroll
                for (int u = 0; u < 4; ++u)
#pragma unroll
                    for (uint32_t q = 0; q < 3; ++q) n[q] += __popcll(__ballot(o[u] >= (kth | (q + 1) << b)));
            }
            uint32_t digit = 0;
#pragma unroll
            for (uint32_t q = 0; q < 3; ++q)
                if (total(n[q], before) >= k) digit = q + 1;
            kth |= digit << b;
        }
        __syncthreads();
        if (threadIdx.x == 0) sh.n = 0;
        __syncthreads();
        for (int c = lo + (int)threadIdx.x; c < hi; c += NT)
            if (order_of(value(c)) > kth) sh.cand[atomicAdd(&sh.n, 1)] = key_of(value(c), c);   // fewer than k
        __syncthreads();
        have = sh.n;
    }
    for (int c0 = lo; have < k && c0 < hi; c0 += NT) {
        const int c = c0 + (int)threadIdx.x;
        const bool eq = c < hi && order_of(value(c)) == kth;
        const unsigned long long mask = __ballot(eq);
        const int n = total(__popcll(mask), before), slot = have + before + lanes_below(mask);
        if (eq && slot < k) sh.cand[slot] = key_of(value_of(kth), c);
        have += n;
    }
    __syncthreads();
    if (threadIdx.x < 8) sh.cand[k + threadIdx.x] = 0;
    if (threadIdx.x == 0) sh.n = k;
    __syncthreads();
}

template <typename T, int NT, int PER, bool MORE>
__global__ __launch_bounds__(NT) __attribute__((amdgpu_waves_per_eu(PER == 64 ? 4 : MORE ? 6 : 1))) void answers_kernel(AnswersParams p, int segs, int rounds, int seglen) {
    constexpr int W = NT / 64;
    __shared__ Shared<W> sh;
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const unsigned block = blockIdx.y << kGridBits | blockIdx.x;
    const int row = block / segs, seg = block - row * segs;
    if (row >= p.rows) return;
    const T *x = (const T *)p.x + (size_t)row * p.cols;
    // channels of the lists, their values next, both long before they are used
    int listed[kAnswerLists];
    float value[kAnswerLists];
#pragma unroll
    for (int l = 0; l < kAnswerLists; ++l) {
        listed[l] = -1;
        if (tid < p.list_given[l]) listed[l] = p.list[l][(size_t)row * p.list_given[l] + tid];
    }
    clear(sh, p.k);
    const bool stats = p.n_lists > 0 || p.entropy;
    int lo = seg * rounds * seglen, hi = min(p.cols, lo + seglen);
    Held<T, NT, PER> h;
    h.load(x, lo, hi);
    float m = -FLT_MAX, s = 0.0f, t = 0.0f;    // (rows of -inf only: s = 0)
    int k = 0;                                 // keys in sh.best
    for (int round = 0;;) {
        // Where at least k lanes hold values, the k-th largest is at least the
        // smallest of the waves' r-th largest lane maxima, each wave with its
        // share r of k by its lanes that hold some: few values pass it.  Of a
        // later stretch of the row only what reaches the k-th so far does.
        const int len = hi - lo, kc = min(p.k, len);
        const int vecs = min(NT, (len + h.VEC - 1) / h.VEC), lanes = min(64, max(0, vecs - wave * 64));
        const int r = kc <= vecs ? (kc * lanes + vecs - 1) / vecs : 0;
        float mx = -INFINITY;
#pragma unroll
        for (int q = 0; q < PER; ++q) mx = fmaxf(mx, h.v[q]);
        const float wm = wave_max(mx);
        float bound = -INFINITY;
        if (r <= 5) {
            bound = wave_rth(mx, -INFINITY, r, [](float a, float b) { return fmaxf(a, b); });
        } else {
            const uint32_t near = wave_rth_near(order_of(mx), r);
            if (near >= order_of(-FLT_MAX)) bound = value_of(near);
        }
        if (lane == 0) {
            sh.m[wave] = wm;
            sh.bound[wave] = lanes > 0 ? bound : INFINITY;
        }
        __syncthreads();
        if (round == 0) {
#pragma unroll
            for (int l = 0; l < kAnswerLists; ++l)
                value[l] = listed[l] >= 0 && listed[l] < p.cols ? (float)x[listed[l]] : NAN;
        }
        const float before = m;
        bound = INFINITY;
#pragma unroll
        for (int w = 0; w < W; ++w) {
            m = fmaxf(m, sh.m[w]);
            bound = fminf(bound, sh.bound[w]);
        }
        if (MORE && round > 0 && p.k > 0) bound = fmaxf(bound, value_of((uint32_t)(sh.best[p.k - 1] >> 32)));
        if (kc > 0) push(sh, h, x, fmaxf(bound, -FLT_MAX));   // (-inf: push_exact)
        if (stats) {
            float s0 = 0.0f, t0 = 0.0f;
#pragma unroll
            for (int q = 0; q < PER; ++q) {
                const float d = h.v[q] - m, e = __builtin_amdgcn_exp2f(d * kLog2e);
                s0 += e;
                t0 = fmaf(e, fmaxf(d, -1e30f), t0);     // (0 times -inf)
            }
            s0 = wave_sum(s0);
            t0 = wave_sum(t0);
            if (lane == 0) {
                sh.s[wave] = s0;
                sh.t[wave] = t0;
            }
        }
        __syncthreads();
        if (stats) {
            if (MORE) {
                const float d = fmaxf(before - m, -1e30f), w0 = __builtin_amdgcn_exp2f(d * kLog2e);
                t = w0 * fmaf(s, d, t);
                s *= w0;
            }
#pragma unroll
            for (int w = 0; w < W; ++w) {
                s += sh.s[w];
                t += sh.t[w];
            }
        }
        if (kc > 0) {
            int n = sh.n;
            if (n > kCap || (k == 0 && n < kc)) {
                push_exact<T, NT>(sh, x, lo, hi, kc);
                n = kc;
            }
            if (MORE && k > 0) {                       // and the best so far
                if (tid < k + 8) sh.cand[n + tid] = tid < k ? sh.best[tid] : 0;   // (push_exact leaves what it dropped)
                n += k;
                __syncthreads();
            }
            k = min(p.k, k + len);
            rank(sh, n, k);
        }
        if (!MORE || ++round == rounds || hi == p.cols) break;
        lo = hi;
        hi = min(p.cols, hi + seglen);
        h.load(x, lo, hi);
        clear(sh, p.k);
    }
    if (segs > 1) {
        const int stride = answers_stride(p.k);
        for (int r = tid; r < stride; r += NT) put(p.part_keys + ((size_t)row * segs + seg) * stride + r, r < k ? sh.best[r] : 0ull);
        float *st = p.part_stats + (size_t)row * segs * 4;
        if (tid == 0) {
            put((unsigned long long *)(st + 4 * seg), (unsigned long long)__float_as_uint(s) << 32 | __float_as_uint(m));
            put((unsigned long long *)(st + 4 * seg) + 1, (unsigned long long)__float_as_uint(t));
        }
        if (!arrive_last(p.cnt + row, segs, &sh.last)) return;
        constexpr int C = kCap / NT;
        const int n = segs * stride;
        unsigned long long key[C];
        // (a segment to a lane: there are at most 64)
        f4 found = *(const f4 *)(st + 4 * min(lane, segs - 1));
        if (lane >= segs) found = f4{-FLT_MAX, 0.0f, 0.0f, 0.0f};
        if (p.k > 0) {
            // as above: a bound from the lanes' largest, then what reaches it.
            // Waves take eight keys in turns that shift by one, so that each has some of the first
            // and some of the last of the segments' (33 x 49999, k = 50: 268
            // candidates if each took one stretch, 141 so).
            const int at = ((lane >> 3) * W + ((wave + (lane >> 3)) & (W - 1))) * 8 + (lane & 7);
            uint32_t top = 0;
#pragma unroll
            for (int c = 0; c < C; ++c) key[c] = p.part_keys[(size_t)row * n + min(c * NT + at, n - 1)];
            clear(sh, p.k);
#pragma unroll
            for (int c = 0; c < C; ++c) {
                if (c * NT + at >= n) key[c] = 0;
                top = max(top, (uint32_t)(key[c] >> 32));
            }
            const int all = min(n, NT), units = all / 8, lanes = 8 * (units / W + (((wave + units / W) & (W - 1)) < units % W ? 1 : 0));
            const int r = (p.k * lanes + all - 1) / all;
            const uint32_t bound = r <= 5 ? wave_rth(top, 0u, r, [](uint32_t a, uint32_t b) { return max(a, b); }) : wave_rth_near(top, r);
            if (lane == 0) sh.key_bound[wave] = lanes > 0 ? bound : 0xFFFFFFFFu;
        }
        if (stats) {
            m = wave_max(found[0]);
            const float d = fmaxf(found[0] - m, -1e30f), w = __builtin_amdgcn_exp2f(d * kLog2e);
            s = wave_sum(w * found[1]);
            t = wave_sum(w * fmaf(found[1], d, found[2]));
        }
        __syncthreads();
        if (p.k > 0) {
            uint32_t bound = 0xFFFFFFFFu;
#pragma unroll
            for (int w = 0; w < W; ++w) bound = min(bound, sh.key_bound[w]);
            bound = max(bound, 1u);                // (not the filling of short segments)
            int mine = 0;
#pragma unroll
            for (int c = 0; c < C; ++c) mine += (uint32_t)(key[c] >> 32) >= bound;
            int slot = take_slots(&sh.n, mine);
#pragma unroll
            for (int c = 0; c < C; ++c)
                if ((uint32_t)(key[c] >> 32) >= bound) sh.cand[slot++] = key[c];
            __syncthreads();
            rank(sh, sh.n, p.k);
        }
    }
    for (int r = tid; r < p.k; r += NT) p.top[(size_t)row * p.k + r] = (int)~(uint32_t)sh.best[r];
    if (!stats) return;
    const float logs = logf(s);
#pragma unroll
    for (int l = 0; l < kAnswerLists; ++l) {
        if (l >= p.n_lists) break;
        const int *list = p.list[l];
        const int nl = p.list_n[l];
        for (int q = tid; q < nl; q += NT) {
            float v = value[l];
            if (!list) {
                v = value_of((uint32_t)(sh.best[q] >> 32));
            } else if (q != tid) {
                const int c = list[(size_t)row * nl + q];
                v = c >= 0 && c < p.cols ? (float)x[c] : NAN;
            }
            p.list_out[l][(size_t)row * nl + q] = s == 0.0f && v == v ? -INFINITY : (v - m) - logs;
        }
    }
    if (p.entropy && tid == 0) p.entropy[row] = s == 0.0f ? 0.0f : logs - t / s;
}

template <typename T>
hipError_t launch_t(const AnswersParams &p, const AnswersGeom &g, hipStream_t st) {
    const unsigned blocks = (unsigned)p.rows * (unsigned)g.segs;
    const dim3 grid(std::min(blocks, 1u << kGridBits), (blocks + (1u << kGridBits) - 1) >> kGridBits);
#define MGI_ANSWERS(NT_, PER_, MORE_)                                                                   \
    if (g.nt == NT_ && g.per == PER_ && (g.rounds > 1) == MORE_) {                                       \
        launch(answers_kernel<T, NT_, PER_, MORE_>, grid, dim3(NT_), 0, st, p, g.segs, g.rounds, g.seglen); \
        return hipGetLastError();                                                                       \
    }
    MGI_ANSWERS(64, 8, false) MGI_ANSWERS(256, 8, false) MGI_ANSWERS(256, 16, false) MGI_ANSWERS(256, 32, false)
    MGI_ANSWERS(512, 16, false) MGI_ANSWERS(512, 32, false) MGI_ANSWERS(512, 64, false) MGI_ANSWERS(512, 32, true)
#undef MGI_ANSWERS
    return hipErrorInvalidValue;
}

}  // namespace

// Segments: more than one where rows alone would leave compute units idle, none
// shorter than 2048 columns, and no more than the last workgroup can rank.  A
// workgroup takes a segment that its registers cannot hold in rounds (668 x
// 68012, k = 20: 50 us; as three segments with a join 128), of half of what they
// could hold: three workgroups to a compute unit then read while others compute
// (3269 x 38521, k = 5: 121 us; two with rounds of twice the length 157; four, for
// which 24 registers spill in fp32 and 37 in fp16, 142; three spill 2 and 14).  The more there is to rank, the more waves help
// (33 x 49999 fp16, k = 50: eight save 1.8 of 18.2 us; 23 x 69767, k = 3: they
// cost 2.7 on 12.4).
AnswersGeom answers_geom(int rows, int cols, int k) {
    AnswersGeom g{};
    const int most = k > 0 ? std::min(kCap / answers_stride(k), 64) : 64;
    g.segs = std::max(1, std::min({256 / std::max(rows, 1), (cols + 2047) / 2048, most}));
    const int len = (cols + g.segs - 1) / g.segs;
    g.rounds = len <= 32768 ? 1 : (len + 16383) / 16384;
    g.seglen = ((len + g.rounds - 1) / g.rounds + 7) / 8 * 8;
    g.segs = (cols + g.rounds * g.seglen - 1) / (g.rounds * g.seglen);
    const int sizes[6][2] = {{64, 8}, {256, 8}, {256, 16}, {256, 32}, {512, 32}, {512, 64}};
    for (auto &s : sizes) {
        g.nt = s[0];
        g.per = s[1];
        if (g.nt * g.per >= g.seglen) break;
    }
    if (g.nt == 256 && g.per == 32 && k > 16) {
        g.nt = 512;
        g.per = 16;
    }
    return g;
}

hipError_t launch_answers(const AnswersParams &p, const AnswersGeom &g, hipStream_t st) {
    if (p.rows <= 0) return hipSuccess;
    const long len = (long)g.rounds * g.seglen;
    if (g.segs < 1 || g.rounds < 1 || (long)g.nt * g.per < g.seglen || g.segs * len < p.cols || (g.segs - 1) * len >= p.cols ||
        (g.rounds > 1 && g.seglen < kMaxTopK) ||
        g.segs > 64 || (long)g.segs * answers_stride(p.k) > kCap || p.k > kMaxTopK || (g.segs > 1 && (!p.cnt || !p.part_stats)) ||
        (size_t)p.rows * g.segs > 0x7fffffffu)
        return hipErrorInvalidValue;
    AnswersParams q = p;
    for (int l = 0; l < kAnswerLists; ++l) {
        q.list_given[l] = l < p.n_lists && p.list[l] ? p.list_n[l] : 0;
        if (l < p.n_lists && !p.list[l] && p.list_n[l] != p.k) return hipErrorInvalidValue;
    }
    return p.fp16_in ? launch_t<_Float16>(q, g, st) : launch_t<float>(q, g, st);
}

}  // namespace kern
}  // namespace mgi
