// Questions about the channels of each pixel: the k largest, the logarithm of
// the softmax at given channels, the softmax's entropy.
//
// With m the row's maximum, s = sum exp(x - m) and t = sum exp(x - m) (x - m):
//     log softmax(x)_i = (x_i - m) - log s,    entropy = log s - t / s.
// Both terms of the entropy are non-negative, so neither loses digits to the
// other.  Sums are fp32.
//
// One workgroup owns a row, or a segment of one, and holds it in registers, so
// the row is read once whatever is asked: a call is bound by the row's bytes.
// Where rows are few or long they are split into segments; each leaves its
// (m, s, t) and its own k best, and the workgroup that arrives last joins them.
#include "device.h"

namespace mgi {
namespace kern {

namespace {

constexpr int kCap = 1024;            // candidates a workgroup ranks
constexpr float kLog2e = 1.44269504088896341f;

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

// A bound that at least r of a wave's 64 integers, all from lo to hi, reach: the
// r-th largest, or less where exactly r reach it already.  Two bits a step,
// from the first that differ.
__device__ __forceinline__ uint32_t wave_bound(uint32_t o, uint32_t lo, uint32_t hi, int r) {
    if (lo == hi) return hi;
    int b = (31 - __builtin_clz(lo ^ hi)) & ~1;
    uint32_t ans = hi >> b >> 2 << b << 2;
#pragma unroll 1
    for (; b >= 0; b -= 2) {
        int n[3];
#pragma unroll
        for (uint32_t q = 0; q < 3; ++q) n[q] = __popcll(__ballot(o >= (ans | (q + 1) << b)));
        const int got = n[2] >= r ? n[2] : n[1] >= r ? n[1] : n[0];
        ans |= (n[2] >= r ? 3u : n[1] >= r ? 2u : n[0] >= r ? 1u : 0u) << b;
        if (got == r) break;
    }
    return ans;
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
    alignas(16) unsigned long long cand[kCap + 8];
    float top_val[kMaxTopK];
    float m[W], s[W], t[W];
    uint32_t bound[W];
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

// Adds the values of at least `th` to the candidates.  A lane marks its own and
// then takes them one after the other, reading them again from memory (the
// cache): few lanes have more than two or three, but among a wave's lanes
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
#pragma unroll
    for (int w = 0; w < (PER + 31) / 32; ++w)
#pragma unroll 1
        for (uint32_t m = mark[w]; m; m &= m - 1) {
            const int q = w * 32 + __ffs(m) - 1, c = h.at(q / H::VEC) + q % H::VEC;
            if (slot < kCap) sh.cand[slot] = key_of((float)x[c], c);
            ++slot;
        }
}

// Hands every candidate of the first k to `found`, with its rank: the number of
// larger ones.  Behind the last there are seven zeros, below every key.
template <int NT, typename F>
__device__ __forceinline__ void rank(const unsigned long long *cand, int n, int k, F found) {
    n = __builtin_amdgcn_readfirstlane(n);
    for (int j = threadIdx.x; j < n; j += NT) {
        const unsigned long long key = cand[j];
        int r = 0;
#pragma unroll 1
        for (int q = 0; q < n; q += 8) {
#pragma unroll
            for (int u = 0; u < 8; ++u) r += cand[q + u] > key;
        }
        if (r < k) found(r, key);
    }
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

template <typename T, int NT, int PER>
__global__ __launch_bounds__(NT) __attribute__((amdgpu_waves_per_eu(PER == 64 ? 4 : 1))) void answers_kernel(AnswersParams p, int segs, int seglen) {
    constexpr int W = NT / 64;
    __shared__ Shared<W> sh;
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int row = blockIdx.x / segs, seg = blockIdx.x - row * segs;
    const T *x = (const T *)p.x + (size_t)row * p.cols;
    // channels of the lists, their values next, both long before they are used
    int listed[kAnswerLists];
    float value[kAnswerLists];
#pragma unroll
    for (int l = 0; l < kAnswerLists; ++l) {
        listed[l] = -1;
        if (tid < p.list_given[l]) listed[l] = p.list[l][(size_t)row * p.list_given[l] + tid];
    }
    for (int j = tid; j < kCap + 8; j += NT) sh.cand[j] = 0;
    Held<T, NT, PER> h;
    h.load(x, seg * seglen, min(p.cols, (seg + 1) * seglen));
    const int k = min(p.k, h.hi - h.lo);
    const bool stats = p.n_lists > 0 || p.entropy;

    // The k-th largest value is at least the smallest of the waves' r-th
    // largest lane maxima, r = ceil(k / waves): few values pass it.  (Waves
    // past the end of a short row hold nothing and do not count.)
    const int held = min(W, (h.hi - h.lo + 64 * h.VEC - 1) / (64 * h.VEC));
    float mx = -INFINITY;
#pragma unroll
    for (int q = 0; q < PER; ++q) mx = fmaxf(mx, h.v[q]);
    {
        const float wm = wave_max(mx), wl = -wave_max(-mx);
        const int r = (k + held - 1) / held;
        const uint32_t bound = r > 1 ? wave_bound(order_of(mx), order_of(wl), order_of(wm), r) : order_of(wm);
        if (lane == 0) {
            sh.m[wave] = wm;
            sh.bound[wave] = wave < held ? bound : 0xFFFFFFFFu;
        }
        if (tid == 0) sh.n = 0;
    }
    __syncthreads();
#pragma unroll
    for (int l = 0; l < kAnswerLists; ++l)
        value[l] = listed[l] >= 0 && listed[l] < p.cols ? (float)x[listed[l]] : NAN;
    float m = -FLT_MAX;                   // (rows of -inf only: s = 0)
    uint32_t bound = 0xFFFFFFFFu;
#pragma unroll
    for (int w = 0; w < W; ++w) {
        m = fmaxf(m, sh.m[w]);
        bound = min(bound, sh.bound[w]);
    }
    if (k > 0) push(sh, h, x, value_of(max(bound, order_of(-FLT_MAX))));   // (-inf: push_exact)
    float s = 0.0f, t = 0.0f;
    if (stats) {
#pragma unroll
        for (int q = 0; q < PER; ++q) {
            const float d = h.v[q] - m, e = __builtin_amdgcn_exp2f(d * kLog2e);
            s += e;
            t = fmaf(e, fmaxf(d, -1e30f), t);     // (0 times -inf)
        }
        s = wave_sum(s);
        t = wave_sum(t);
        if (lane == 0) {
            sh.s[wave] = s;
            sh.t[wave] = t;
        }
    }
    __syncthreads();
    if (stats) {
        s = t = 0.0f;
#pragma unroll
        for (int w = 0; w < W; ++w) {
            s += sh.s[w];
            t += sh.t[w];
        }
    }
    if (k > 0) {
        if (sh.n < k || sh.n > kCap) push_exact<T, NT>(sh, x, h.lo, h.hi, k);
        rank<NT>(sh.cand, sh.n, k, [&](int r, unsigned long long key) {
            if (segs > 1) {
                put(p.part_keys + ((size_t)row * segs + seg) * p.k + r, key);
            } else {
                p.top[(size_t)row * p.k + r] = (int)~(uint32_t)key;
                sh.top_val[r] = value_of((uint32_t)(key >> 32));
            }
        });
        if (segs > 1)
            for (int r = k + tid; r < p.k; r += NT) put(p.part_keys + ((size_t)row * segs + seg) * p.k + r, 0ull);
    }
    if (segs > 1) {
        float *st = p.part_stats + (size_t)row * segs * 4;
        if (tid == 0) {
            put((unsigned long long *)(st + 4 * seg), (unsigned long long)__float_as_uint(s) << 32 | __float_as_uint(m));
            put((unsigned long long *)(st + 4 * seg) + 1, (unsigned long long)__float_as_uint(t));
        }
        if (!arrive_last(p.cnt + row, segs, &sh.last)) return;
        constexpr int C = kCap / NT;
        const int n = segs * p.k;
        unsigned long long key[C];
        // (a segment to a lane: there are at most 64)
        f4 found = *(const f4 *)(st + 4 * min(lane, segs - 1));
        if (lane >= segs) found = f4{-FLT_MAX, 0.0f, 0.0f, 0.0f};
        if (p.k > 0) {
            // as above: a bound from the lanes' largest, of the waves that
            // hold keys; then what reaches it
            uint32_t top = 0;
#pragma unroll
            for (int c = 0; c < C; ++c) {
                const int j = c * NT + tid;
                key[c] = p.part_keys[(size_t)row * n + min(j, n - 1)];
            }
#pragma unroll
            for (int c = 0; c < C; ++c) {
                const int j = c * NT + tid;
                if (j >= n) key[c] = 0;
                sh.cand[j] = 0;
            }
#pragma unroll
            for (int c = 0; c < C; ++c) top = max(top, (uint32_t)(key[c] >> 32));
            const int have = min(W, (n + 63) / 64);
            const uint32_t hi = wave_all(top, 0u, [](uint32_t a, uint32_t b) { return max(a, b); });
            const uint32_t lo = wave_all(top, 0xFFFFFFFFu, [](uint32_t a, uint32_t b) { return min(a, b); });
            const int r = (p.k + have - 1) / have;
            const uint32_t bound = r > 1 ? wave_bound(top, lo, hi, r) : hi;
            if (lane == 0) sh.bound[wave] = wave < have ? bound : 0xFFFFFFFFu;
            if (tid == 0) sh.n = 0;
        }
        if (stats) {
            m = wave_max(found[0]);
            const float d = fmaxf(found[0] - m, -1e30f), w = __builtin_amdgcn_exp2f(d * kLog2e);
            s = wave_sum(w * found[1]);
            t = wave_sum(w * fmaf(found[1], d, found[2]));
        }
        __syncthreads();
        if (p.k > 0) {
            bound = 0xFFFFFFFFu;
#pragma unroll
            for (int w = 0; w < W; ++w) bound = min(bound, sh.bound[w]);
            bound = max(bound, 1u);                // (not the filling of short segments)
            int mine = 0;
#pragma unroll
            for (int c = 0; c < C; ++c) mine += (uint32_t)(key[c] >> 32) >= bound;
            int slot = take_slots(&sh.n, mine);
#pragma unroll
            for (int c = 0; c < C; ++c)
                if ((uint32_t)(key[c] >> 32) >= bound) sh.cand[slot++] = key[c];
            __syncthreads();
            rank<NT>(sh.cand, sh.n, p.k, [&](int r, unsigned long long k1) {
                p.top[(size_t)row * p.k + r] = (int)~(uint32_t)k1;
                sh.top_val[r] = value_of((uint32_t)(k1 >> 32));
            });
        }
    }
    if (!stats) return;
    __syncthreads();
    const float logs = logf(s);
#pragma unroll
    for (int l = 0; l < kAnswerLists; ++l) {
        if (l >= p.n_lists) break;
        const int *list = p.list[l];
        const int nl = p.list_n[l];
        for (int q = tid; q < nl; q += NT) {
            float v = list ? value[l] : sh.top_val[q];
            if (list && q != tid) {
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
    const dim3 grid((unsigned)p.rows * (unsigned)g.segs);
#define MGI_ANSWERS(NT_, PER_)                                                                   \
    if (g.nt == NT_ && g.per == PER_) {                                                           \
        launch(answers_kernel<T, NT_, PER_>, grid, dim3(NT_), 0, st, p, g.segs, g.seglen);       \
        return hipGetLastError();                                                                 \
    }
    MGI_ANSWERS(64, 8) MGI_ANSWERS(256, 8) MGI_ANSWERS(256, 16) MGI_ANSWERS(256, 32)
    MGI_ANSWERS(512, 32) MGI_ANSWERS(512, 64)
#undef MGI_ANSWERS
    return hipErrorInvalidValue;
}

}  // namespace

// Segments: as many as a workgroup's registers make necessary, more where rows
// alone would leave compute units idle, none shorter than 2048 columns, and no
// more than the last workgroup can rank.
AnswersGeom answers_geom(int rows, int cols, int k) {
    AnswersGeom g{};
    const int most = k > 0 ? std::min(kCap / k, 64) : 64;
    int segs = (cols + 32767) / 32768;
    segs = std::max(segs, std::min({256 / std::max(rows, 1), (cols + 2047) / 2048, most}));
    g.seglen = ((cols + segs - 1) / segs + 7) / 8 * 8;
    g.segs = (cols + g.seglen - 1) / g.seglen;
    const int sizes[6][2] = {{64, 8}, {256, 8}, {256, 16}, {256, 32}, {512, 32}, {512, 64}};
    for (auto &s : sizes) {
        g.nt = s[0];
        g.per = s[1];
        if (g.nt * g.per >= g.seglen) break;
    }
    return g;
}

hipError_t launch_answers(const AnswersParams &p, const AnswersGeom &g, hipStream_t st) {
    if (p.rows <= 0) return hipSuccess;
    if (g.segs < 1 || (long)g.nt * g.per < g.seglen || (long)g.segs * g.seglen < p.cols || (g.segs - 1) * g.seglen >= p.cols ||
        g.segs > 64 || (long)g.segs * p.k > kCap || p.k > kMaxTopK || (g.segs > 1 && (!p.cnt || !p.part_stats)) ||
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
