// Log probabilities of given tokens under a softmax over the vocabulary, its
// entropy and its most probable tokens, and their gradient.
//
// Forward, one pass over a row's logits x: every thread keeps its own maximum m,
// M = m log2 e rounded to float32, and with t = x log2 e - M (one fused operation)
// the sums s = sum 2^t and u = sum 2^t t, rescaled when m grows.  Joined over
// threads, with the rounding left out of M, r = m log2 e - M, they give
// z = sum e^(x - m) = s 2^-r, logprob = (x - m) - ln z, lse = m + ln z and
// entropy = ln z - (u / s - r) ln 2 (no difference of large numbers).  Each thread
// has four 16-byte units in flight.  Bound by issue slots for 16-bit logits (8 to
// 9 instructions a logit: 8192 x 32000 bfloat16 97 us, 5.4 TB/s), by memory for
// float32 (2048 x 131072 157 us, 6.8 TB/s).  (Rows in a loop with the next row's
// first units in flight: 149 us for 108 at that state; it cost too many registers.)
//
// Alternatives.  Lower bounds of a row's k-th largest logit: the k-th largest of the
// 32 thread maxima of any warp, and, with W warps, the least of all warps'
// ceil(k / W)-th largest ones.  A thread also remembers the unit of its maximum and
// the maximum of its other units.  The threads whose maximum reaches the larger
// bound read that unit again and list its logits above the bound; the k-th largest
// of the list is a bound close to the k-th largest logit itself, and only threads
// whose second maximum reaches that one, hardly any, read their other units again
// (from L2).  Where the list is too short for the logits above the bound (rows with
// many equal logits), every warp keeps a sorted list of its own instead.  Five
// of 32000 take 123 us for the 97, 32 take 160; five of 131072 168 to 170 for 157.
#include <math.h>

#include <algorithm>

#include "rows.cuh"
#include "tc_common.cuh"

namespace jarq {
namespace {

using namespace rows;

constexpr int kMaxTop = 32, kMaxTokens = 256;
constexpr int kMaxSplit = 8;         // CTAs of a cluster that share a row
constexpr int kAhead = 4;            // units of a thread in flight
constexpr int kList = 512;           // candidates
constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;

struct ScoreArgs {
    const void *x;
    const int64_t *tokens;
    float *logprob, *entropy, *lse, *top_logprob;
    int32_t *top_token;
    int64_t ld;
    int n, vocab, t, k;
};

__device__ __forceinline__ float neg_inf() { return __int_as_float(0xFF800000); }
__device__ __forceinline__ float not_a_number() { return __int_as_float(0x7FC00000); }
// 2^x; the hardware's approximation, 2 units in the last place
__device__ __forceinline__ float exp2_fast(float x) {
    float r;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
    return r;
}
// the larger, or NaN if either is
__device__ __forceinline__ float max_nan(float a, float b) {
    float r;
    asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b));
    return r;
}
__device__ __forceinline__ float max_nan(float a, float b, float c) {
    float r;
    asm("max.NaN.f32 %0, %1, %2, %3;" : "=f"(r) : "f"(a), "f"(b), "f"(c));
    return r;
}
// float32 as an integer in the same order (-0 as +0); 0 is below -inf
__device__ __forceinline__ uint32_t ordered(float x) {
    const uint32_t b = __float_as_uint(x + 0.f);
    return b & 0x80000000u ? ~b : b | 0x80000000u;
}
__device__ __forceinline__ float unordered(uint32_t k) {
    return __uint_as_float(k & 0x80000000u ? k & 0x7FFFFFFFu : ~k);
}
// larger logits first, of equal ones the smaller position
__device__ __forceinline__ uint64_t key_of(float x, int pos) {
    return (uint64_t)ordered(x) << 32 | (0xFFFFFFFFu - (uint32_t)pos);
}
__device__ __forceinline__ int pos_of(uint64_t key) { return (int)(0xFFFFFFFFu - (uint32_t)key); }

// The reference M of a maximum m, and what its rounding leaves out.  Above 10^6
// that would be too much: t is then (x - m) log2 e, and nothing is left out.
__device__ __forceinline__ bool big(float m) { return !(fabsf(m) <= 1e6f); }
__device__ __forceinline__ float reference(float m) { return __fmul_rn(m, kLog2e); }
__device__ __forceinline__ float left_out(float m) { return big(m) ? 0.f : fmaf(m, kLog2e, -reference(m)); }

// m, s and u of some of a row's elements.  m = -inf: none that is not masked (s is
// 0, or NaN where one is NaN).
struct Sums {
    float m, s, u;
    // the same sums with the reference of top >= m
    __device__ void to(float top) {
        if (m == neg_inf() || m == top) return;
        // s d stays finite
        const float d = fmaxf((m - top) * kLog2e - left_out(m) + left_out(top), -1e30f), f = exp2_fast(d);
        u = (u + s * d) * f;
        s *= f;
        m = top;
    }
    __device__ void add(Sums o) {
        const float top = fmaxf(m, o.m);
        to(top);
        o.to(top);
        m = top;
        s += o.s;
        u += o.u;
    }
};

// The sums of a warp's lanes, in every lane.
__device__ __forceinline__ Sums warp_sums(Sums a) {
    const float top = unordered(__reduce_max_sync(0xffffffffu, ordered(a.m)));
    a.to(top);
#pragma unroll
    for (int i = 16; i > 0; i /= 2) {
        a.s += __shfl_xor_sync(0xffffffffu, a.s, i);
        a.u += __shfl_xor_sync(0xffffffffu, a.u, i);
    }
    return {top, a.s, a.u};
}

// Sorted over the warp's lanes, the largest in lane 0.
__device__ __forceinline__ uint32_t warp_sorted(uint32_t key, int lane) {
#pragma unroll
    for (int k = 2; k <= 32; k *= 2)
#pragma unroll
        for (int j = k / 2; j > 0; j /= 2) {
            const uint32_t o = __shfl_xor_sync(0xffffffffu, key, j);
            key = ((lane & j) == 0) == ((lane & k) == 0) ? max(key, o) : min(key, o);
        }
    return key;
}

// Keys of a falling list of 32 that are larger than `key`.
__device__ __forceinline__ int count_larger(const uint64_t *list, uint64_t key) {
    int c = 0;
#pragma unroll
    for (int step = 16; step > 0; step /= 2)
        if (list[c + step - 1] > key) c += step;
    return c + (list[c] > key);
}

// `key` into a falling list held one a lane.
__device__ __forceinline__ uint64_t inserted(uint64_t list, uint64_t key, int lane) {
    const int pos = __popc(__ballot_sync(0xffffffffu, list > key));
    const uint64_t up = __shfl_up_sync(0xffffffffu, list, 1);
    return lane < pos ? list : lane == pos ? key : up;
}

template <int kThreads>
struct Shared {
    static constexpr int kWarps = kThreads / 32, kLists = kWarps > kMaxSplit ? kWarps : kMaxSplit;
    union {
        uint64_t list[kList];
        uint64_t lists[kLists][32];
    };
    uint64_t best[kMaxTop];
    Sums sums[kWarps], total;
    uint32_t kth[kWarps], share[kWarps];    // of a warp's maxima: the k-th and the ceil(k / W)-th largest
    uint32_t near;                          // the k-th largest of the list
    int count;
};

// Address of a shared variable in CTA `rank` of the cluster.
template <class V>
__device__ __forceinline__ const V *in_cta(const V *p, int rank) {
    uint64_t r;
    asm("mapa.u64 %0, %1, %2;" : "=l"(r) : "l"((uint64_t)p), "r"(rank));
    return reinterpret_cast<const V *>(r);
}
__device__ __forceinline__ void cluster_barrier() {
    __syncwarp();
    asm volatile("barrier.cluster.arrive.release.aligned;\n barrier.cluster.wait.acquire.aligned;" ::: "memory");
}

// A CTA's part of a row: units u0 .. u1 - 1, of which lo .. hi - 1 lie in the row
// as a whole and are shared out kThreads apart; a cut first unit is thread 0's, a
// cut last one thread 1's.
template <class T, int kThreads>
struct Part {
    Row<T> row;
    int u0, u1, lo, hi;
    __device__ Part(const T *x, int vocab, int split, int rank) : row(x, vocab) {
        const int units = row.units(), per = (units + split - 1) / split;
        u0 = min(units, rank * per);
        u1 = min(units, u0 + per);
        lo = u0 + (u0 < u1 && !row.whole(u0));
        hi = max(lo, u1 - (lo < u1 && !row.whole(u1 - 1)));
    }
    // the whole units, and any unit with -inf, as if masked, outside the row
    __device__ const uint4 *units() const { return reinterpret_cast<const uint4 *>(row.p - row.skip); }
    __device__ uint4 load(int u) const { return row.load(u, from_float<T>(neg_inf())); }
    // f(u) for the cut units of thread `tid`
    template <class F>
    __device__ void cut(int tid, F f) const {
        if (tid == 0 && lo > u0) f(u0);
        if (tid == 1 && hi < u1) f(u1 - 1);
    }
};

// A thread's largest logit with its unit, and the largest of its other units.
struct Heads {
    float first, second;
    int unit;
};

// Ranks the listed candidates by counting; those below k go to sh.best, the k-th
// is the new bound.
template <int kThreads>
__device__ __forceinline__ void rank_list(Shared<kThreads> &sh, int count, int k) {
    for (int i = threadIdx.x; i < count; i += kThreads) {
        const uint64_t key = sh.list[i];
        int r = 0;
        for (int j = 0; j < count; ++j) r += sh.list[j] > key;
        if (r < k) sh.best[r] = key;
        if (r == k - 1) sh.near = (uint32_t)(key >> 32);
    }
}

// The k largest of a CTA's part into sh.best (0: none).  All threads; ends
// without a barrier.
template <class T, int kThreads>
__device__ __forceinline__ void select_top(Shared<kThreads> &sh, const Part<T, kThreads> &part, const Heads &h, int k) {
    constexpr int E = kUnit<T>, kWarps = kThreads / 32;
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    uint32_t bound = max(__reduce_max_sync(0xffffffffu, sh.kth[lane % kWarps]),
                         __reduce_min_sync(0xffffffffu, sh.share[lane % kWarps]));
    auto list = [&](int u) {
        float v[E];
        unpack(part.load(u), v, T());
#pragma unroll
        for (int e = 0; e < E; ++e)
            if (v[e] > neg_inf() && ordered(v[e]) >= bound) {
                const int at = atomicAdd(&sh.count, 1);
                if (at < kList) sh.list[at] = key_of(v[e], part.row.first(u) + e);
            }
    };
    if (h.first > neg_inf() && ordered(h.first) >= bound) list(h.unit);
    if (tid == 0) sh.near = bound;              // fewer than k listed: the bound stays
    __syncthreads();
    int count = sh.count;
    if (count <= kList) {
        rank_list(sh, count, k);
        __syncthreads();
        bound = sh.near;
        unsigned more = __ballot_sync(0xffffffffu, h.second > neg_inf() && ordered(h.second) >= bound);
        if (!__syncthreads_or(more != 0)) return;
        while (more) {
            // the other units of a thread, 32 at a time
            const int i = __ffs(more) - 1, skip = __shfl_sync(0xffffffffu, h.unit, i);
            more &= more - 1;
            for (int u = part.lo + 32 * warp + i + lane * kThreads; u < part.hi; u += 32 * kThreads)
                if (u != skip) list(u);
            if (lane == i)
                part.cut(tid, [&](int u) {
                    if (u != skip) list(u);
                });
            __syncwarp();
        }
        __syncthreads();
        count = sh.count;
        if (count <= kList) {
            rank_list(sh, count, k);
            return;
        }
    }
    __syncthreads();
    uint64_t best = 0;                      // the warp's largest so far, falling over the lanes
    for (int b = part.u0 + 32 * warp; b < part.u1; b += kThreads) {
        float v[E];
#pragma unroll
        for (int e = 0; e < E; ++e) v[e] = neg_inf();
        if (b + lane < part.u1) unpack(part.load(b + lane), v, T());
        const int f = part.row.first(b + lane);
#pragma unroll
        for (int e = 0; e < E; ++e) {
            const uint64_t c = v[e] > neg_inf() && ordered(v[e]) >= bound ? key_of(v[e], f + e) : 0;
            unsigned more = __ballot_sync(0xffffffffu, c > __shfl_sync(0xffffffffu, best, k - 1));
            while (more) {
                best = inserted(best, __shfl_sync(0xffffffffu, c, __ffs(more) - 1), lane);
                more &= more - 1;
            }
        }
    }
    if (tid < kMaxTop) sh.best[tid] = 0;
    sh.lists[warp][lane] = best;
    __syncthreads();
    if (best) {
        int r = lane;
        for (int w = 0; w < kWarps; ++w)
            if (w != warp) r += count_larger(sh.lists[w], best);
        if (r < k) sh.best[r] = best;
    }
}

template <class T, int kThreads, bool kTop>
__global__ void __launch_bounds__(kThreads, 1024 / kThreads) token_logprobs_kernel(ScoreArgs a) {
    constexpr int E = kUnit<T>, kWarps = kThreads / 32;
    __shared__ Shared<kThreads> sh;
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    uint32_t split, rank;
    asm("mov.u32 %0, %%cluster_nctarank;" : "=r"(split));
    asm("mov.u32 %0, %%cluster_ctarank;" : "=r"(rank));
    const int r = blockIdx.x / split;
    const T *x = static_cast<const T *>(a.x) + (size_t)r * a.ld;
    const Part<T, kThreads> part(x, a.vocab, split, rank);
    constexpr int kChunk = kAhead * kThreads;
    const int chunks = (part.hi - part.lo) / kChunk;       // whole ones
    const uint4 *next = part.units() + part.lo + tid;
    uint4 raw[kAhead];
    if (chunks > 0) {
#pragma unroll
        for (int i = 0; i < kAhead; ++i) raw[i] = next[i * kThreads];
    }
    // the given tokens' logits, on their way under the row
    int64_t tok = -1;
    float xt = 0.f;
    if (rank == 0 && tid < a.t) {
        tok = a.tokens[(size_t)r * a.t + tid];
        if (tok >= 0 && tok < a.vocab) xt = to_float(x[tok]);
    }
    float m = neg_inf(), ref = 0.f;
    Heads heads{neg_inf(), neg_inf(), -1};
    tc::F2 s2 = tc::f2(0.f), u2 = tc::f2(0.f);
    auto take = [&](const uint4 &w, int unit) {
        float v[E];
        unpack(w, v, T());
        float top = max_nan(v[0], v[1], v[2]);
#pragma unroll
        for (int e = 3; e < E; e += 2) top = e + 1 < E ? max_nan(top, v[e], v[e + 1]) : max_nan(top, v[e]);
        if (kTop) heads.second = fmaxf(heads.second, fminf(top, m));
        if (top > m) {
            Sums lo{m, 0.f, 0.f}, hi{m, 0.f, 0.f};
            tc::f2_get(s2, lo.s, hi.s);
            tc::f2_get(u2, lo.u, hi.u);
            lo.to(top);
            hi.to(top);
            s2 = tc::f2(lo.s, hi.s);
            u2 = tc::f2(lo.u, hi.u);
            m = top;
            ref = big(m) ? not_a_number() : reference(m);
            heads.unit = unit;
        }
        const tc::F2 scale = tc::f2(kLog2e), minus = tc::f2(-ref);
        tc::F2 t[E / 2], all = tc::f2(0.f);
#pragma unroll
        for (int i = 0; i < E / 2; ++i) {
            t[i] = tc::f2_fma(tc::f2(v[2 * i], v[2 * i + 1]), scale, minus);
            all = i ? tc::f2_add(all, t[i]) : t[i];
        }
        float a0, a1;
        tc::f2_get(all, a0, a1);
        if (!(fabsf(a0 + a1) <= 1e30f)) {       // -inf among them adds 0, not NaN; a large maximum
            const bool large = big(m) && m > neg_inf();
#pragma unroll
            for (int i = 0; i < E / 2; ++i) {
                tc::f2_get(t[i], a0, a1);
                if (large) {
                    a0 = (v[2 * i] - m) * kLog2e;
                    a1 = (v[2 * i + 1] - m) * kLog2e;
                }
                t[i] = tc::f2(a0 < -1e30f ? -1e30f : a0, a1 < -1e30f ? -1e30f : a1);     // NaN stays
            }
        }
#pragma unroll
        for (int i = 0; i < E / 2; ++i) {
            float t0, t1;
            tc::f2_get(t[i], t0, t1);
            const tc::F2 w2 = tc::f2(exp2_fast(t0), exp2_fast(t1));
            s2 = tc::f2_add(s2, w2);
            u2 = tc::f2_fma(w2, t[i], u2);
        }
    };
    int u = part.lo + tid;
    for (int c = 1; c < chunks; ++c) {
        next += kChunk;
#pragma unroll
        for (int i = 0; i < kAhead; ++i) {
            const uint4 w = raw[i];
            raw[i] = next[i * kThreads];
            take(w, u + i * kThreads);
        }
        u += kChunk;
    }
    if (chunks > 0) {
#pragma unroll
        for (int i = 0; i < kAhead; ++i) take(raw[i], u + i * kThreads);
        u += kChunk;
    }
    // what is left: up to kAhead units a thread
#pragma unroll
    for (int i = 0; i < kAhead; ++i)
        if (u + i * kThreads < part.hi) raw[i] = part.units()[u + i * kThreads];
#pragma unroll
    for (int i = 0; i < kAhead; ++i)
        if (u + i * kThreads < part.hi) take(raw[i], u + i * kThreads);
    part.cut(tid, [&](int cut) { take(part.load(cut), cut); });
    if (kTop) {
        const uint32_t sorted = warp_sorted(ordered(m), lane);
        if (lane == a.k - 1) sh.kth[warp] = sorted;
        if (lane == (a.k - 1) / kWarps) sh.share[warp] = sorted;
        if (tid < kMaxTop) sh.best[tid] = 0;
        if (tid == 0) sh.count = 0;
    }
    float s0, s1, u0, u1;
    tc::f2_get(s2, s0, s1);
    tc::f2_get(u2, u0, u1);
    Sums c = warp_sums({m, s0 + s1, u0 + u1});
    if (lane == 0) sh.sums[warp] = c;
    __syncthreads();
    if (kTop) {
        heads.first = m;
        select_top<T, kThreads>(sh, part, heads, a.k);
    }
    if (warp == 0) {
        c = warp_sums(lane < kWarps ? sh.sums[lane] : Sums{neg_inf(), 0.f, 0.f});
        if (lane == 0) sh.total = c;
    }
    if (split > 1) {
        cluster_barrier();
        if (rank == 0) {
            uint64_t key = 0;
            if (kTop && warp < kMaxSplit) {
                key = warp < (int)split ? in_cta(sh.best, warp)[lane] : 0;
                sh.lists[warp][lane] = key;
            }
            c = *in_cta(&sh.total, 0);
            for (int i = 1; i < (int)split; ++i) c.add(*in_cta(&sh.total, i));
            __syncthreads();
            if (kTop && tid < kMaxTop) sh.best[tid] = 0;
            if (tid == 0) sh.total = c;
            __syncthreads();
            if (kTop && key) {
                int p = lane;
                for (int i = 0; i < (int)split; ++i)
                    if (i != warp) p += count_larger(sh.lists[i], key);
                if (p < a.k) sh.best[p] = key;
            }
        }
    }
    __syncthreads();
    if (rank == 0) {
        c = sh.total;
        const bool bad = isnan(c.s), empty = !bad && c.m == neg_inf();
        // z is at least 1, its largest term: what the exponentials' rounding takes from
        // that would make probabilities above 1, and the entropy may fall below 0 alike
        const float rest = left_out(c.m), logz = empty ? 0.f : logf(fmaxf(c.s * exp2_fast(-rest), 1.f));
        if (tid == 0) {
            if (a.lse) a.lse[r] = bad ? not_a_number() : empty ? neg_inf() : c.m + logz;
            if (a.entropy) a.entropy[r] = bad ? not_a_number() : empty ? 0.f : fmaxf(logz - (c.u / c.s - rest) * kLn2, 0.f);
        }
        auto logprob = [&](float v) { return bad ? not_a_number() : v == neg_inf() ? v : (v - c.m) - logz; };
        for (int j = tid; j < a.t; j += kThreads) {
            if (j != tid) {
                tok = a.tokens[(size_t)r * a.t + j];
                if (tok >= 0 && tok < a.vocab) xt = to_float(x[tok]);
            }
            a.logprob[(size_t)r * a.t + j] = tok < 0 ? 0.f : tok >= a.vocab ? not_a_number() : logprob(xt);
        }
        if (kTop && tid < a.k) {
            const uint64_t key = sh.best[tid];
            const bool none = bad || key == 0;
            a.top_token[(size_t)r * a.k + tid] = none ? -1 : pos_of(key);
            a.top_logprob[(size_t)r * a.k + tid] =
                bad ? not_a_number() : none ? neg_inf() : logprob(unordered((uint32_t)(key >> 32)));
        }
    }
    if (split > 1) cluster_barrier();       // rank 0 reads the others' results until here
}

struct GradArgs {
    const void *x;
    const int64_t *tokens;
    const float *lse, *entropy, *g_logprob, *g_entropy;
    void *dx;
    int64_t ld, ldd;
    int n, vocab, t, chunks;            // CTAs of a row
};

// dx_v = sum_j g_j [v = tokens_j] - p_v (G + g_H (ln p_v + H)), G = sum_j g_j.
// A CTA writes the second term of its 16-byte units of a row, four a thread, then
// the tokens among them with both terms; all its logits are read first.  Bound by
// memory: 8192 x 32000 bf16, 1.05 GB, take 166 to 169 us with three sets of inputs in
// turn (6.2 TB/s); near issue slots too, and with the entropy's term 176.  kSame:
// logits and gradient have the same alignment.
constexpr int kGradThreads = 256, kGradUnits = kAhead * kGradThreads;

template <class T, bool kSame>
__global__ void __launch_bounds__(kGradThreads) token_grad_kernel(GradArgs a) {
    constexpr int E = kUnit<T>;
    __shared__ float sg[kMaxTokens];
    __shared__ int stok[kMaxTokens];
    const int tid = threadIdx.x, r = blockIdx.x / a.chunks, c = blockIdx.x % a.chunks;
    const T *x = static_cast<const T *>(a.x) + (size_t)r * a.ld;
    T *dx = static_cast<T *>(a.dx) + (size_t)r * a.ldd;
    const Row<T> row(x, a.vocab);
    const int u0 = c * kGradUnits, u1 = min(row.units(), u0 + kGradUnits);
    uint4 raw[kAhead];
#pragma unroll
    for (int i = 0; i < kAhead; ++i) {
        const int u = u0 + tid + i * kGradThreads;
        if (u < u1) raw[i] = row.load(u, from_float<T>(0.f));
    }
    const float lse = a.lse[r], gh = a.g_entropy ? a.g_entropy[r] : 0.f, h = a.g_entropy ? a.entropy[r] : 0.f;
    // the row's tokens: their weights, and the logits of those in this chunk
    // before they may be overwritten
    int tok = -1;
    float g = 0.f, xt = 0.f;
    if (tid < a.t) {
        const int64_t id = a.tokens[(size_t)r * a.t + tid];
        g = id < 0 ? 0.f : id >= a.vocab ? not_a_number() : a.g_logprob[(size_t)r * a.t + tid];
        if (id >= 0 && id < a.vocab) {
            const int unit = ((int)id + row.skip) / E;
            if (unit >= u0 && unit < u1) {
                tok = (int)id;
                xt = to_float(x[tok]);
            }
        }
        sg[tid] = g;
        stok[tid] = tok;
    }
    __syncthreads();
    float G = 0.f;
    for (int j = 0; j < a.t; ++j) G += sg[j];
    // Logits up to here get 0: masked ones, and those whose p is 0 by far, where v - lse
    // may overflow and 0 lp be NaN.  Only masked ones where a factor is not finite.
    const bool finite = isfinite(lse) && isfinite(G) && isfinite(gh) && isfinite(h);
    const float dead = finite ? lse - (1000.f + fabsf(lse) * 0x1p-10f) : neg_inf();
    auto soft = [&](float v) {
        const float lp = v - lse, p = exp2_fast(lp * kLog2e);
        float d = -G * p;
        if (a.g_entropy) d -= gh * (p * (lp + h));
        return v <= dead ? 0.f : d;
    };
#pragma unroll
    for (int i = 0; i < kAhead; ++i) {
        const int u = u0 + tid + i * kGradThreads;
        if (u >= u1) break;
        float v[E];
        unpack(raw[i], v, T());
#pragma unroll
        for (int e = 0; e < E; ++e) v[e] = soft(v[e]);
        const int f = row.first(u);
        if (kSame && row.whole(u)) {
            *reinterpret_cast<uint4 *>(dx + f) = pack(v, T());
        } else {
#pragma unroll
            for (int e = 0; e < E; ++e)
                if (f + e >= 0 && f + e < a.vocab) dx[f + e] = from_float<T>(v[e]);
        }
    }
    __syncthreads();
    if (tok >= 0 && xt != neg_inf()) {
        float d = soft(xt);
        for (int j = 0; j < a.t; ++j)
            if (stok[j] == tok) d += sg[j];
        dx[tok] = from_float<T>(d);
    }
}

template <class T, int kThreads>
cudaError_t launch_rows(const ScoreArgs &a, int split, cudaStream_t s) {
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)a.n * split);
    cfg.blockDim = dim3(kThreads);
    cfg.stream = s;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = split;
    attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    return a.k ? cudaLaunchKernelEx(&cfg, token_logprobs_kernel<T, kThreads, true>, a)
               : cudaLaunchKernelEx(&cfg, token_logprobs_kernel<T, kThreads, false>, a);
}

cudaError_t launch_logprobs(const ScoreArgs &a, jarq_dtype dtype, cudaStream_t s) {
    const int64_t units = (int64_t)a.vocab * (int64_t)size_of(dtype) / 16;
    // Few rows: the CTAs of a cluster share one, as long as each has some 900 units
    // (48 x 50001 fp16: 11.3 us by one CTA a row, 9.9 by four, 11.3 by eight).  Of
    // many rows or short ones a CTA of 128 threads is better, since each has its
    // own sums to join (8192 x 32000 bf16: 109 us, 121 with 256 threads; 600 x
    // 131072 float32: 78 us, 56 with 256).
    int split = 1;
    while (split < kMaxSplit && 2 * (int64_t)a.n * split < 3 * num_sms() && units / (2 * split) >= 900) split *= 2;
    const bool small = split == 1 && (units <= 2048 || a.n >= 8 * num_sms());
    return with_type(dtype, [&](auto type) {
        using T = decltype(type);
        return small ? launch_rows<T, 128>(a, 1, s) : launch_rows<T, 256>(a, split, s);
    });
}

cudaError_t launch_grad(GradArgs a, jarq_dtype dtype, cudaStream_t s) {
    const size_t b = size_of(dtype);
    const int units = (int)(((size_t)a.vocab * b + 15) / 16 + 1);
    a.chunks = (units + kGradUnits - 1) / kGradUnits;
    const int64_t grid = (int64_t)a.n * a.chunks;
    if (grid > 0x7FFFFFFF) return cudaErrorInvalidValue;
    const bool same = (((uintptr_t)a.x ^ (uintptr_t)a.dx) & 15) == 0 && (a.n == 1 || ((a.ld - a.ldd) * (int64_t)b) % 16 == 0);
    with_type(dtype, [&](auto type) {
        using T = decltype(type);
        if (same)
            token_grad_kernel<T, true><<<(unsigned)grid, kGradThreads, 0, s>>>(a);
        else
            token_grad_kernel<T, false><<<(unsigned)grid, kGradThreads, 0, s>>>(a);
        return 0;
    });
    return cudaGetLastError();
}

bool aligned(const void *p, size_t b) { return ((uintptr_t)p & (b - 1)) == 0; }

jarq_status check_logits(const void *x, jarq_dtype dtype, int n, int vocab, int64_t ld,
                         const int64_t *tokens, int t) {
    if (n < 0 || vocab < 1 || vocab > 1 << 30 || ld < vocab || t < 0 || t > kMaxTokens || !is_dtype(dtype)) return JARQ_ERR_ARG;
    if (n == 0) return JARQ_OK;
    if (!x || !on_device(x) || !aligned(x, size_of(dtype))) return JARQ_ERR_ARG;
    if (t && (!tokens || !on_device(tokens) || !aligned(tokens, 8))) return JARQ_ERR_ARG;
    return JARQ_OK;
}
bool is_floats(const void *p) { return p && on_device(p) && aligned(p, 4); }

jarq_status finish(cudaError_t e) {
    count_launches(1);
    if (e == cudaSuccess) return JARQ_OK;
    (void)cudaGetLastError();
    return JARQ_ERR_CUDA;
}

}  // namespace
}  // namespace jarq

using namespace jarq;

extern "C" {

jarq_status jarq_token_logprobs(const void *logits, jarq_dtype dtype, int n, int vocab, int64_t ld,
                                const int64_t *tokens, int t, int k, float *logprob,
                                float *entropy, float *lse, float *top_logprob,
                                int32_t *top_token, void *stream) {
    const jarq_status ok = check_logits(logits, dtype, n, vocab, ld, tokens, t);
    if (ok != JARQ_OK || k < 0 || k > kMaxTop || k > vocab) return JARQ_ERR_ARG;
    if (n == 0) return JARQ_OK;
    if ((t && !is_floats(logprob)) || (entropy && !is_floats(entropy)) || (lse && !is_floats(lse)) ||
        (k && (!is_floats(top_logprob) || !is_floats(top_token))))
        return JARQ_ERR_ARG;
    if (const jarq_status late = async_failure()) return late;
    cudaStream_t st = (cudaStream_t)stream;
    ProfScope ps("token_logprobs", st);
    const cudaError_t e = launch_logprobs({logits, tokens, logprob, entropy, lse, top_logprob, top_token, ld, n, vocab, t, k},
                                          dtype, st);
    ps.done();
    return finish(e);
}

jarq_status jarq_token_logprobs_grad(const void *logits, jarq_dtype dtype, int n, int vocab,
                                     int64_t ld, const int64_t *tokens, int t, const float *lse,
                                     const float *entropy, const float *g_logprob,
                                     const float *g_entropy, void *dlogits, int64_t ldd,
                                     void *stream) {
    const jarq_status ok = check_logits(logits, dtype, n, vocab, ld, tokens, t);
    if (ok != JARQ_OK || t < 1 || ldd < vocab) return JARQ_ERR_ARG;
    if (n == 0) return JARQ_OK;
    if (!dlogits || !on_device(dlogits) || !aligned(dlogits, size_of(dtype)) || (dlogits == logits && n > 1 && ldd != ld))
        return JARQ_ERR_ARG;
    if (!is_floats(lse) || !is_floats(g_logprob) || (g_entropy && (!is_floats(g_entropy) || !is_floats(entropy))))
        return JARQ_ERR_ARG;
    if (const jarq_status late = async_failure()) return late;
    cudaStream_t st = (cudaStream_t)stream;
    ProfScope ps("token_grad", st);
    const cudaError_t e = launch_grad({logits, tokens, lse, entropy, g_logprob, g_entropy, dlogits, ld, ldd, n, vocab, t, 0},
                                      dtype, st);
    ps.done();
    return finish(e);
}

}  // extern "C"
