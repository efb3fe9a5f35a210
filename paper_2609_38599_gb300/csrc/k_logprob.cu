// Log probabilities of given tokens under a softmax over the vocabulary, its
// entropy and its most probable tokens, and their gradient.
//
// Forward, one pass over a row's logits x: every thread keeps its own maximum m
// and the sums s = sum e^(x - m), u = sum e^(x - m) (x - m), rescaled when m
// grows; joined over threads they give lse = m + ln s, logprob = (x - m) - ln s
// and entropy = ln s - u / s (no difference of large numbers).
//
// Alternatives.  A thread also remembers the 16-byte unit in which its maximum
// stands, so (maximum, unit) orders the threads without ties, in the order of
// (logit falling, token rising).  The k largest of these pairs are k different
// elements, and every element of another thread comes after all of them:
// the k largest elements of the row lie in the k threads with the largest
// pairs.  Only those threads' elements, about k / 256 of the row, are read a
// second time (from L2).
#include <math.h>

#include "rows.cuh"

namespace jarq {
namespace {

using namespace rows;

constexpr int kThreads = 256, kWarps = kThreads / 32;
constexpr int kMaxTop = 32, kMaxTokens = 256;
constexpr int kMaxSplit = 8;         // CTAs of a cluster that share a row
constexpr int kAhead = 4;            // units of a thread in flight
constexpr float kLog2e = 1.4426950408889634f;

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

// m, s, u of some of a row's elements.  m = -inf: none that is not masked (s is
// 0, or NaN where one is NaN).
struct Sums {
    float m, s, u;
    // the same sums with respect to M >= m
    __device__ void to(float M) {
        if (m == neg_inf()) return;
        if (m == M) return;
        const float d = fmaxf(m - M, -1e30f), f = exp2_fast(d * kLog2e);   // s d stays finite
        u = (u + s * d) * f;
        s *= f;
    }
    __device__ void add(Sums o) {
        const float M = fmaxf(m, o.m);
        to(M);
        o.to(M);
        m = M;
        s += o.s;
        u += o.u;
    }
};

__device__ __forceinline__ Sums shuffled(const Sums &a, int mask) {
    return {__shfl_xor_sync(0xffffffffu, a.m, mask), __shfl_xor_sync(0xffffffffu, a.s, mask),
            __shfl_xor_sync(0xffffffffu, a.u, mask)};
}

// Sorted over the warp's lanes, the largest in lane 0.
__device__ __forceinline__ uint64_t warp_sorted(uint64_t key, int lane) {
#pragma unroll
    for (int k = 2; k <= 32; k *= 2)
#pragma unroll
        for (int j = k / 2; j > 0; j /= 2) {
            const uint64_t o = __shfl_xor_sync(0xffffffffu, key, j);
            const bool larger = ((lane & j) == 0) == ((lane & k) == 0);
            if ((o > key) == larger) key = o;
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

struct Shared {
    uint64_t lists[kWarps][32];
    uint64_t seg[kMaxTop], best[kMaxTop];
    Sums sums[kWarps];
    Sums total;
};

// Position of the calling thread's key, lists[warp][lane], among all lists.
__device__ __forceinline__ int rank_of(const Shared &sh, uint64_t key, int warp, int lane) {
    int r = lane;
#pragma unroll
    for (int w = 0; w < kWarps; ++w)
        if (w != warp) r += count_larger(sh.lists[w], key);
    return r;
}

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

template <class T, bool kTop>
__global__ void __launch_bounds__(kThreads) token_logprobs_kernel(ScoreArgs a) {
    constexpr int E = kUnit<T>;
    __shared__ Shared sh;
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    uint32_t split, rank;
    asm("mov.u32 %0, %%cluster_nctarank;" : "=r"(split));
    asm("mov.u32 %0, %%cluster_ctarank;" : "=r"(rank));
    const int r = blockIdx.x / split;
    const T *x = static_cast<const T *>(a.x) + (size_t)r * a.ld;
    const Row<T> row(x, a.vocab);
    const int units = row.units(), per = (units + split - 1) / split;
    const int u0 = min(units, (int)rank * per), u1 = min(units, u0 + per);
    const T masked = from_float<T>(neg_inf());      // what lies outside the row counts as masked

    Sums a0{neg_inf(), 0.f, 0.f};
    int best = -1;
    auto take = [&](const uint4 &raw, int u) {
        float v[E];
        unpack(raw, v, T());
        float top = v[0];
#pragma unroll
        for (int e = 1; e < E; ++e) top = max_nan(top, v[e]);
        if (top > a0.m) {
            a0.to(top);
            a0.m = top;
            best = u;
        }
        if (top == neg_inf()) return;
#pragma unroll
        for (int e = 0; e < E; ++e) {
            const float d = v[e] - a0.m, w = exp2_fast(d * kLog2e);
            a0.s += w;
            a0.u += w * fmaxf(d, -1e30f);       // 0, not NaN, for a masked element
        }
    };
    int u = u0 + tid;
    for (; u + (kAhead - 1) * kThreads < u1; u += kAhead * kThreads) {
        uint4 raw[kAhead];
#pragma unroll
        for (int i = 0; i < kAhead; ++i) raw[i] = row.load(u + i * kThreads, masked);
#pragma unroll
        for (int i = 0; i < kAhead; ++i) take(raw[i], u + i * kThreads);
    }
    for (; u < u1; u += kThreads) take(row.load(u, masked), u);
    const float own_max = a0.m;

    if (kTop) sh.lists[warp][lane] = warp_sorted(best < 0 ? (uint64_t)tid : key_of(own_max, best), lane);
#pragma unroll
    for (int i = 16; i > 0; i /= 2) a0.add(shuffled(a0, i));
    if (lane == 0) sh.sums[warp] = a0;
    if (kTop && tid < kMaxTop) sh.best[tid] = 0;
    __syncthreads();
    if (kTop) {
        const uint64_t key = sh.lists[warp][lane];
        const int at = rank_of(sh, key, warp, lane);
        if (at < a.k) sh.seg[at] = key;
        __syncthreads();
        const uint32_t least = (uint32_t)(sh.seg[a.k - 1] >> 32);
        uint64_t list = 0;                      // the warp's largest so far, falling over the lanes
        for (int i = warp; i < a.k; i += kWarps) {
            const uint64_t head = sh.seg[i];
            if (head >> 32 == 0) break;         // threads without a token
            const int first = u0 + (pos_of(head) - u0) % kThreads;
            for (int b = first; b < u1; b += 32 * kThreads) {
                const int w = b + lane * kThreads;
                float v[E];
                const bool in = w < u1;
                if (in) unpack(row.load(w, masked), v, T());
                const int f = row.first(w);
#pragma unroll
                for (int e = 0; e < E; ++e) {
                    const uint64_t c = in && v[e] > neg_inf() && ordered(v[e]) >= least ? key_of(v[e], f + e) : 0;
                    const uint64_t last = __shfl_sync(0xffffffffu, list, a.k - 1);
                    unsigned more = __ballot_sync(0xffffffffu, c > last);
                    while (more) {
                        const uint64_t ins = __shfl_sync(0xffffffffu, c, __ffs(more) - 1);
                        more &= more - 1;
                        const int pos = __popc(__ballot_sync(0xffffffffu, list > ins));
                        const uint64_t up = __shfl_up_sync(0xffffffffu, list, 1);
                        if (lane >= pos) list = lane == pos ? ins : up;
                    }
                }
            }
        }
        sh.lists[warp][lane] = list;
        __syncthreads();
        if (list) {
            const int p = rank_of(sh, list, warp, lane);
            if (p < a.k) sh.best[p] = list;
        }
    }
    if (warp == 0) {
        Sums c = sh.sums[lane % kWarps];
#pragma unroll
        for (int i = kWarps / 2; i > 0; i /= 2) c.add(shuffled(c, i));
        if (lane == 0) sh.total = c;
    }
    if (split > 1) {
        cluster_barrier();
        if (rank != 0) {
            cluster_barrier();                  // rank 0 still reads this CTA's results
            return;
        }
        if (kTop) {
            const uint64_t key = warp < (int)split ? in_cta(sh.best, warp)[lane] : 0;
            sh.lists[warp][lane] = key;
        }
        Sums c = *in_cta(&sh.total, 0);
        for (int i = 1; i < (int)split; ++i) c.add(*in_cta(&sh.total, i));
        cluster_barrier();                      // nothing of the others is read from here on
        if (tid == 0) sh.total = c;
        if (kTop && tid < kMaxTop) sh.best[tid] = 0;
        __syncthreads();
        if (kTop) {
            const uint64_t key = sh.lists[warp][lane];
            if (key) {
                const int p = rank_of(sh, key, warp, lane);
                if (p < a.k) sh.best[p] = key;
            }
        }
    }
    __syncthreads();
    const Sums c = sh.total;
    const bool bad = isnan(c.s), empty = !bad && c.m == neg_inf();
    const float logz = empty ? 0.f : logf(c.s);
    if (tid == 0) {
        if (a.lse) a.lse[r] = bad ? not_a_number() : empty ? neg_inf() : c.m + logz;
        if (a.entropy) a.entropy[r] = bad ? not_a_number() : empty ? 0.f : logz - c.u / c.s;
    }
    auto logprob = [&](float v) { return bad ? not_a_number() : v == neg_inf() ? v : (v - c.m) - logz; };
    if (tid < a.t) {
        const int64_t tok = a.tokens[(size_t)r * a.t + tid];
        a.logprob[(size_t)r * a.t + tid] = tok < 0 ? 0.f : tok >= a.vocab ? not_a_number() : logprob(to_float(x[tok]));
    }
    if (kTop && tid < a.k) {
        const uint64_t key = sh.best[tid];
        const bool none = bad || key == 0;
        a.top_token[(size_t)r * a.k + tid] = none ? -1 : pos_of(key);
        a.top_logprob[(size_t)r * a.k + tid] =
            bad ? not_a_number() : none ? neg_inf() : logprob(unordered((uint32_t)(key >> 32)));
    }
}

struct GradArgs {
    const void *x;
    const int64_t *tokens;
    const float *lse, *entropy, *g_logprob, *g_entropy;
    void *dx;
    int64_t ld, ldd;
    int n, vocab, t, chunks, per;       // CTAs of a row, units of each
};

// dx_v = sum_j g_j [v = tokens_j] - p_v (G + g_H (ln p_v + H)), G = sum_j g_j.
// A CTA writes the second term of `per` 16-byte units of a row, then the tokens
// among them with both terms.  kSame: logits and gradient have the same
// alignment.
template <class T, bool kSame>
__global__ void __launch_bounds__(kThreads) token_grad_kernel(GradArgs a) {
    constexpr int E = kUnit<T>;
    __shared__ float sg[kMaxTokens];
    __shared__ int stok[kMaxTokens];
    const int tid = threadIdx.x, r = blockIdx.x / a.chunks, c = blockIdx.x % a.chunks;
    const T *x = static_cast<const T *>(a.x) + (size_t)r * a.ld;
    T *dx = static_cast<T *>(a.dx) + (size_t)r * a.ldd;
    const Row<T> row(x, a.vocab);
    const int u0 = c * a.per, u1 = min(row.units(), u0 + a.per);
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
    auto soft = [&](float v) {
        const float lp = v - lse, p = exp2_fast(lp * kLog2e);
        float d = -G * p;
        if (a.g_entropy) d -= gh * (p * (lp + h));
        return v == neg_inf() ? 0.f : d;
    };
    for (int u = u0 + tid; u < u1; u += kThreads) {
        float v[E];
        unpack(row.load(u, from_float<T>(0.f)), v, T());
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

cudaError_t launch_logprobs(const ScoreArgs &a, jarq_dtype dtype, cudaStream_t s) {
    // few rows: several CTAs share one, as long as each has a few units a thread
    int split = 1;
    while (split < kMaxSplit && (int64_t)a.n * split < 2 * num_sms() &&
           (int64_t)a.vocab * (int64_t)size_of(dtype) / split > 2 * kThreads * 16)
        split *= 2;
    return with_type(dtype, [&](auto type) {
        using T = decltype(type);
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
        return a.k ? cudaLaunchKernelEx(&cfg, token_logprobs_kernel<T, true>, a)
                   : cudaLaunchKernelEx(&cfg, token_logprobs_kernel<T, false>, a);
    });
}

cudaError_t launch_grad(GradArgs a, jarq_dtype dtype, cudaStream_t s) {
    const size_t b = size_of(dtype);
    const int units = (int)(((size_t)a.vocab * b + 15) / 16 + 1);
    a.per = 4 * kThreads;
    a.chunks = (units + a.per - 1) / a.per;
    const int64_t grid = (int64_t)a.n * a.chunks;
    if (grid > 0x7FFFFFFF) return cudaErrorInvalidValue;
    const bool same = (((uintptr_t)a.x ^ (uintptr_t)a.dx) & 15) == 0 && (a.n == 1 || ((a.ld - a.ldd) * (int64_t)b) % 16 == 0);
    with_type(dtype, [&](auto type) {
        using T = decltype(type);
        if (same)
            token_grad_kernel<T, true><<<(unsigned)grid, kThreads, 0, s>>>(a);
        else
            token_grad_kernel<T, false><<<(unsigned)grid, kThreads, 0, s>>>(a);
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
    const cudaError_t e = launch_grad({logits, tokens, lse, entropy, g_logprob, g_entropy, dlogits, ld, ldd, n, vocab, t, 0, 0},
                                      dtype, st);
    ps.done();
    return finish(e);
}

}  // extern "C"
