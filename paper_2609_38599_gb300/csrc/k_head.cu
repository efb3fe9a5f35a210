// Softmax cross entropy of an output head over hidden states, and its gradient, in
// pieces of the vocabulary:
//   l = X W^T,  lse_r = ln sum_v exp l_rv,  loss_r = lse_r - l_r,token,
//   D_rv = g_r (exp(l_rv - lse_r) - [v = token_r]),  dX = D W,  dW = D^T X.
// The products run on the tensor cores (k_tc_head.cu); here are the join of the
// loss's parts, copies of rows that TMA cannot read, and the calls.
//
// D is formed for a piece of the vocabulary (512 MB), which both products then read: dX
// is added up over the pieces in float32, dW's rows belong to one piece.  A training
// step's loss and gradients of 8192 x 4096 -> 32000 in bfloat16 take 5.0 ms on the device: 8
// n V d operations at 1.7 PFLOP/s.  6 n V d would do if the loss kept its
// logits.  The copy of X without its ignored rows, for dW, takes 23 us of that, the
// join 9 to 11, what rounding took from dW (below) 47.
#include <limits.h>

#include <algorithm>

#include "head.cuh"
#include "integer.cuh"
#include "tc_common.cuh"

namespace jarq {
namespace head {
namespace {

using namespace rows;

constexpr int kPairs = 76;                  // of CTAs that run at one time
constexpr size_t kPieceBytes = 512u << 20;  // of D at a time
constexpr int kLeastPiece = 4096;           // but at least so many tokens
constexpr int kMostSplits = 16;             // of a sum over K
constexpr int kMostRows = 1 << 22, kMostWidth = 1 << 20, kMostVocab = 1 << 30;

// loss and lse of a row from the maxima m and sums s of its parts: with M the
// largest m and S = sum s exp(m - M), lse = M + ln S, and the loss is ln S + (M -
// logit), neither below 0: S has the largest term, 1, whose two approximate factors may
// make it less.  PER: threads of a row, over its parts.
template <int PER>
__global__ void __launch_bounds__(256) loss_join_kernel(const float2 *parts, int count, const float *target,
                                                        const int64_t *tokens, int n, int vocab, float *loss, float *lse) {
    constexpr int kRows = 256 / PER;
    __shared__ float2 all[PER][kRows + 1];
    tc::pdl_launch_dependents();
    tc::pdl_wait();
    const int i = threadIdx.x % kRows, t = threadIdx.x / kRows;
    const int r = blockIdx.x * kRows + i;
    float m = -INFINITY, s = 0.f;
    constexpr int kBatch = 8;
    auto take = [&](const float2 *p, int k) {
        float top = m;
        for (int j = 0; j < k; ++j) top = fmaxf(top, p[j].x);
        const float ref = top == -INFINITY ? 0.f : top;
        s *= expf(m - ref);
        for (int j = 0; j < k; ++j) s += p[j].y * expf(p[j].x - ref);
        m = top;
    };
    if (r < n)
        for (int p = t; p < count; p += kBatch * PER) {
            float2 v[kBatch];
#pragma unroll
            for (int j = 0; j < kBatch; ++j) v[j] = p + j * PER < count ? parts[(size_t)(p + j * PER) * n + r] : make_float2(-INFINITY, 0.f);
            take(v, kBatch);
        }
    all[t][i] = make_float2(m, s);
    for (int left = PER / 2; left; left /= 2) {
        __syncthreads();
        if (t < left) {
            take(&all[t + left][i], 1);
            all[t][i] = make_float2(m, s);
        }
    }
    if (t || r >= n) return;
    s = s < 1.f ? 1.f : s;                         // NaN stays; with M = -inf it counts for nothing
    const float logs = logf(s);
    if (lse) lse[r] = m + logs;
    if (loss) {
        const int64_t tok = tokens[r];
        float v = 0.f;
        if (tok >= vocab) v = __int_as_float(0x7FC00000);
        else if (tok >= 0) v = m == -INFINITY ? INFINITY + s : logs + (m - target[r]);
        loss[r] = v;
    }
}

// A byte of a token, to look for others of it.
__device__ __forceinline__ uint32_t mark_of(int64_t tok) { return (uint32_t)tok * 0x9E3779B1u >> 24; }

// 16-bit rows of any alignment to rows on 16-byte boundaries, pitch a multiple of 8.
// WEIGH: those of ignored tokens become zero, whatever they hold, and of float16
// row r is multiplied by 2^(e_r - top), as head.cuh has D's rows and row_tops_kernel `top`;
// and each row's token gets its mark, and every token's tally begins.
template <class T, bool WEIGH>
__global__ void __launch_bounds__(256) copy_rows_kernel(const T *x, int64_t ld, int n, int d, T *out, int pitch,
                                                        const int64_t *tokens, const float *g, const int *top, uint8_t *marks, int2 *tally, int vocab) {
    const int per = pitch / 8;
    const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
    const int64_t r = i / per;
    const int k = (int)(i % per) * 8;
    tc::pdl_launch_dependents();
    tc::pdl_wait();
    if constexpr (WEIGH)
        for (int64_t v = i; v < vocab; v += (int64_t)gridDim.x * 256) tally[v] = make_int2(0x7FFFFFFF, 0);
    if (r >= n) return;
    const T *p = x + r * ld + k;
    uint4 raw = make_uint4(0, 0, 0, 0);
    const bool live = !WEIGH || tokens[r] >= 0;
    if (WEIGH && k == 0) marks[r] = (uint8_t)mark_of(tokens[r]);
    if (live) {
        if (((uintptr_t)p & 15) == 0 && k + 8 <= d) {
            raw = *reinterpret_cast<const uint4 *>(p);
        } else {
            alignas(16) T t[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) t[e] = k + e < d ? p[e] : T(0.f);
            raw = *reinterpret_cast<const uint4 *>(t);
        }
        if constexpr (WEIGH && std::is_same_v<T, __half>) {
            const float by = ldexpf(1.f, exponent(g[r]) - *top);
            float v[8];
            unpack(raw, v, T());
#pragma unroll
            for (int e = 0; e < 8; ++e) v[e] *= by;
            raw = pack(v, T());
        }
    }
    *reinterpret_cast<uint4 *>(out + r * pitch + k) = raw;
}

// Float16's exponent of dW: rows of x are weighed by 2^(e_r - top), with which the largest
// |x_rk| 2^e_r of a row that counts lies in [2^14, 2^15).  An entry of x keeps its bits then
// unless |x_rk g_r| is 2^28 below the largest.  First what each block's rows have (a warp a
// row; what is not finite is left out), then their maximum.
// (With the largest e_r for top, whatever x, states of 0.002 with weights that differ by 2^10
// kept two to five bits.  8192 x 4096: 16 us and 3.)
constexpr int kTopBlocks = 1024;
__global__ void __launch_bounds__(256) row_tops_kernel(const __half *x, int64_t ld, int n, int d, const int64_t *tokens,
                                                       const float *g, int *tops) {
    __shared__ int part[8];
    int best = INT_MIN;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    tc::pdl_launch_dependents();
    tc::pdl_wait();
    for (int r = blockIdx.x * 8 + warp; r < n; r += 8 * gridDim.x) {
        if (tokens[r] < 0) continue;
        const Row<__half> row(x + r * ld, d);
        uint32_t top = 0;
        for (int u = lane; u < row.units(); u += 32) {
            const uint4 raw = row.load(u, __half(0.f));
            const uint32_t w[4] = {raw.x, raw.y, raw.z, raw.w};
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const uint32_t a = w[i] & 0x7FFF7FFFu;
                top = __vmaxu2(top, a & __vcmpltu2(a, 0x7C007C00u));
            }
        }
        top = __reduce_max_sync(0xffffffffu, max(top & 0xFFFFu, top >> 16));
        // |x| < 2^exponent; 2^-24 is the smallest that there is, and stands for a row of zeros
        const int most = max(-24, exponent(__half2float(__ushort_as_half((unsigned short)top))));
        best = max(best, exponent(g[r]) + most);
    }
    if (lane == 0) part[warp] = best;
    __syncthreads();
    if (warp == 0) {
        best = __reduce_max_sync(0xffffffffu, lane < 8 ? part[lane] : INT_MIN);
        if (lane == 0) tops[blockIdx.x] = best;
    }
}
__global__ void __launch_bounds__(kTopBlocks) top_exponent_kernel(const int *tops, int count, int *top) {
    __shared__ int part[32];
    tc::pdl_launch_dependents();
    tc::pdl_wait();
    int e = (int)threadIdx.x < count ? tops[threadIdx.x] : INT_MIN;
    e = __reduce_max_sync(0xffffffffu, e);
    if ((threadIdx.x & 31) == 0) part[threadIdx.x >> 5] = e;
    __syncthreads();
    if (threadIdx.x < 32) {
        e = __reduce_max_sync(0xffffffffu, part[threadIdx.x]);
        if (threadIdx.x == 0) *top = e == INT_MIN ? 0 : e - 15;            // no row counts: any
    }
}

// Every token's first row and number of rows, from {INT_MAX, 0}: whole numbers, the same
// in any order.
__global__ void __launch_bounds__(256) tally_kernel(const int64_t *tokens, int n, int vocab, int2 *tally) {
    const int r = blockIdx.x * 256 + threadIdx.x;
    tc::pdl_launch_dependents();
    tc::pdl_wait();
    if (r >= n) return;
    const int64_t tok = tokens[r];
    if (tok < 0 || tok >= vocab) return;
    atomicMin(&tally[tok].x, r);
    atomicAdd(&tally[tok].y, 1);
}

// What dW lacks of D's entries of the tokens first .. first + window - 1 that have several
// rows (of one row, dW's product takes it from there): for each the sum of lost_t x_t
// over its rows t, in their order, at its first row.  No atomics: the same bits every time.
// x: rows as dW's product reads them.
// A block, of 8 rows and 512 columns, takes those that are a token's first in turn: it looks
// through the rows from there by a byte of each, 4096 at a time, until it has all of the
// token's, and four groups of its threads add them up, every fourth row each.
// 8192 rows of 4096 with any of 32000 tokens 44 us.  Such a gradient without this and with
// it: 3.30 and 3.39 ms, its most frequent token in 610 rows 3.5 to 3.7 and 3.7 to 3.8, one
// token in all rows 3.3 and 4.4 (they go through 8 blocks), 100000 x 512 -> 32000, in eight pieces, 7.2 and 8.2.
// On the way: every row's block through all tokens, 8 bytes each, sums in memory 137 us
// (one token in all rows 13.4 ms); eight tokens a thread at a time 77; a byte each but
// every row's block and sixteen rows in flight 175 (two blocks an SM); a block a row
// and 2048 columns 27, but one token in all rows 6.2 ms.
template <class T>
__global__ void __launch_bounds__(256) lost_rows_kernel(const int64_t *tokens, const int2 *tally, const uint8_t *marks,
                                                        const float *lost, const T *x, int n, int d, int pitch, int first,
                                                        int window, float *rest) {
    constexpr int kSpan = 4096, kBatch = 8, kGroups = 4;
    __shared__ int row_of[kSpan];
    __shared__ int counts[8];
    __shared__ float parts[kGroups - 1][64][9];
    tc::pdl_launch_dependents();
    tc::pdl_wait();
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, unit = threadIdx.x & 63, group = threadIdx.x >> 6;
    const int k = (blockIdx.y * 64 + unit) * 8;
    // lanes 0 .. 7 of every warp have the block's rows
    const int own_row = blockIdx.x * 8 + lane;
    int64_t own_tok = -1;
    int rows = 0;
    if (lane < 8 && own_row < n) own_tok = tokens[own_row];
    if (own_tok >= first && own_tok < (int64_t)first + window) {
        const int2 all = tally[own_tok];
        if (all.x == own_row) rows = all.y;
    }
    for (uint32_t todo = __ballot_sync(0xffffffffu, rows > 1); todo; todo &= todo - 1) {
        const int from = __ffs(todo) - 1, t = blockIdx.x * 8 + from;
        const int64_t tok = __shfl_sync(0xffffffffu, own_tok, from);
        const int most = __shfl_sync(0xffffffffu, rows, from);
        const uint32_t mark = mark_of(tok) * 0x01010101u;
        float sum[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) sum[e] = 0.f;
        int had = 0;
        for (int i = t & ~(kSpan - 1); i < n && had < most; i += kSpan) {
            // this thread's 16 rows; marks past n are read up to the next 16 and not taken
            const int r0 = i + 16 * threadIdx.x;
            uint32_t mine = 0;
            if (r0 < n) {
                const uint4 m = *reinterpret_cast<const uint4 *>(marks + r0);
                const uint32_t w[4] = {m.x, m.y, m.z, m.w};
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    uint32_t hits = __vcmpeq4(w[j], mark) & 0x08040201u;
                    hits |= hits >> 16;
                    mine |= ((hits | hits >> 8) & 15u) << (4 * j);
                }
                for (uint32_t left = mine; left; left &= left - 1) {
                    const int e = __ffs(left) - 1;
                    if (r0 + e >= n || tokens[r0 + e] != tok) mine &= ~(1u << e);
                }
            }
            // their places, in the rows' order
            const int own = __popc(mine);
            int upto = own;
#pragma unroll
            for (int off = 1; off < 32; off *= 2) {
                const int v = __shfl_up_sync(0xffffffffu, upto, off);
                if (lane >= off) upto += v;
            }
            if (lane == 31) counts[warp] = upto;
            __syncthreads();
            int at = upto - own, total = 0;
#pragma unroll
            for (int w = 0; w < 8; ++w) {
                if (w < warp) at += counts[w];
                total += counts[w];
            }
            for (uint32_t left = mine; left; left &= left - 1, ++at) row_of[at] = r0 + __ffs(left) - 1;
            had += total;
            __syncthreads();
            if (k < d)
                for (int j0 = group; j0 < total; j0 += kGroups * kBatch) {
                    uint4 raw[kBatch];
                    float by[kBatch];
#pragma unroll
                    for (int j = 0; j < kBatch; ++j) {
                        const int at_j = j0 + kGroups * j, r = row_of[min(at_j, total - 1)];
                        raw[j] = *reinterpret_cast<const uint4 *>(x + (size_t)r * pitch + k);
                        by[j] = at_j < total ? lost[r] : 0.f;
                    }
#pragma unroll
                    for (int j = 0; j < kBatch; ++j) {
                        float v[8];
                        unpack(raw[j], v, T());
                        // what is not finite has had its effect in the product
#pragma unroll
                        for (int e = 0; e < 8; ++e) sum[e] += fabsf(v[e]) < INFINITY ? by[j] * v[e] : 0.f;
                    }
                }
            __syncthreads();
        }
        if (group)
#pragma unroll
            for (int e = 0; e < 8; ++e) parts[group - 1][unit][e] = sum[e];
        __syncthreads();
        if (group == 0 && k < d) {
#pragma unroll
            for (int g = 0; g < kGroups - 1; ++g)
#pragma unroll
                for (int e = 0; e < 8; ++e) sum[e] += parts[g][unit][e];
            float4 *to = reinterpret_cast<float4 *>(rest + (size_t)t * pitch + k);
            to[0] = make_float4(sum[0], sum[1], sum[2], sum[3]);
            to[1] = make_float4(sum[4], sum[5], sum[6], sum[7]);
        }
        __syncthreads();
    }
}

// The splits' sums, added in their order, scaled and rounded.
template <class T>
__global__ void __launch_bounds__(256) sum_splits_kernel(const float *slab, int splits, int n, int d, int pitch, T *out,
                                                         int64_t ld, const float *g, const int *top) {
    const int per = pitch / 4;
    const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
    tc::pdl_launch_dependents();
    tc::pdl_wait();
    const int64_t r = i / per;
    const int k = (int)(i % per) * 4;
    if (r >= n || k >= d) return;
    float4 y = *reinterpret_cast<const float4 *>(slab + r * pitch + k);
    for (int s = 1; s < splits; ++s) {
        const float4 o = *reinterpret_cast<const float4 *>(slab + ((int64_t)s * n + r) * pitch + k);
        y.x += o.x, y.y += o.y, y.z += o.z, y.w += o.w;
    }
    float by = 1.f;
    if (std::is_same_v<T, __half>) by = ldexpf(1.f, (g ? exponent(g[r]) : *top) - 14);
    const float v[4] = {y.x * by, y.y * by, y.z * by, y.w * by};
#pragma unroll
    for (int e = 0; e < 4; ++e)
        if (k + e < d) out[r * ld + k + e] = from_float<T>(v[e]);
}

template <class T>
__global__ void __launch_bounds__(256) zero_rows_kernel(T *out, int64_t ld, int n, int d) {
    const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (i / d < n) out[i / d * ld + i % d] = T(0.f);
}

int ceil_div(int64_t a, int64_t b) { return (int)((a + b - 1) / b); }

// A product's tiles: columns and splits of K that take the least time. Waves of pairs,
// each so many chunks of K at a time that goes with the columns (64 of them stand for the
// rows' operand and what a tile costs besides), and with splits their float32 sums through memory.
struct Tiles {
    int cols = 256, splits = 1;
    Tiles(int m, int n, int chunks, int most_splits) {
        double best = 0;
        for (int c = 256; c >= 32; c -= 32)
            for (int s = 1; s <= std::min(most_splits, std::max(1, chunks / 8)); ++s) {
                const int per = ceil_div(chunks, s), real = ceil_div(chunks, per);
                const int64_t tiles = (int64_t)ceil_div(m, 256) * ceil_div(n, c) * real;
                // two cycles a column and chunk; some 3500 bytes a cycle from memory
                const double t = (double)((tiles + kPairs - 1) / kPairs) * per * (c + 64) +
                                 (real > 1 ? 8.0 * real * m * n / 3500 / 2 : 0);
                if (best == 0 || t < best) {
                    best = t;
                    cols = c;
                    splits = real;
                }
            }
    }
};

// The parts of a workspace, each on a 256-byte boundary.
struct Layout {
    size_t bytes = 0;
    size_t take(size_t n) {
        const size_t at = bytes;
        bytes += (n + 255) / 256 * 256;
        return at;
    }
};

struct Plan {
    int pitch, pieces, width;            // of copies and sums; pieces of the vocabulary
    int split_x, split_w;
    bool slab_x, slab_w;
    size_t copy_x, copy_w, parts, target, weighed, top, D, sums_x, sums_w, lost, tally, rest, marks, bytes;

    // the loss
    Plan(int n, int d, int vocab, bool aligned) : pitch(round_up(d, 8)) {
        Layout l;
        parts = l.take((size_t)2 * ceil_div(vocab, Tiles(n, vocab, ceil_div(d, 64), 1).cols) * n * sizeof(float2));
        target = l.take((size_t)n * sizeof(float));
        copies(l, n, vocab, aligned);
        bytes = l.bytes;
    }
    // its gradient
    Plan(int n, int d, int vocab, bool aligned, bool hidden, bool head) : pitch(round_up(d, 8)) {
        const int64_t most = std::max<int64_t>(kLeastPiece, (int64_t)(kPieceBytes / 2 / std::max(n, 1)) / 256 * 256);
        const int even = ceil_div(vocab, ceil_div(vocab, most));
        width = round_up(even, 256);
        pieces = ceil_div(vocab, width);
        split_x = Tiles(n, d, ceil_div(std::min(width, vocab), 64), kMostSplits).splits;
        split_w = Tiles(std::min(width, vocab), d, ceil_div(n, 64), kMostSplits).splits;
        slab_x = hidden && (split_x > 1 || pieces > 1);
        slab_w = head && split_w > 1;
        Layout l;
        D = l.take((size_t)n * width * 2);
        sums_x = l.take(slab_x ? (size_t)split_x * n * pitch * sizeof(float) : 0);
        sums_w = l.take(slab_w ? (size_t)split_w * width * pitch * sizeof(float) : 0);
        weighed = l.take(head ? (size_t)n * pitch * 2 : 0);
        top = l.take((1 + kTopBlocks) * sizeof(int));
        lost = l.take((size_t)n * sizeof(float));
        tally = l.take(head ? (size_t)vocab * sizeof(int2) : 0);
        marks = l.take(head ? (size_t)round_up(n, 16) : 0);
        rest = l.take(head ? (size_t)n * pitch * sizeof(float) : 0);
        copies(l, n, vocab, aligned);
        bytes = l.bytes;
    }
    void copies(Layout &l, int n, int vocab, bool aligned) {
        copy_x = l.take(aligned ? 0 : (size_t)n * pitch * 2);
        copy_w = l.take(aligned ? 0 : (size_t)vocab * pitch * 2);
    }
};

bool is_aligned(const void *p, size_t b) { return ((uintptr_t)p & (b - 1)) == 0; }
bool rows_aligned(const void *p, int64_t ld, int n) { return is_aligned(p, 16) && (n == 1 || ld % 8 == 0); }
bool usable(const void *p, size_t size) { return p && on_device(p) && is_aligned(p, size); }

// A 16-bit matrix with rows on 16-byte boundaries.
struct Matrix {
    const char *p;
    int64_t ld;
    const char *row(int64_t r) const { return p + r * ld * 2; }
};
// boxes of `box` rows x 64 elements, moved as they are whatever the type
cudaError_t tensor_map(CUtensorMap *map, const char *p, int rows, int cols, int64_t ld, int box) {
    return make_tmap_half(map, p, rows, cols, rows > 1 ? ld : round_up(cols, 8), box);
}

// A call's arguments and the launches that it makes, one after the other: each but the
// first may start while the one before it ends, and waits for it before it reads.
struct Call {
    jarq_dtype dtype;
    int n, d, vocab;
    const int64_t *tokens;
    char *work;
    cudaStream_t s;
    int *failed;
    int launches = 0;

    template <class F>
    cudaError_t typed(F f) {
        return dtype == JARQ_F16 ? f(__half()) : f(__nv_bfloat16());
    }
    template <class... KArgs, class... Args>
    cudaError_t run(void (*kernel)(KArgs...), int64_t blocks, int threads, Args... args) {
        return launch_k(kernel, dim3((unsigned)blocks), dim3(threads), 0, s, launches++ > 0, args...);
    }
    cudaError_t copy(const void *x, int64_t ld, int rows, char *out, int pitch) {
        return typed([&](auto type) {
            using T = decltype(type);
            return run(copy_rows_kernel<T, false>, ceil_div((int64_t)rows * (pitch / 8), 256), 256, static_cast<const T *>(x), ld,
                       rows, d, reinterpret_cast<T *>(out), pitch, (const int64_t *)nullptr, (const float *)nullptr,
                       (const int *)nullptr, (uint8_t *)nullptr, (int2 *)nullptr, 0);
        });
    }
    cudaError_t weigh(const void *x, int64_t ld, char *out, int pitch, const float *g, const int *top, uint8_t *marks, int2 *tally) {
        return typed([&](auto type) {
            using T = decltype(type);
            return run(copy_rows_kernel<T, true>, ceil_div((int64_t)n * (pitch / 8), 256), 256, static_cast<const T *>(x), ld, n, d,
                       reinterpret_cast<T *>(out), pitch, tokens, g, top, marks, tally, vocab);
        });
    }
    cudaError_t lost_rows(const int2 *tally, const uint8_t *marks, const float *lost, const char *x, int pitch, int first, int window,
                          float *rest) {
        return typed([&](auto type) {
            using T = decltype(type);
            return launch_k(lost_rows_kernel<T>, dim3(ceil_div(n, 8), ceil_div(d, 512)), dim3(256), 0, s, launches++ > 0, tokens, tally, marks,
                            lost, reinterpret_cast<const T *>(x), n, d, pitch, first, window, rest);
        });
    }
    cudaError_t sum_splits(const float *slab, int splits, int rows, int pitch, void *out, int64_t ld, const float *g,
                           const int *top) {
        return typed([&](auto type) {
            using T = decltype(type);
            return run(sum_splits_kernel<T>, ceil_div((int64_t)rows * (pitch / 4), 256), 256, slab, splits, rows, d, pitch,
                       static_cast<T *>(out), ld, g, top);
        });
    }
    // the rows of x as TMA can read them: themselves, or a copy of them
    cudaError_t readable(const void *x, int64_t ld, int rows, char *room, int pitch, Matrix *m) {
        *m = {static_cast<const char *>(x), ld};
        if (rows_aligned(x, ld, rows)) return cudaSuccess;
        *m = {room, pitch};
        return copy(x, ld, rows, room, pitch);
    }
    ProductArgs shape(int m, int cols, int k, int most_splits) const {
        const Tiles tile(m, cols, ceil_div(k, 64), most_splits);
        ProductArgs a{};
        a.m = m, a.n = cols;
        a.chunks = ceil_div(k, 64);
        a.splits = tile.splits;
        a.per = ceil_div(a.chunks, a.splits);
        a.cols = tile.cols;
        a.rows = m < 128 ? round_up(m, 8) : 128;
        a.mt = ceil_div(m, 256), a.nt = ceil_div(cols, a.cols);
        a.half = dtype == JARQ_F16;
        a.tokens = tokens, a.vocab = vocab;
        a.last = true;
        a.failed = failed;
        return a;
    }
    cudaError_t product(Product which, const CUtensorMap &a, const CUtensorMap &b, const ProductArgs &args) {
        return launch_product(which, a, b, args, s, launches++ > 0);
    }
};

#define TRY(x)                                                  \
    do {                                                        \
        if (const cudaError_t e_ = (x); e_ != cudaSuccess) return e_; \
    } while (0)

cudaError_t run_loss(Call &c, const void *X, int64_t ldx, const void *W, int64_t ldw, const Plan &p, float *loss, float *lse) {
    Matrix x, w;
    TRY(c.readable(X, ldx, c.n, c.work + p.copy_x, p.pitch, &x));
    TRY(c.readable(W, ldw, c.vocab, c.work + p.copy_w, p.pitch, &w));
    CUtensorMap mx, mw;
    ProductArgs a = c.shape(c.n, c.vocab, c.d, 1);
    TRY(tensor_map(&mx, x.p, c.n, c.d, x.ld, a.rows));
    TRY(tensor_map(&mw, w.p, c.vocab, c.d, w.ld, a.cols / 2));
    a.part = reinterpret_cast<float2 *>(c.work + p.parts);
    a.target = reinterpret_cast<float *>(c.work + p.target);
    TRY(c.product(kLoss, mx, mw, a));
    // 32 threads a row (8192 rows of 250 parts: 21 us by 8); few rows: 64
    auto join = [&](auto *kernel, int per) {
        return c.run(kernel, ceil_div(c.n, 256 / per), 256, (const float2 *)a.part, 2 * a.nt, (const float *)a.target, c.tokens,
                     c.n, c.vocab, loss, lse);
    };
    return c.n < kPairs ? join(loss_join_kernel<64>, 64) : join(loss_join_kernel<32>, 32);
}

cudaError_t run_grad(Call &c, const void *X, int64_t ldx, const void *W, int64_t ldw, const Plan &p, const float *lse,
                     const float *g, void *dX, int64_t lddx, void *dW, int64_t lddw) {
    Matrix x, w;
    TRY(c.readable(X, ldx, c.n, c.work + p.copy_x, p.pitch, &x));
    TRY(c.readable(W, ldw, c.vocab, c.work + p.copy_w, p.pitch, &w));
    int *top = reinterpret_cast<int *>(c.work + p.top);
    uint8_t *marks = reinterpret_cast<uint8_t *>(c.work + p.marks);
    int2 *tally = reinterpret_cast<int2 *>(c.work + p.tally);
    CUtensorMap mx, mw, md, mb;
    if (dW) {
        if (c.dtype == JARQ_F16) {
            const int blocks = std::min(kTopBlocks, ceil_div(c.n, 8));
            TRY(c.run(row_tops_kernel, blocks, 256, static_cast<const __half *>(X), ldx, c.n, c.d, c.tokens, g, top + 1));
            TRY(c.run(top_exponent_kernel, 1, kTopBlocks, (const int *)(top + 1), blocks, top));
        }
        TRY(c.weigh(X, ldx, c.work + p.weighed, p.pitch, g, top, marks, tally));
        TRY(c.run(tally_kernel, ceil_div(c.n, 256), 256, c.tokens, c.n, c.vocab, tally));
    }
    char *D = c.work + p.D;
    float *sums_x = p.slab_x ? reinterpret_cast<float *>(c.work + p.sums_x) : nullptr;
    float *sums_w = p.slab_w ? reinterpret_cast<float *>(c.work + p.sums_w) : nullptr;
    int sums = 1;                                    // splits of dX
    float *lost = reinterpret_cast<float *>(c.work + p.lost), *rest = reinterpret_cast<float *>(c.work + p.rest);
    for (int i = 0; i < p.pieces; ++i) {
        const int v0 = i * p.width, width = std::min(p.width, c.vocab - v0);
        {
            ProductArgs a = c.shape(c.n, width, c.d, 1);
            TRY(tensor_map(&mx, x.p, c.n, c.d, x.ld, a.rows));
            TRY(tensor_map(&mw, w.row(v0), width, c.d, w.ld, a.cols / 2));
            a.lse = lse, a.g = g, a.first = v0;
            a.out = D, a.ldo = p.width;
            a.lost = lost;
            TRY(c.product(kLogits, mx, mw, a));
        }
        if (dX) {
            ProductArgs a = c.shape(c.n, c.d, width, i == 0 ? p.split_x : sums);
            TRY(tensor_map(&md, D, c.n, width, p.width, a.rows));
            TRY(tensor_map(&mb, w.row(v0), width, c.d, w.ld, 64));
            if (i == 0) sums = a.splits;             // a shorter piece may have fewer
            a.g = g;
            a.out = dX, a.ldo = lddx;
            a.slab = sums_x, a.pitch = p.pitch;
            a.add = i > 0;
            a.lost = lost, a.first = v0, a.window = width;
            a.w = reinterpret_cast<const uint16_t *>(w.row(v0)), a.ldw = w.ld;
            a.last = sums == 1 && i + 1 == p.pieces;
            TRY(c.product(kHidden, md, mb, a));
        }
        if (dW) {
            void *out = static_cast<char *>(dW) + (int64_t)v0 * lddw * 2;
            TRY(tensor_map(&md, D, c.n, width, p.width, 64));
            TRY(tensor_map(&mb, c.work + p.weighed, c.n, c.d, p.pitch, 64));
            ProductArgs a = c.shape(width, c.d, c.n, p.split_w);
            a.out = out, a.ldo = lddw;
            a.slab = sums_w, a.pitch = p.pitch;
            a.last = !p.slab_w;
            a.top = top;
            a.first = v0;
            a.tally = tally + v0, a.rest = rest, a.rest_pitch = p.pitch;
            a.lost = lost, a.w = reinterpret_cast<const uint16_t *>(c.work + p.weighed), a.ldw = p.pitch;
            TRY(c.lost_rows(tally, marks, lost, c.work + p.weighed, p.pitch, v0, width, rest));
            TRY(c.product(kHead, md, mb, a));
            if (p.slab_w) TRY(c.sum_splits(sums_w, a.splits, width, p.pitch, out, lddw, nullptr, top));
        }
    }
    if (dX && sums > 1) TRY(c.sum_splits(sums_x, sums, c.n, p.pitch, dX, lddx, g, nullptr));
    return cudaSuccess;
}

jarq_status check(const void *X, jarq_dtype dtype, int n, int d, int64_t ldx, const void *W, int vocab, int64_t ldw,
                  const int64_t *tokens) {
    if ((dtype != JARQ_F16 && dtype != JARQ_BF16) || n < 0 || n > kMostRows || d < 1 || d > kMostWidth || vocab < 1 ||
        vocab > kMostVocab || ldx < d || ldw < d)
        return JARQ_ERR_ARG;
    if (n == 0) return JARQ_OK;
    if (!usable(X, 2) || !usable(W, 2) || !usable(tokens, 8)) return JARQ_ERR_ARG;
    return JARQ_OK;
}

jarq_status finish(cudaError_t e, int launches) {
    count_launches(launches);
    if (e == cudaSuccess) return JARQ_OK;
    (void)cudaGetLastError();
    return JARQ_ERR_CUDA;
}

// More tiles than pairs, so that some have a second one, which is never summed.
constexpr int kStalledRows = 2048, kStalledTokens = 4096, kStalledWidth = 256;

}  // namespace

size_t stalled_bytes() {
    return (size_t)(kStalledRows + kStalledTokens) * kStalledWidth * 2 + kStalledRows * (sizeof(int64_t) + sizeof(float)) +
           (size_t)2 * (kStalledTokens / 32) * kStalledRows * sizeof(float2);
}
cudaError_t launch_stalled(char *zeros, int *failed, cudaStream_t s) {
    char *w = zeros + (size_t)kStalledRows * kStalledWidth * 2, *rest = w + (size_t)kStalledTokens * kStalledWidth * 2;
    Call c{JARQ_F16, kStalledRows, kStalledWidth, kStalledTokens, reinterpret_cast<const int64_t *>(rest), zeros, s, failed};
    ProductArgs a = c.shape(c.n, c.vocab, c.d, 1);
    a.part = reinterpret_cast<float2 *>(rest + kStalledRows * sizeof(int64_t));
    a.target = reinterpret_cast<float *>(a.part + (size_t)2 * a.nt * c.n);
    CUtensorMap mx, mw;
    TRY(tensor_map(&mx, zeros, c.n, c.d, c.d, a.rows));
    TRY(tensor_map(&mw, w, c.vocab, c.d, c.d, a.cols / 2));
    return launch_product(kLoss, mx, mw, a, s, false, true);
}

}  // namespace head
}  // namespace jarq

using namespace jarq;
using namespace jarq::head;

extern "C" {

size_t jarq_cross_entropy_workspace(int n, int d, int vocab, int rows_aligned) {
    if (n < 1 || n > kMostRows || d < 1 || d > kMostWidth || vocab < 1 || vocab > kMostVocab) return 0;
    return Plan(n, d, vocab, rows_aligned != 0).bytes;
}

jarq_status jarq_cross_entropy(const void *X, jarq_dtype dtype, int n, int d, int64_t ldx, const void *W,
                               int vocab, int64_t ldw, const int64_t *tokens, float *loss, float *lse,
                               void *workspace, size_t workspace_bytes, void *stream) {
    const jarq_status ok = check(X, dtype, n, d, ldx, W, vocab, ldw, tokens);
    if (ok != JARQ_OK || n == 0) return ok;
    if (!usable(loss, 4) || (lse && !usable(lse, 4))) return JARQ_ERR_ARG;
    const Plan plan(n, d, vocab, rows_aligned(X, ldx, n) && rows_aligned(W, ldw, vocab));
    if (!usable(workspace, 16) || workspace_bytes < plan.bytes) return JARQ_ERR_ARG;
    if (const jarq_status late = async_failure()) return late;
    Call c{dtype, n, d, vocab, tokens, static_cast<char *>(workspace), (cudaStream_t)stream, async_word()};
    if (!c.failed) return JARQ_ERR_NOMEM;
    ProfScope ps("cross_entropy", c.s);
    const cudaError_t e = run_loss(c, X, ldx, W, ldw, plan, loss, lse);
    ps.done();
    return finish(e, c.launches);
}

size_t jarq_cross_entropy_grad_workspace(int n, int d, int vocab, int rows_aligned, int hidden, int head) {
    if (n < 1 || n > kMostRows || d < 1 || d > kMostWidth || vocab < 1 || vocab > kMostVocab) return 0;
    return Plan(n, d, vocab, rows_aligned != 0, hidden != 0, head != 0).bytes;
}

jarq_status jarq_cross_entropy_grad(const void *X, jarq_dtype dtype, int n, int d, int64_t ldx, const void *W,
                                    int vocab, int64_t ldw, const int64_t *tokens, const float *lse,
                                    const float *g_loss, void *dX, int64_t lddx, void *dW, int64_t lddw,
                                    void *workspace, size_t workspace_bytes, void *stream) {
    const jarq_status ok = check(X, dtype, n, d, ldx, W, vocab, ldw, tokens);
    if (ok != JARQ_OK || (!dX && !dW) || (dX && lddx < d) || (dW && lddw < d)) return JARQ_ERR_ARG;
    cudaStream_t st = (cudaStream_t)stream;
    if (n == 0) {
        // no rows: no gradient reaches the head
        if (!dW) return JARQ_OK;
        if (!usable(dW, 2)) return JARQ_ERR_ARG;
        const int64_t blocks = ((int64_t)vocab * d + 255) / 256;
        if (blocks > 0x7FFFFFFF) return JARQ_ERR_ARG;
        if (const jarq_status late = async_failure()) return late;
        zero_rows_kernel<<<(unsigned)blocks, 256, 0, st>>>(static_cast<__half *>(dW), lddw, vocab, d);
        return finish(cudaGetLastError(), 1);
    }
    if (!usable(lse, 4) || !usable(g_loss, 4) || (dX && !usable(dX, 2)) || (dW && !usable(dW, 2))) return JARQ_ERR_ARG;
    const Plan plan(n, d, vocab, rows_aligned(X, ldx, n) && rows_aligned(W, ldw, vocab), dX != nullptr, dW != nullptr);
    if (!usable(workspace, 16) || workspace_bytes < plan.bytes) return JARQ_ERR_ARG;
    if (const jarq_status late = async_failure()) return late;
    Call c{dtype, n, d, vocab, tokens, static_cast<char *>(workspace), st, async_word()};
    if (!c.failed) return JARQ_ERR_NOMEM;
    ProfScope ps("cross_entropy_grad", st);
    const cudaError_t e = run_grad(c, X, ldx, W, ldw, plan, lse, g_loss, dX, lddx, dW, lddw);
    ps.done();
    return finish(e, c.launches);
}

}  // extern "C"
