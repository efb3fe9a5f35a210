// Product of 8-bit integers with scales for each token and channel:
//   Y[t][o] = xs[t] sum_i ws[o][i] (sum_{k in group i} X[t][k] C[o][k]) + bias[o].
//
// One or two tokens: integer dot products of four, bound by reading the weights
// once.  A block goes from one set of R channels to the next; its threads share K,
// 16 codes of each channel at a time with 16 codes of each token, the next weights,
// of these channels or the following ones, on their way while these are used and
// their sums joined.  With one scale a channel the sums are int32 (exact for din <=
// 65536); with groups the 4 or 8 lanes that share one add up its integer sum, which is
// so exact, and share out the scaling into float32 sums.  A linear layer's single token
// is quantized by every block for itself, under its first weights' loads.  One token,
// 4096 -> 11008 (45 MB), quantization included: 10.0 us from cold memory (4.5 TB/s),
// 7.3 us from L2, with groups of 128 10.4 and 7.8; 4096 -> 4096 5.9 and 4.7 us.  11008 ->
// 4096 with groups of 128: one token 12.9 and 8.7, two 14.8 and 10.2.  (Each product of
// 16 scaled by its own lane, which rounds the parts of a group's sum and loads a scale
// for each: 14.1 and 10.7, 16.5 and 12.3.)
#include "integer.cuh"
#include "quantize.cuh"
#include "rows.cuh"
#include "tc_common.cuh"

namespace jarq {
namespace {

using namespace rows;

constexpr int kThreads = 256, kWarps = kThreads / 32;
// Longest row that a single token's blocks quantize for themselves (from a graph,
// cold and warm, against a launch of its own: 4096 -> 11008 10.1 and 7.3 us, 11.1 and
// 7.0, with groups of 128 10.5 and 7.8, 11.9 and 7.7; 6144 -> 8192 12.4 and 8.1, 14.5
// and 8.0; 8192 -> 4096 9.5 and 7.3, 9.7 and 6.3; 11008 -> 4096, groups of 128, 12.6 and
// 9.9, 12.7 and 8.5).  The host's time of a call falls by 4 us of 18.  Two tokens'
// blocks would lose (2 x 4096 -> 1000: 4.6 us for 3.6).
constexpr int kOwnCodes = 6144;

// A group's 16-code chunks lie with LANES neighbouring lanes (4 or 8), which share
// its V integer sums out: a lane has kOwn of them from first() on, and where there
// are more lanes than sums, kSame lanes have the same one.
template <int V, int LANES>
struct Share {
    static constexpr int kOwn = V > LANES ? V / LANES : 1, kSame = V < LANES ? LANES / V : 1;
    __device__ static int first(int lane) { return lane % LANES / kSame * kOwn; }
    // v[i]: this lane's part of sum i; afterwards v[0 .. kOwn - 1] are its own sums
    __device__ static void join(int (&v)[V], int lane) {
        int left = V;
#pragma unroll
        for (int off = LANES / 2; off > 0; off /= 2) {
            if (left > 1) {
                left /= 2;
                const bool up = lane & off;
#pragma unroll
                for (int i = 0; i < V / 2; ++i)
                    if (i < left) {
                        const int give = up ? v[i] : v[i + left], keep = up ? v[i + left] : v[i];
                        v[i] = keep + __shfl_xor_sync(0xffffffffu, give, off);
                    }
            } else {
                v[0] += __shfl_xor_sync(0xffffffffu, v[0], off);
            }
        }
    }
};

// A row of activations to codes q in shared memory, by a block; its scale.
template <class T>
__device__ __forceinline__ float quantize_row(const T *x, int d, int8_t *q, uint32_t (&part)[kWarps]) {
    const Row<T> row(x, d);
    const int units = row.units();
    quant::Largest<T> largest;
    for (int u = threadIdx.x; u < units; u += kThreads) largest.take(row.load(u, T(0.f)));
    uint32_t top = __reduce_max_sync(0xffffffffu, largest.bits());
    if ((threadIdx.x & 31) == 0) part[threadIdx.x >> 5] = top;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < kWarps; ++w) top = max(top, part[w]);
    const quant::RowScale by(top);
    for (int u = threadIdx.x; u < units; u += kThreads) quant::put_codes(row, u, row.load(u, T(0.f)), by, q);
    __syncthreads();
    return by.scale;
}

// M: tokens (a.n <= M); R: channels that a block has at a time.  LANES: 16-code
// chunks of a group, 0 for one scale a channel.  OWN: the token is activations of
// type `xtype`, which each block quantizes for itself.
template <int M, int R, int LANES, bool VEC, bool OWN>
__global__ void __launch_bounds__(kThreads, M == 1 ? 4 : 2) few_tokens_kernel(ProductArgs a, jarq_dtype xtype) {
    constexpr int V = M * R;
    constexpr bool GROUPS = LANES > 0;
    using Mine = Share<V, GROUPS ? LANES : 1>;
    // scales of a lane: of the channels whose sums it has
    constexpr int kScales = GROUPS ? Mine::kOwn / M : 1;
    static_assert(!GROUPS || Mine::kOwn % M == 0, "all tokens of a channel");
    __shared__ uint32_t parts[2][kWarps][V];
    __shared__ uint32_t tops[kWarps];
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const int chunks = (a.din + 15) / 16, step = gridDim.x * R;
    uint4 w[R];
    auto fetch = [&](int r, int o, int c) {
        if (o < a.dout && c < chunks) w[r] = load_codes<VEC>(a.C + (size_t)o * a.ldc, 16 * c, a.din);
    };
    // and the groups' scales of the lane's sums, on their way with them
    float ws[kScales];
    const int first = GROUPS ? Mine::first(lane) : 0;
    auto fetch_scales = [&](int o, int c) {
        if (!GROUPS || c >= chunks) return;
#pragma unroll
        for (int i = 0; i < kScales; ++i)
            if (const int oi = o + first / M + i; oi < a.dout) ws[i] = a.ws[(size_t)oi * a.G + c / (GROUPS ? LANES : 1)];
    };
#pragma unroll
    for (int r = 0; r < R; ++r) w[r] = make_uint4(0, 0, 0, 0);
#pragma unroll
    for (int i = 0; i < kScales; ++i) ws[i] = 0.f;
#pragma unroll
    for (int r = 0; r < R; ++r) fetch(r, blockIdx.x * R + r, tid);
    fetch_scales(blockIdx.x * R, tid);
    extern __shared__ __align__(16) int8_t own[];
    const int8_t *X = static_cast<const int8_t *>(a.X);
    float scale[M];
    static_assert(M == 1 || !OWN, "one token");
    if constexpr (OWN) {
        X = own;
        with_type_device(xtype, [&](auto type) {
            using T = decltype(type);
            scale[0] = quantize_row(static_cast<const T *>(a.X), a.din, own, tops);
        });
    } else {
        // the tokens' codes may be the previous kernel's
        tc::pdl_wait();
#pragma unroll
        for (int m = 0; m < M; ++m) scale[m] = a.xs[min(m, a.n - 1)];
    }
    for (int o0 = blockIdx.x * R, turn = 0; o0 < a.dout; o0 += step, turn ^= 1) {
        int sum[V] = {};
        float acc[Mine::kOwn] = {};
        // with groups a warp goes on together, lanes past the row with nothing
        for (int c = tid; (GROUPS ? c - lane : c) < chunks; c += kThreads) {
            // the next weights: of these channels, else of the block's next ones,
            // which are then on their way under the sums' reduction
            const bool live = !GROUPS || c < chunks, more = c + kThreads < chunks;
            const int on = more ? o0 : o0 + step, cn = live ? more ? c + kThreads : tid : chunks;
            uint4 x[M];
#pragma unroll
            for (int m = 0; m < M; ++m)
                x[m] = load_codes<VEC || OWN>(X + min(m, a.n - 1) * (size_t)a.ldx, 16 * c, a.din);
            int group[V];
#pragma unroll
            for (int r = 0; r < R; ++r) {
                const uint4 wr = w[r];
                fetch(r, on + r, cn);
#pragma unroll
                for (int m = 0; m < M; ++m) {
                    int d = GROUPS ? 0 : sum[r * M + m];
                    d = __dp4a((int)wr.x, (int)x[m].x, d);
                    d = __dp4a((int)wr.y, (int)x[m].y, d);
                    d = __dp4a((int)wr.z, (int)x[m].z, d);
                    d = __dp4a((int)wr.w, (int)x[m].w, d);
                    (GROUPS ? group : sum)[r * M + m] = d;
                }
            }
            if constexpr (GROUPS) {
                // a group's sum is an integer, rounded with its scale into the float32 sum
                Mine::join(group, lane);
                if (live) {
#pragma unroll
                    for (int i = 0; i < Mine::kOwn; ++i) acc[i] = fmaf((float)group[i], ws[i / M], acc[i]);
                }
                fetch_scales(on, cn);
            }
        }
        if constexpr (GROUPS) {
            // over the warp's groups
#pragma unroll
            for (int i = 0; i < Mine::kOwn; ++i) {
#pragma unroll
                for (int off = 16; off >= LANES; off /= 2) acc[i] += __shfl_xor_sync(0xffffffffu, acc[i], off);
                if (lane < LANES && lane % Mine::kSame == 0) parts[turn][warp][first + i] = __float_as_uint(acc[i]);
            }
        } else {
#pragma unroll
            for (int i = 0; i < V; ++i) {
                const int v = __reduce_add_sync(0xffffffffu, sum[i]);
                if (lane == i) parts[turn][warp][i] = (uint32_t)v;
            }
        }
        __syncthreads();                      // and the other half of parts is free
        const int o = o0 + tid / M, m = tid % M;
        if (tid < V && o < a.dout && m < a.n) {
            float f = 0.f;
            int i = 0;
#pragma unroll
            for (int p = 0; p < kWarps; ++p) {
                f += __uint_as_float(parts[turn][p][tid]);
                i += (int)parts[turn][p][tid];
            }
            const float v = GROUPS ? f : (float)i * a.ws[o];
            float xs = scale[0];
#pragma unroll
            for (int j = 1; j < M; ++j) xs = j == m ? scale[j] : xs;
            const float y = fmaf(v, xs, a.bias ? a.bias[o] : 0.f);
            with_type_device(a.dtype, [&](auto type) {
                using T = decltype(type);
                static_cast<T *>(a.Y)[(size_t)m * a.ldy + o] = from_float<T>(y);
            });
        }
    }
}

template <int M, int R, bool OWN>
cudaError_t launch_few(const ProductArgs &a, jarq_dtype xtype, cudaStream_t s, bool pdl) {
    // no more blocks than stay resident (cold weights, one token, 4096 -> 11008 with
    // quantization: 11.1 us, 12.7 with a block for each four channels)
    const int groups = (a.dout + R - 1) / R, resident = (M == 1 ? 4 : 2) * num_sms();
    const dim3 grid(groups < resident ? groups : resident);
    const size_t smem = OWN ? round_up(a.din, 16) : 0;
    const bool vec = OWN ? vector_codes(a) : vector_rows(a);
    auto run = [&](auto kernel) { return launch_k(kernel, grid, dim3(kThreads), smem, s, pdl, a, xtype); };
    if (a.g == 64) return vec ? run(few_tokens_kernel<M, R, 4, true, OWN>) : run(few_tokens_kernel<M, R, 4, false, OWN>);
    if (a.g) return vec ? run(few_tokens_kernel<M, R, 8, true, OWN>) : run(few_tokens_kernel<M, R, 8, false, OWN>);
    return vec ? run(few_tokens_kernel<M, R, 0, true, OWN>) : run(few_tokens_kernel<M, R, 0, false, OWN>);
}

// xtype: of one token's activations in the codes' place, or null
cudaError_t launch_product(const ProductArgs &a, const jarq_dtype *xtype, int *failed, cudaStream_t s, bool pdl) {
    if (xtype) return launch_few<1, 4, true>(a, *xtype, s, false);
    if (a.n == 1) return launch_few<1, 4, false>(a, JARQ_F32, s, pdl);
    if (a.n <= kFewTokens) return launch_few<2, 8, false>(a, JARQ_F32, s, pdl);
    return launch_tc_integer(a, failed, s, pdl);
}

jarq_status check_layer(const int8_t *C, int64_t ldc, const float *ws, int group_size,
                        const float *bias, int n, int dout, int din, jarq_dtype dtype, const void *Y,
                        int64_t ldy) {
    if (n < 0 || n > kMostIndex || dout < 1 || dout > kMostIndex || din < 1 || din > 65536 || ldc < din || ldy < dout ||
        !is_dtype(dtype))
        return JARQ_ERR_ARG;
    if (group_size != 0 && ((group_size != 64 && group_size != 128) || din % group_size)) return JARQ_ERR_ARG;
    if (n == 0) return JARQ_OK;
    if (!C || !ws || !Y || !on_device(C) || !on_device(ws) || !on_device(Y) || (bias && !on_device(bias)))
        return JARQ_ERR_ARG;
    if (((uintptr_t)ws | (uintptr_t)bias) & 3 || (uintptr_t)Y & (size_of(dtype) - 1)) return JARQ_ERR_ARG;
    return JARQ_OK;
}

jarq_status run_product(const ProductArgs &a, const jarq_dtype *xtype, cudaStream_t st, bool pdl) {
    // one and two tokens have no wait that could give up
    int *failed = nullptr;
    if (a.n > kFewTokens && !(failed = async_word())) return JARQ_ERR_NOMEM;
    ProfScope ps("integer_product", st);
    const cudaError_t e = launch_product(a, xtype, failed, st, pdl);
    ps.done();
    count_launches(1);
    if (e != cudaSuccess) {
        (void)cudaGetLastError();
        return JARQ_ERR_CUDA;
    }
    return JARQ_OK;
}

jarq_status run_quantize(const void *X, jarq_dtype dtype, int n, int d, int64_t ldx, void *Q, bool half,
                         int64_t ldq, float *scale, cudaStream_t st) {
    ProfScope ps("quantize_rows", st);
    const cudaError_t e = launch_quantize_rows(X, dtype, n, d, ldx, Q, half, ldq, scale, st);
    ps.done();
    count_launches(1);
    if (e != cudaSuccess) {
        (void)cudaGetLastError();
        return JARQ_ERR_CUDA;
    }
    return JARQ_OK;
}

// A linear layer's workspace: its activations' integers, int8 for a few tokens
// and fp16 for more, rows on 16-byte boundaries; then the scales.
int64_t code_pitch(int din) { return round_up(din, 16); }
size_t code_bytes(int n, int din) { return (size_t)n * code_pitch(din) * (n <= kFewTokens ? 1 : 2); }

}  // namespace
}  // namespace jarq

using namespace jarq;

extern "C" {

jarq_status jarq_quantize_rows(const void *X, jarq_dtype dtype, int n, int d, int64_t ldx,
                               int8_t *Q, int64_t ldq, float *scale, void *stream) {
    if (n < 0 || n > kMostIndex || d < 1 || d > kMostIndex || ldx < d || ldq < d || !is_dtype(dtype)) return JARQ_ERR_ARG;
    if (n == 0) return JARQ_OK;
    if (!X || !Q || !scale || !on_device(X) || !on_device(Q) || !on_device(scale)) return JARQ_ERR_ARG;
    if ((uintptr_t)X & (size_of(dtype) - 1) || (uintptr_t)scale & 3) return JARQ_ERR_ARG;
    if (const jarq_status late = async_failure()) return late;
    return run_quantize(X, dtype, n, d, ldx, Q, false, ldq, scale, (cudaStream_t)stream);
}

jarq_status jarq_integer_product(const int8_t *X, int64_t ldx, const float *xs, const int8_t *C,
                                 int64_t ldc, const float *ws, int group_size, const float *bias,
                                 int n, int dout, int din, jarq_dtype dtype, void *Y, int64_t ldy,
                                 void *stream) {
    if (ldx < din) return JARQ_ERR_ARG;
    const jarq_status ok = check_layer(C, ldc, ws, group_size, bias, n, dout, din, dtype, Y, ldy);
    if (ok != JARQ_OK || n == 0) return ok;
    if (!X || !xs || !on_device(X) || !on_device(xs) || (uintptr_t)xs & 3) return JARQ_ERR_ARG;
    if (const jarq_status late = async_failure()) return late;
    return run_product({X, C, xs, ws, bias, Y, ldx, ldc, ldy, n, dout, din, group_size,
                        group_size ? din / group_size : 1, dtype, false},
                       nullptr, (cudaStream_t)stream, false);
}

size_t jarq_integer_linear_workspace(int n, int din) {
    if (n < 0 || din < 1) return 0;
    return code_bytes(n, din) + (size_t)n * sizeof(float);
}

jarq_status jarq_integer_linear(const void *X, jarq_dtype xdtype, int64_t ldx, const int8_t *C,
                                int64_t ldc, const float *ws, int group_size, const float *bias,
                                int n, int dout, int din, jarq_dtype ydtype, void *Y, int64_t ldy,
                                void *workspace, size_t workspace_bytes, void *stream) {
    if (ldx < din || !is_dtype(xdtype)) return JARQ_ERR_ARG;
    const jarq_status ok = check_layer(C, ldc, ws, group_size, bias, n, dout, din, ydtype, Y, ldy);
    if (ok != JARQ_OK || n == 0) return ok;
    if (!X || !on_device(X) || (uintptr_t)X & (size_of(xdtype) - 1)) return JARQ_ERR_ARG;
    if (!workspace || (uintptr_t)workspace & 15 || !on_device(workspace) ||
        workspace_bytes < jarq_integer_linear_workspace(n, din))
        return JARQ_ERR_ARG;
    if (const jarq_status late = async_failure()) return late;
    cudaStream_t st = (cudaStream_t)stream;
    const int64_t ldq = code_pitch(din);
    const bool half = n > kFewTokens;
    if (n == 1 && din <= kOwnCodes)
        return run_product({X, C, nullptr, ws, bias, Y, ldx, ldc, ldy, n, dout, din, group_size,
                            group_size ? din / group_size : 1, ydtype, false},
                           &xdtype, st, false);
    float *xs = reinterpret_cast<float *>(static_cast<char *>(workspace) + code_bytes(n, din));
    const jarq_status e = run_quantize(X, xdtype, n, din, ldx, workspace, half, ldq, xs, st);
    if (e != JARQ_OK) return e;
    // the product starts under the quantization and reads weights meanwhile
    return run_product({workspace, C, xs, ws, bias, Y, ldq, ldc, ldy, n, dout, din, group_size,
                        group_size ? din / group_size : 1, ydtype, half},
                       nullptr, st, true);
}

jarq_status jarq_async_status(void *stream) {
    if (cudaStreamSynchronize((cudaStream_t)stream) != cudaSuccess) {
        (void)cudaGetLastError();
        return JARQ_ERR_CUDA;
    }
    return take_async_failure();
}

}  // extern "C"
