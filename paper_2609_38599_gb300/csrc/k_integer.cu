// Product of 8-bit integers with scales for each token and channel:
//   Y[t][o] = xs[t] sum_i ws[o][i] (sum_{k in group i} X[t][k] C[o][k]) + bias[o].
#include "rows.cuh"

namespace jarq {
namespace {

using namespace rows;

struct ProductArgs {
    const int8_t *X, *C;
    const float *xs, *ws, *bias;
    void *Y;
    int64_t ldx, ldc, ldy;
    int n, dout, din, g, G;
};

constexpr int kTile = 64, kStep = 64;      // 64 x 64 outputs, 64 of K a step

// Simple form: 256 threads, 4 x 4 outputs each, integer dot products of four.
template <class T>
__global__ void __launch_bounds__(256) integer_product_kernel(ProductArgs a) {
    __shared__ uint32_t sx[kTile][kStep / 4 + 1], sc[kTile][kStep / 4 + 1];
    const int t0 = blockIdx.y * kTile, o0 = blockIdx.x * kTile;
    const int tx = threadIdx.x & 15, ty = threadIdx.x >> 4;
    float acc[4][4] = {};
    int sum[4][4] = {};
    for (int k0 = 0; k0 < a.din; k0 += kStep) {
        for (int i = threadIdx.x; i < kTile * kStep / 4; i += 256) {
            const int r = i / (kStep / 4), c = i % (kStep / 4);
            uint32_t wx = 0, wc = 0;
#pragma unroll
            for (int b = 0; b < 4; ++b) {
                const int k = k0 + 4 * c + b;
                if (k < a.din && t0 + r < a.n) wx |= (uint32_t)(uint8_t)a.X[(size_t)(t0 + r) * a.ldx + k] << (8 * b);
                if (k < a.din && o0 + r < a.dout)
                    wc |= (uint32_t)(uint8_t)a.C[(size_t)(o0 + r) * a.ldc + k] << (8 * b);
            }
            sx[r][c] = wx;
            sc[r][c] = wc;
        }
        __syncthreads();
        for (int c = 0; c < kStep / 4; ++c) {
#pragma unroll
            for (int i = 0; i < 4; ++i)
#pragma unroll
                for (int j = 0; j < 4; ++j)
                    sum[i][j] = __dp4a((int)sx[ty + 16 * i][c], (int)sc[tx + 16 * j][c], sum[i][j]);
        }
        __syncthreads();
        if (a.g && (k0 + kStep) % a.g == 0) {
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const int o = o0 + tx + 16 * j;
                const float w = o < a.dout ? a.ws[(size_t)o * a.G + k0 / a.g] : 0.f;
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    acc[i][j] = fmaf((float)sum[i][j], w, acc[i][j]);
                    sum[i][j] = 0;
                }
            }
        }
    }
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const int t = t0 + ty + 16 * i, o = o0 + tx + 16 * j;
            if (t >= a.n || o >= a.dout) continue;
            const float v = a.g ? acc[i][j] : (float)sum[i][j] * a.ws[o];
            static_cast<T *>(a.Y)[(size_t)t * a.ldy + o] = from_float<T>(fmaf(v, a.xs[t], a.bias ? a.bias[o] : 0.f));
        }
}

cudaError_t launch_product(const ProductArgs &a, jarq_dtype dtype, cudaStream_t s) {
    const dim3 grid((a.dout + kTile - 1) / kTile, (a.n + kTile - 1) / kTile);
    if (grid.y > 65535) return cudaErrorInvalidValue;
    with_type(dtype, [&](auto type) {
        integer_product_kernel<decltype(type)><<<grid, 256, 0, s>>>(a);
        return 0;
    });
    return cudaGetLastError();
}

jarq_status check_layer(const int8_t *C, int64_t ldc, const float *ws, int group_size,
                        const float *bias, int n, int dout, int din, jarq_dtype dtype, const void *Y,
                        int64_t ldy) {
    if (n < 0 || dout < 1 || din < 1 || din > 65536 || ldc < din || ldy < dout || !is_dtype(dtype)) return JARQ_ERR_ARG;
    if (group_size != 0 && ((group_size != 64 && group_size != 128) || din % group_size)) return JARQ_ERR_ARG;
    if (n == 0) return JARQ_OK;
    if (!C || !ws || !Y || !on_device(C) || !on_device(ws) || !on_device(Y) || (bias && !on_device(bias)))
        return JARQ_ERR_ARG;
    if (((uintptr_t)ws | (uintptr_t)bias) & 3 || (uintptr_t)Y & (size_of(dtype) - 1)) return JARQ_ERR_ARG;
    return JARQ_OK;
}

jarq_status run_product(const ProductArgs &a, jarq_dtype dtype, cudaStream_t st) {
    ProfScope ps("integer_product", st);
    const cudaError_t e = launch_product(a, dtype, st);
    ps.done();
    count_launches(1);
    if (e != cudaSuccess) {
        (void)cudaGetLastError();
        return JARQ_ERR_CUDA;
    }
    return JARQ_OK;
}

jarq_status run_quantize(const void *X, jarq_dtype dtype, int n, int d, int64_t ldx, int8_t *Q,
                         int64_t ldq, float *scale, cudaStream_t st) {
    ProfScope ps("quantize_rows", st);
    const cudaError_t e = launch_quantize_rows(X, dtype, n, d, ldx, Q, ldq, scale, st);
    ps.done();
    count_launches(1);
    if (e != cudaSuccess) {
        (void)cudaGetLastError();
        return JARQ_ERR_CUDA;
    }
    return JARQ_OK;
}

// Codes of a linear layer's activations in its workspace: rows on 16-byte
// boundaries, then the scales.
int64_t code_pitch(int din) { return round_up(din, 16); }

}  // namespace
}  // namespace jarq

using namespace jarq;

extern "C" {

jarq_status jarq_quantize_rows(const void *X, jarq_dtype dtype, int n, int d, int64_t ldx,
                               int8_t *Q, int64_t ldq, float *scale, void *stream) {
    if (n < 0 || d < 1 || ldx < d || ldq < d || !is_dtype(dtype)) return JARQ_ERR_ARG;
    if (n == 0) return JARQ_OK;
    if (!X || !Q || !scale || !on_device(X) || !on_device(Q) || !on_device(scale)) return JARQ_ERR_ARG;
    if ((uintptr_t)X & (size_of(dtype) - 1) || (uintptr_t)scale & 3) return JARQ_ERR_ARG;
    return run_quantize(X, dtype, n, d, ldx, Q, ldq, scale, (cudaStream_t)stream);
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
                        group_size ? din / group_size : 1},
                       dtype, (cudaStream_t)stream);
}

size_t jarq_integer_linear_workspace(int n, int din) {
    if (n < 0 || din < 1) return 0;
    return (size_t)n * (size_t)(code_pitch(din) + (int64_t)sizeof(float));
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
    int8_t *q = static_cast<int8_t *>(workspace);
    float *xs = reinterpret_cast<float *>(q + (size_t)n * ldq);
    const jarq_status e = run_quantize(X, xdtype, n, din, ldx, q, ldq, xs, st);
    if (e != JARQ_OK) return e;
    return run_product({q, C, xs, ws, bias, Y, ldq, ldc, ldy, n, dout, din, group_size,
                        group_size ? din / group_size : 1},
                       ydtype, st);
}

jarq_status jarq_async_status(void *stream) {
    if (cudaStreamSynchronize((cudaStream_t)stream) != cudaSuccess) {
        (void)cudaGetLastError();
        return JARQ_ERR_CUDA;
    }
    return take_async_failure();
}

}  // extern "C"
