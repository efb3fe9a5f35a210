// Rows of activations to 8-bit integers with a scale for each row: with a the
// row's largest magnitude, scale = a / 127 and q = rint(x (127 / a)).
//
// One pass over memory: a row is read into registers 16 bytes at a time, its
// maximum is taken over the threads that share it, and the codes are formed
// from the registers.
//
// Bound by memory where there are many rows: 8192 x 11008 in float16, 270 MB read
// and written, take 44 us (6.2 TB/s).  Two elements are handled an instruction,
// in the maximum and in the rounding: at one each, the same rows took 47 us.
#include <type_traits>

#include "quantize.cuh"

namespace jarq {
namespace {

using namespace quant;
using namespace rows;

constexpr int kThreads = 256;
constexpr int kHeld = 8;              // units of a row that a thread holds

struct QuantArgs {
    const void *X;
    void *Q;
    float *scale;
    int64_t ldx, ldq;
    int n, d;
};

// T: element type; HALF: codes in fp16; kPerRow: threads that share a row.
template <class T, bool HALF, int kPerRow>
__global__ void __launch_bounds__(kThreads) quantize_rows_kernel(QuantArgs a) {
    tc::pdl_launch_dependents();          // a product may read its weights meanwhile
    __shared__ uint32_t part[kThreads / 32];
    const int r = blockIdx.x * (kThreads / kPerRow) + threadIdx.x / kPerRow, t = threadIdx.x % kPerRow;
    if (kPerRow == 32 && r >= a.n) return;
    const Row<T> row(static_cast<const T *>(a.X) + (size_t)r * a.ldx, a.d);
    const int units = row.units();
    uint4 held[kHeld];
    Largest<T> largest;
#pragma unroll
    for (int i = 0; i < kHeld; ++i) {
        const int u = t + i * kPerRow;
        if (u < units) held[i] = row.load(u, T(0.f));
    }
#pragma unroll
    for (int i = 0; i < kHeld; ++i)
        if (t + i * kPerRow < units) largest.take(held[i]);
    for (int u = t + kHeld * kPerRow; u < units; u += kPerRow) largest.take(row.load(u, T(0.f)));
    uint32_t top = __reduce_max_sync(0xffffffffu, largest.bits());
    if (kPerRow > 32) {
        if ((threadIdx.x & 31) == 0) part[threadIdx.x >> 5] = top;
        __syncthreads();
#pragma unroll
        for (int w = 0; w < kThreads / 32; ++w) top = max(top, part[w]);
    }
    const RowScale by(top);
    if (t == 0) a.scale[r] = by.scale;
    using Code = std::conditional_t<HALF, __half, int8_t>;
    Code *q = static_cast<Code *>(a.Q) + (size_t)r * a.ldq;
#pragma unroll
    for (int i = 0; i < kHeld; ++i) {
        const int u = t + i * kPerRow;
        if (u < units) put_codes(row, u, held[i], by, q);
    }
    for (int u = t + kHeld * kPerRow; u < units; u += kPerRow) put_codes(row, u, row.load(u, T(0.f)), by, q);
}

template <class T, bool HALF>
void launch_rows(const QuantArgs &a, cudaStream_t s) {
    // a warp per row where it can hold the row
    if (a.d <= kUnit<T> * 32 * (kHeld - 1))
        quantize_rows_kernel<T, HALF, 32><<<(a.n + 7) / 8, kThreads, 0, s>>>(a);
    else
        quantize_rows_kernel<T, HALF, kThreads><<<a.n, kThreads, 0, s>>>(a);
}

}  // namespace

cudaError_t launch_quantize_rows(const void *X, jarq_dtype dtype, int n, int d, int64_t ldx, void *Q,
                                 bool half, int64_t ldq, float *scale, cudaStream_t s) {
    const QuantArgs a{X, Q, scale, ldx, ldq, n, d};
    with_type(dtype, [&](auto type) {
        using T = decltype(type);
        half ? launch_rows<T, true>(a, s) : launch_rows<T, false>(a, s);
        return 0;
    });
    return cudaGetLastError();
}

}  // namespace jarq
