// Rows of activations to 8-bit integers with a scale for each row: with a the
// row's largest magnitude, scale = a / 127 and q = rint(x (127 / a)).
//
// One pass over memory: a row is read into registers 16 bytes at a time, its
// maximum is taken over the threads that share it, and the codes are formed
// from the registers.
#include <type_traits>

#include "rows.cuh"
#include "tc_common.cuh"

namespace jarq {
namespace {

using namespace rows;

constexpr int kThreads = 256;
constexpr int kHeld = 8;              // units of a row that a thread holds
constexpr float kTiny = 0x1p-120f;    // 127 / a stays finite above it

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
    constexpr int E = kUnit<T>;
    tc::pdl_launch_dependents();          // a product may read its weights meanwhile
    __shared__ uint32_t part[kThreads / 32];
    const int r = blockIdx.x * (kThreads / kPerRow) + threadIdx.x / kPerRow, t = threadIdx.x % kPerRow;
    if (kPerRow == 32 && r >= a.n) return;
    const Row<T> row(static_cast<const T *>(a.X) + (size_t)r * a.ldx, a.d);
    const int units = row.units();
    uint4 held[kHeld];
    // magnitudes as integers: NaN above infinity above every finite value
    uint32_t top = 0;
    auto take = [&](const uint4 &raw) {
        float v[E];
        unpack(raw, v, T());
#pragma unroll
        for (int e = 0; e < E; ++e) top = max(top, __float_as_uint(v[e]) & 0x7FFFFFFFu);
    };
#pragma unroll
    for (int i = 0; i < kHeld; ++i) {
        const int u = t + i * kPerRow;
        if (u < units) held[i] = row.load(u, T(0.f));
    }
#pragma unroll
    for (int i = 0; i < kHeld; ++i)
        if (t + i * kPerRow < units) take(held[i]);
    for (int u = t + kHeld * kPerRow; u < units; u += kPerRow) take(row.load(u, T(0.f)));
    top = __reduce_max_sync(0xffffffffu, top);
    if (kPerRow > 32) {
        if ((threadIdx.x & 31) == 0) part[threadIdx.x >> 5] = top;
        __syncthreads();
#pragma unroll
        for (int w = 0; w < kThreads / 32; ++w) top = max(top, part[w]);
    }
    const float amax = __uint_as_float(top);
    const bool bad = top >= 0x7F800000u, zero = amax < kTiny;     // not finite; too small to scale
    const float inv = zero || bad ? 0.f : __fdiv_rn(127.f, amax);
    if (t == 0) a.scale[r] = bad ? __int_as_float(0x7FC00000) : zero ? 0.f : __fdiv_rn(amax, 127.f);
    using Code = std::conditional_t<HALF, __half, int8_t>;
    Code *q = static_cast<Code *>(a.Q) + (size_t)r * a.ldq;
    auto put = [&](int u, const uint4 &raw) {
        float v[E];
        unpack(raw, v, T());
        // fl(x inv) has magnitude below 2^8: adding 1.5 2^23 rounds it to an
        // integer, half to even, which then stands in the low bits
        constexpr float kRound = 12582912.f;
        const int f = row.first(u);
        const bool whole = row.whole(u) && ((uintptr_t)(q + f) & (E * sizeof(Code) - 1)) == 0;
        if constexpr (HALF) {
            alignas(16) Code c[E];
#pragma unroll
            for (int e = 0; e < E; ++e)
                c[e] = __float2half_rn(bad ? 0.f : __fsub_rn(__fadd_rn(__fmul_rn(v[e], inv), kRound), kRound));
            if (whole) {
                if (E == 8)
                    *reinterpret_cast<uint4 *>(q + f) = *reinterpret_cast<const uint4 *>(c);
                else
                    *reinterpret_cast<uint2 *>(q + f) = *reinterpret_cast<const uint2 *>(c);
            } else {
#pragma unroll
                for (int e = 0; e < E; ++e)
                    if (f + e >= 0 && f + e < row.n) q[f + e] = c[e];
            }
        } else {
            uint32_t c[E];
#pragma unroll
            for (int e = 0; e < E; ++e)
                c[e] = bad ? 0u : __float_as_uint(__fadd_rn(__fmul_rn(v[e], inv), kRound));
            if (whole) {
                uint32_t w[E / 4];
#pragma unroll
                for (int i = 0; i < E / 4; ++i)
                    w[i] = __byte_perm(__byte_perm(c[4 * i], c[4 * i + 1], 0x0040),
                                       __byte_perm(c[4 * i + 2], c[4 * i + 3], 0x0040), 0x5410);
                if (E == 8)
                    *reinterpret_cast<uint2 *>(q + f) = make_uint2(w[0], w[E / 4 - 1]);
                else
                    *reinterpret_cast<uint32_t *>(q + f) = w[0];
            } else {
#pragma unroll
                for (int e = 0; e < E; ++e)
                    if (f + e >= 0 && f + e < row.n) q[f + e] = (int8_t)(c[e] & 0xFF);
            }
        }
    };
#pragma unroll
    for (int i = 0; i < kHeld; ++i) {
        const int u = t + i * kPerRow;
        if (u < units) put(u, held[i]);
    }
    for (int u = t + kHeld * kPerRow; u < units; u += kPerRow) put(u, row.load(u, T(0.f)));
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
