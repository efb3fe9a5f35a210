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

#include "rows.cuh"
#include "tc_common.cuh"

namespace jarq {
namespace {

using namespace rows;

constexpr int kThreads = 256;
constexpr int kHeld = 8;              // units of a row that a thread holds
constexpr float kTiny = 0x1p-120f;    // 127 / a stays finite above it

// The largest magnitude among the elements of several units, as the bits of a
// float32: NaN above infinity above every finite value.
template <class T>
struct Largest;
template <>
struct Largest<float> {
    uint32_t top = 0;
    __device__ void take(const uint4 &r) {
        const uint32_t w[4] = {r.x, r.y, r.z, r.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) top = max(top, w[i] & 0x7FFFFFFFu);
    }
    __device__ uint32_t bits() const { return top; }
};
// 16-bit types: two at a time, NaN stays
template <class T, class T2>
struct Largest16 {
    T2 top;
    __device__ Largest16() {
        const uint32_t zero = 0;
        top = *reinterpret_cast<const T2 *>(&zero);
    }
    __device__ void take(const uint4 &r) {
        const uint32_t w[4] = {r.x, r.y, r.z, r.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) top = __hmax2_nan(top, __habs2(*reinterpret_cast<const T2 *>(&w[i])));
    }
    __device__ uint32_t bits() const {
        const uint32_t lo = __float_as_uint((float)top.x), hi = __float_as_uint((float)top.y);
        return max(lo & 0x7FFFFFFFu, hi & 0x7FFFFFFFu);
    }
};
template <>
struct Largest<__half> : Largest16<__half, __half2> {};
template <>
struct Largest<__nv_bfloat16> : Largest16<__nv_bfloat16, __nv_bfloat162> {};

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
        // integer, half to even, which then stands in the low bits.  (The product
        // is negated and subtracted: fused with an addition it would not be rounded.)
        const tc::F2 scale = tc::f2(-inv), round = tc::f2(12582912.f);
        tc::F2 c[E / 2];
#pragma unroll
        for (int i = 0; i < E / 2; ++i) {
            c[i] = tc::f2_sub(round, tc::f2_mul(tc::f2(v[2 * i], v[2 * i + 1]), scale));
            if (bad) c[i] = round;
        }
        const int f = row.first(u);
        const bool whole = row.whole(u) && ((uintptr_t)(q + f) & (E * sizeof(Code) - 1)) == 0;
        if constexpr (HALF) {
            alignas(16) __half2 h[E / 2];
#pragma unroll
            for (int i = 0; i < E / 2; ++i) {
                float x0, x1;
                tc::f2_get(tc::f2_sub(c[i], round), x0, x1);
                h[i] = __floats2half2_rn(x0, x1);
            }
            if (whole) {
                if (E == 8)
                    *reinterpret_cast<uint4 *>(q + f) = *reinterpret_cast<const uint4 *>(h);
                else
                    *reinterpret_cast<uint2 *>(q + f) = *reinterpret_cast<const uint2 *>(h);
            } else {
#pragma unroll
                for (int e = 0; e < E; ++e)
                    if (f + e >= 0 && f + e < row.n) q[f + e] = e % 2 ? h[e / 2].y : h[e / 2].x;
            }
        } else {
            uint32_t b[E];
#pragma unroll
            for (int i = 0; i < E / 2; ++i) {
                float x0, x1;
                tc::f2_get(c[i], x0, x1);
                b[2 * i] = __float_as_uint(x0);
                b[2 * i + 1] = __float_as_uint(x1);
            }
            if (whole) {
                uint32_t w[E / 4];
#pragma unroll
                for (int i = 0; i < E / 4; ++i)
                    w[i] = __byte_perm(__byte_perm(b[4 * i], b[4 * i + 1], 0x0040),
                                       __byte_perm(b[4 * i + 2], b[4 * i + 3], 0x0040), 0x5410);
                if (E == 8)
                    *reinterpret_cast<uint2 *>(q + f) = make_uint2(w[0], w[E / 4 - 1]);
                else
                    *reinterpret_cast<uint32_t *>(q + f) = w[0];
            } else {
#pragma unroll
                for (int e = 0; e < E; ++e)
                    if (f + e >= 0 && f + e < row.n) q[f + e] = (int8_t)(b[e] & 0xFF);
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
