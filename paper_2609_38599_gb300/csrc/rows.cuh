// Rows of float32, float16 or bfloat16 values read and written 16 bytes at a
// time at any alignment, and what the kernels that read such rows share.
#pragma once

#include <float.h>

#include "jarq_internal.cuh"

namespace jarq {
namespace rows {

template <class T>
constexpr int kUnit = 16 / (int)sizeof(T);     // elements of 16 bytes

template <class T>
__device__ __forceinline__ float to_float(T x) {
    return (float)x;
}
template <class T>
__device__ __forceinline__ T from_float(float x);
template <>
__device__ __forceinline__ float from_float<float>(float x) {
    return x;
}
template <>
__device__ __forceinline__ __half from_float<__half>(float x) {
    return __float2half_rn(x);
}
template <>
__device__ __forceinline__ __nv_bfloat16 from_float<__nv_bfloat16>(float x) {
    return __float2bfloat16_rn(x);
}

// The elements of 16 bytes as float32.
__device__ __forceinline__ void unpack(const uint4 &r, float (&v)[4], float) {
    v[0] = __uint_as_float(r.x);
    v[1] = __uint_as_float(r.y);
    v[2] = __uint_as_float(r.z);
    v[3] = __uint_as_float(r.w);
}
__device__ __forceinline__ void unpack(const uint4 &r, float (&v)[8], __half) {
    const uint32_t w[4] = {r.x, r.y, r.z, r.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const float2 f = __half22float2(*reinterpret_cast<const __half2 *>(&w[i]));
        v[2 * i] = f.x;
        v[2 * i + 1] = f.y;
    }
}
__device__ __forceinline__ void unpack(const uint4 &r, float (&v)[8], __nv_bfloat16) {
    const uint32_t w[4] = {r.x, r.y, r.z, r.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        v[2 * i] = __uint_as_float(w[i] << 16);
        v[2 * i + 1] = __uint_as_float(w[i] & 0xFFFF0000u);
    }
}
// float32 values rounded to T, as 16 bytes.
__device__ __forceinline__ uint4 pack(const float (&v)[4], float) {
    return make_uint4(__float_as_uint(v[0]), __float_as_uint(v[1]), __float_as_uint(v[2]), __float_as_uint(v[3]));
}
__device__ __forceinline__ uint4 pack(const float (&v)[8], __half) {
    uint32_t w[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const __half2 h = __floats2half2_rn(v[2 * i], v[2 * i + 1]);
        w[i] = *reinterpret_cast<const uint32_t *>(&h);
    }
    return make_uint4(w[0], w[1], w[2], w[3]);
}
__device__ __forceinline__ uint4 pack(const float (&v)[8], __nv_bfloat16) {
    uint32_t w[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const __nv_bfloat162 h = __floats2bfloat162_rn(v[2 * i], v[2 * i + 1]);
        w[i] = *reinterpret_cast<const uint32_t *>(&h);
    }
    return make_uint4(w[0], w[1], w[2], w[3]);
}

// A row of n elements cut into units of 16 bytes at 16-byte boundaries; the
// first and the last unit may lie partly outside the row, and what lies
// outside is never read.
template <class T>
struct Row {
    static constexpr int E = kUnit<T>;
    const T *p;       // first element
    int n, skip;      // elements; those of unit 0 that lie before the row
    __device__ Row(const T *row, int len)
        : p(row), n(len), skip((int)(((uintptr_t)row & 15) / sizeof(T))) {}
    __device__ int units() const { return (n + skip + E - 1) / E; }
    __device__ int first(int u) const { return u * E - skip; }      // < 0 in a cut unit 0
    __device__ bool whole(int u) const { return first(u) >= 0 && first(u) + E <= n; }
    // unit u, elements outside the row as `fill`
    __device__ uint4 load(int u, T fill) const {
        const int f = first(u);
        if (whole(u)) return *reinterpret_cast<const uint4 *>(p + f);
        alignas(16) T t[E];
#pragma unroll
        for (int e = 0; e < E; ++e) t[e] = f + e >= 0 && f + e < n ? p[f + e] : fill;
        return *reinterpret_cast<const uint4 *>(t);
    }
};

}  // namespace rows

// `f(T())` for the element type of `dtype`.
template <class F>
auto with_type(jarq_dtype dtype, F f) {
    if (dtype == JARQ_F16) return f(__half());
    if (dtype == JARQ_BF16) return f(__nv_bfloat16());
    return f(float());
}
template <class F>
__device__ __forceinline__ void with_type_device(jarq_dtype dtype, F f) {
    if (dtype == JARQ_F16)
        f(__half());
    else if (dtype == JARQ_BF16)
        f(__nv_bfloat16());
    else
        f(float());
}
inline bool is_dtype(jarq_dtype t) { return t == JARQ_F32 || t == JARQ_F16 || t == JARQ_BF16; }
inline size_t size_of(jarq_dtype t) { return t == JARQ_F32 ? 4 : 2; }

}  // namespace jarq
