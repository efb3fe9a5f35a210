// A row's scale and the integers of its elements: q = rint(x (127 / a)), a the
// row's largest magnitude.
#pragma once

#include <type_traits>

#include "rows.cuh"
#include "tc_common.cuh"

namespace jarq {
namespace quant {

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

// What a row is scaled by, from the bits of its largest magnitude.
struct RowScale {
    bool bad;                          // an infinity or a NaN in the row
    float inv, scale;
    __device__ explicit RowScale(uint32_t top) {
        const float amax = __uint_as_float(top);
        const bool zero = amax < kTiny;                // too small to scale
        bad = top >= 0x7F800000u;
        inv = zero || bad ? 0.f : __fdiv_rn(127.f, amax);
        scale = bad ? __int_as_float(0x7FC00000) : zero ? 0.f : __fdiv_rn(amax, 127.f);
    }
};

// The integers of unit u of a row, read as `raw`, to the row's codes q: int8, or
// the same in fp16.
template <class T, class Code>
__device__ __forceinline__ void put_codes(const rows::Row<T> &row, int u, const uint4 &raw, const RowScale &by, Code *q) {
    constexpr int E = rows::kUnit<T>;
    constexpr bool HALF = std::is_same_v<Code, __half>;
    float v[E];
    rows::unpack(raw, v, T());
    // fl(x inv) has magnitude below 2^8: adding 1.5 2^23 rounds it to an
    // integer, half to even, which then stands in the low bits.  (The product
    // is negated and subtracted: fused with an addition it would not be rounded.)
    const tc::F2 scale = tc::f2(-by.inv), round = tc::f2(12582912.f);
    tc::F2 c[E / 2];
#pragma unroll
    for (int i = 0; i < E / 2; ++i) {
        c[i] = tc::f2_sub(round, tc::f2_mul(tc::f2(v[2 * i], v[2 * i + 1]), scale));
        if (by.bad) c[i] = round;
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
}

}  // namespace quant
}  // namespace jarq
