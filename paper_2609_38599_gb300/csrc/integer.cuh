// The integer product's arguments, shared by its kernels.
#pragma once

#include "jarq_internal.cuh"

namespace jarq {

// Y[t][o] = xs[t] sum_i ws[o][i] (sum_{k in group i} X[t][k] C[o][k]) + bias[o]
struct ProductArgs {
    const void *X;               // int8 codes, or (half) the same integers in fp16
    const int8_t *C;
    const float *xs, *ws, *bias;
    void *Y;
    int64_t ldx, ldc, ldy;
    int n, dout, din, g, G;      // g: group size, 0 for one scale a channel (G = 1)
    jarq_dtype dtype;            // of Y
    bool half;
};

// Most tokens, channels and elements of a row to quantize: the kernels' int indexes
// go up to a wave of tiles (4096) beyond them.
constexpr int kMostIndex = 0x7FFFFFFF - 4095;

// Most tokens of the form without tensor cores, which takes int8 codes.  Two tokens,
// cold and from L2: 4096 -> 11008 13.3 and 9.4 us, on the tensor cores 17.0 and 15.0;
// 11008 -> 4096 with groups of 128 14.8 and 10.2, there 17.1 and 14.0.  Four tokens of
// the latter, by dot products of four tokens at a time: 22.4 against 14.0.
constexpr int kFewTokens = 2;

// Codes k .. k + 15 of a row of `len`; zeros beyond it, which are not read.  VEC:
// the row and k are multiples of 16 bytes; otherwise whole words inside the row
// are read and shifted, and single codes at its ends.
template <bool VEC>
__device__ __forceinline__ uint4 load_codes(const int8_t *row, int k, int len) {
    const int8_t *p = row + k;
    if (VEC && k + 16 <= len) return *reinterpret_cast<const uint4 *>(p);
    uint32_t w[4] = {0, 0, 0, 0};
    if (!VEC && k >= 4 && k + 20 <= len) {
        const uint32_t off = (uint32_t)((uintptr_t)p & 3), sel = 0x3210u + 0x1111u * off;
        const uint32_t *q = reinterpret_cast<const uint32_t *>(p - off);
        uint32_t v[5];
#pragma unroll
        for (int i = 0; i < 5; ++i) v[i] = q[i];
#pragma unroll
        for (int i = 0; i < 4; ++i) w[i] = __byte_perm(v[i], v[i + 1], sel);
    } else if (k < len) {
#pragma unroll
        for (int b = 0; b < 16; ++b)
            if (k + b < len) w[b / 4] |= (uint32_t)(uint8_t)p[b] << (8 * (b % 4));
    }
    return make_uint4(w[0], w[1], w[2], w[3]);
}

// Whether all rows of weight codes (of all codes) lie on 16-byte boundaries.
inline bool vector_codes(const ProductArgs &a) {
    return ((uintptr_t)a.C & 15) == 0 && (a.ldc % 16 == 0 || a.dout == 1);
}
inline bool vector_rows(const ProductArgs &a) {
    return vector_codes(a) && ((uintptr_t)a.X & 15) == 0 && (a.ldx % 16 == 0 || a.n == 1);
}

// More than a few tokens, on the tensor cores (k_tc_integer.cu).  `failed`: set
// to 1 by a kernel whose waits gave up.  pdl: X and xs are the previous kernel's
// results, and that kernel reads or writes nothing else of a's.
cudaError_t launch_tc_integer(const ProductArgs &a, int *failed, cudaStream_t s, bool pdl);
// The self-test's form (256 tokens, fp16, aligned), whose issuer stops early and whose waits give up.
cudaError_t launch_tc_integer_stalled(const ProductArgs &a, int *failed, cudaStream_t s);

}  // namespace jarq
