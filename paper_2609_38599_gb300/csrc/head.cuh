// What the kernels of the output head's loss share.
#pragma once

#include "rows.cuh"

namespace jarq {
namespace head {

// The products of a loss and its gradient, by their operands: `a` rows and `b`
// rows contiguous along the sum (K), or along what is kept (MN).
enum Product {
    kLoss,      // X W^T, reduced to a maximum and a sum of exponentials a row
    kLogits,    // X W^T, turned into its gradient D
    kHidden,    // D W:   a along K, b along MN
    kHead       // D^T X: both along MN
};

struct ProductArgs {
    int m, n;                   // rows and columns of the result
    int chunks, per, splits;    // 64-wide chunks of K, of a split, splits
    int cols;                   // columns of a tile: a multiple of 32, up to 256
    int mt, nt;                 // tiles of 256 x cols
    bool half;                  // float16, else bfloat16
    // kLoss, kLogits
    const int64_t *tokens;
    const float *lse, *g;       // kLogits; g also of kHidden
    int first, vocab;           // token of column 0; tokens of the vocabulary
    int rows;                   // of A's box of 128: fewer where the result has no more
    float2 *part;               // kLoss: [2 nt][m] maxima and sums of half a tile's columns
    float *target;              // kLoss: [m] logit of the row's token
    // kLogits: D [m][ldo].  kHidden, kHead: the result, or with `slab` float32 sums
    void *out;
    int64_t ldo;
    float *slab;                // [splits][m][pitch], null: none
    int pitch;
    bool add, last;             // to what slab holds; into out
    const int *top;             // kHead of float16: exponent of the rows' scale
    float *lost;                // [rows of X] what rounding took from D of a row's token, scaled as D is
    // kHidden, kHead: that goes into the result; `first` as above
    int window;                 // kHidden: tokens of the piece
    const uint16_t *w;          // kHidden: W from token `first` on; kHead: rows of X as the product reads them
    int64_t ldw;
    const int2 *tally;          // kHead: a token's first row and number of rows, from token `first` on
    const float *rest;          // kHead: of a token with several rows, at its first: what goes in
    int rest_pitch;
    int *failed;
};

// Float16 holds too few exponents for a gradient: row r of D is kept as
// D_r 2^(14 - e_r) with |g_r| 2^-e_r in [1/2, 1), so |D| <= 2^14, and probabilities
// down to 2^-27 keep all their bits (float16's smallest normal number is 2^-14); smaller
// ones are rounded to multiples of 2^-38 to 2^-37.  Powers of two are exact, and undone at the end.
__device__ __forceinline__ int exponent(float g) { return (int)((__float_as_uint(g) >> 23) & 255) - 126; }
__device__ __forceinline__ float scaled(float g) {
    const int e = exponent(g);
    if (e == -126) return 0.f;                    // zero, or below 2^-126
    if (e == 129) return g;                       // an infinity, a NaN
    return __uint_as_float((__float_as_uint(g) & 0x807FFFFFu) | (140u << 23));
}

// pdl: the launch before it in the stream is one of the same call's.
cudaError_t launch_product(Product which, const CUtensorMap &a, const CUtensorMap &b, const ProductArgs &args,
                           cudaStream_t s, bool pdl, bool stalled = false);

// The self-test's form of the loss's product, on `stalled_bytes` of zeros, whose
// issuer stops early and whose waits give up.
size_t stalled_bytes();
cudaError_t launch_stalled(char *zeros, int *failed, cudaStream_t s);

}  // namespace head
}  // namespace jarq
