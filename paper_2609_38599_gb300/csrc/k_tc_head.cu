// The products of an output head's loss and its gradient on the tensor cores:
//   logits = X W^T            reduced to a maximum and a sum of exponentials a row,
//   D = g (softmax - onehot)  from the same product once more, in the inputs' type,
//   dX = D W,  dW = D^T X.
// Logits exist in the accumulators alone.
//
// A pair of CTAs (cta_group::2) computes tiles of 256 x up to 256, K in chunks of 64, over
// a ring that TMA fills; an operand is read as it lies in memory, along K or (W of
// dX, D and X of dW) along MN, so that nothing is transposed.  In each CTA:
//   warp 0      TMA producer: its own 128 rows of A and half of B's columns
//   warp 1      TMEM allocation; in the even CTA the MMA issuer
//   warps 2..9  drain: lane quarter w % 4, half of the columns, of one accumulator
//               while the MMAs of the next fill the other (of the same tile, over a long K)
// A row of the loss lies in one thread: its maximum and sum need no exchange.
// Results leave through 4 KB of shared memory a warp, 128 bytes of a row at a time.
//
// Bound by the MMAs where there are many rows, by reading W where there are few:
//   2048 x 4096 -> 32000 bfloat16, loss    277 us, 1.94 PFLOP/s (in a long loop under the
//                                          power cap 314, 1.71: a library's product in both)
//   8192 x 4096 -> 32000, the four products of a step 1.07, 1.10, 1.16 and 1.17 ms
//   6144 x 2048 -> 16000, the same          203, 212, 236 and 226 us; tensor pipes 92, 89, 77 and
//                                          83 % active
//   1000 x 1344 -> 50001 float16           77, 85 and 87 us for logits, D and dX (1.6 PFLOP/s:
//                                          21 chunks of K a tile, the last wave's tail)
//   48 x 2048 -> 50001 float16             40 us (205 MB); one row, 7976 -> 86781 226 us (6.1 TB/s)
// Rows past the tokens: their boxes, filled with zeros by TMA, held the one row's call to
// 383 us.  D's exponentials as subtract, multiply, compare for masks and token, select, an
// element each: 113 us for 84.  Measured and not kept: sixteen drain warps with stages as
// small as their boxes (42 -> 44 us, 254 -> 266; only K below 200 gains), rows of W fetched
// into L2 a kilobyte ahead (42 -> 73), tiles of 160 columns where their waves come out even
// (1.47 ms for 1.18: the rows' operand is read as often as for 256).
#include <algorithm>
#include <type_traits>

#include "head.cuh"
#include "tc_common.cuh"
#include "turns.cuh"

namespace jarq {
namespace head {
namespace {

using namespace rows;

constexpr int kBox = 64 * 64 * 2;          // a TMA box of an operand along MN
constexpr int kTile = 128 * 64 * 2;        // a CTA's part of an operand's chunk
constexpr int kStage = 2 * kTile;
constexpr int kStages = 6;
constexpr int kDrainWarps = 8;
constexpr int kPart = 32 * 128;            // bytes that a drain warp stages
constexpr int kBars = 2 * kStages + 5;     // full, empty, afull[2], aempty[2], closing
constexpr int kSmem = 1024 + kStages * kStage + kDrainWarps * kPart + 8 * kBars + 16;
constexpr int kThreads = 32 * (2 + kDrainWarps);
// Chunks of K in one accumulator: the tensor cores' float32 additions round toward zero,
// which over a long K moves every sum the same way (logits over K = 4096 in one: lse off by
// 2e-6 of itself; dW over 13000 rows of one sign by 8e-5, dX over 15000 tokens by 1.4e-4).
// Logits go to the drain's registers after 1024 of it. Those of the gradient have to be the
// loss's own to the last bits: lse is subtracted, and of a token that has nearly all of the
// mass 1 as well. dX and dW, which are rounded to 16 bits, do so after 4096: 4e-5 then, a
// twelfth of float16's rounding (after 1024 a step of 8192 x 4096 -> 32000 took 2 % longer,
// of 100000 x 512 -> 32000 5 %).
template <Product kWhich>
constexpr int kSumChunks = kWhich == kLoss || kWhich == kLogits ? 16 : 64;
constexpr int kBand = 9;                   // tiles of rows of a band: with as many columns' tiles at one time, the fewest panels
static_assert(kSmem <= 227 * 1024, "ring and staged parts must fit an SM's shared memory");

// Descriptor of an operand along MN (128-byte swizzle): 64 elements of MN a row,
// rows of K 128 bytes apart, 8 of them 1024, the next 64 of MN one box further.
__device__ __forceinline__ uint64_t sdesc_mn(uint32_t saddr) {
    uint64_t d = 0;
    d |= (uint64_t)((saddr >> 4) & 0x3FFFu);
    d |= (uint64_t)(kBox >> 4) << 16;
    d |= (uint64_t)(1024 >> 4) << 32;
    d |= (uint64_t)1 << 46;
    d |= (uint64_t)2 << 61;
    return d;
}

// A pair's units of work: tiles in bands of kBand tiles of rows, column after column
// of a band, for one split of K after the other.
struct Unit {
    int ri, cj, split;
    __device__ Unit(int64_t u, const ProductArgs &a) {
        const int64_t tiles = (int64_t)a.mt * a.nt;
        split = (int)(u / tiles);
        u -= split * tiles;
        const int band = (int)(u / ((int64_t)kBand * a.nt));
        u -= (int64_t)band * kBand * a.nt;
        const int rows = min(kBand, a.mt - band * kBand);
        cj = (int)(u / rows);
        ri = band * kBand + (int)(u - (int64_t)cj * rows);
    }
};

__device__ __forceinline__ uint4 load_shared(uint32_t addr) {
    uint4 v;
    asm volatile("ld.shared.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(addr) : "memory");
    return v;
}
__device__ __forceinline__ void store_shared(uint32_t addr, uint32_t x, uint32_t y, uint32_t z, uint32_t w) {
    asm volatile("st.shared.v4.u32 [%0], {%1, %2, %3, %4};" ::"r"(addr), "r"(x), "r"(y), "r"(z), "r"(w) : "memory");
}
// 32 columns of this warp's lanes
__device__ __forceinline__ void load_columns(uint32_t taddr, float (&x)[32]) {
    uint32_t v[2][16];
    tc::tmem_ld16(taddr, v[0]);
    tc::tmem_ld16(taddr + 16, v[1]);
    tc::tmem_wait_ld();
#pragma unroll
    for (int e = 0; e < 32; ++e) x[e] = __uint_as_float(v[e / 16][e % 16]);
}
// This lane's 128 bytes of 32 rows to shared memory, and 16 bytes of four rows at a
// time back: row 4 i + lane / 8, bytes 16 (lane % 8) ..
__device__ __forceinline__ void stage_row(uint32_t part, int lane, const uint32_t (&w)[32]) {
    __syncwarp();
#pragma unroll
    for (int i = 0; i < 8; ++i)
        store_shared(part + lane * 128 + ((i ^ (lane & 7)) << 4), w[4 * i], w[4 * i + 1], w[4 * i + 2], w[4 * i + 3]);
    __syncwarp();
}
__device__ __forceinline__ uint4 staged(uint32_t part, int lane, int i) {
    const int row = 4 * i + (lane >> 3);
    return load_shared(part + row * 128 + (((lane & 7) ^ (row & 7)) << 4));
}
__device__ __forceinline__ uint32_t pack2(float lo, float hi, bool half) {
    if (half) {
        const __half2 h = __floats2half2_rn(lo, hi);
        return *reinterpret_cast<const uint32_t *>(&h);
    }
    const __nv_bfloat162 h = __floats2bfloat162_rn(lo, hi);
    return *reinterpret_cast<const uint32_t *>(&h);
}

// exp(x - y) of two x as 2^(x L - y L), L = log2 e: with the product y L rounded first,
// every exponential of a row is off by the same 2^rho, rho = y L - fl(y L), which the
// caller takes out of their sum or factor.  For |y| below 2^16; rho is below 2^-7 then.
__device__ __forceinline__ float exp2_approx(float x) {
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
constexpr float kLog2e = 1.44269504f, kNear = 65536.f;
struct Exponentials {
    tc::F2 scale, shift;
    float rho;
    __device__ explicit Exponentials(float y) : scale(tc::f2(kLog2e)) {
        const float p = __fmul_rn(y, kLog2e);
        shift = tc::f2(-p);
        rho = fmaf(y, kLog2e, -p);
    }
    __device__ tc::F2 of(tc::F2 x) const {
        float lo, hi;
        tc::f2_get(tc::f2_fma(x, scale, shift), lo, hi);
        return tc::f2(exp2_approx(lo), exp2_approx(hi));
    }
};

// A row of `cols` columns of logits: maximum, sum of exponentials less the maximum, and
// the token's logit where it is among them.
__device__ __forceinline__ void reduce_loss(tc::F2 (&acc)[64], const ProductArgs &a, int row, int64_t token, int col, int cols,
                                            int part) {
    const int64_t tok = token - col;
    const int limit = min(cols, a.n - col);
    const int mine = tok >= 0 && tok < limit ? (int)tok : -1;
    float m = -INFINITY, s = 0.f;
#pragma unroll
    for (int c = 0; c < 128; c += 32) {
        if (c >= limit) break;
        float x[32];
#pragma unroll
        for (int e = 0; e < 32; e += 2) tc::f2_get(acc[(c + e) / 2], x[e], x[e + 1]);
        if (c + 32 > limit) {
#pragma unroll
            for (int e = 0; e < 32; ++e)
                if (c + e >= limit) x[e] = -INFINITY;
        }
        if (mine >= c && mine < c + 32) {
            float t = 0.f;
#pragma unroll
            for (int e = 0; e < 32; ++e) t = mine == c + e ? x[e] : t;
            a.target[row] = t;
        }
        float top = m;
#pragma unroll
        for (int e = 0; e < 32; e += 2) top = fmaxf(fmaxf(x[e], x[e + 1]), top);
        const float ref = top == -INFINITY ? 0.f : top;
        float sum;
        if (fabsf(ref) < kNear) {
            const Exponentials exps(ref);
            tc::F2 t[2] = {tc::f2(0.f), tc::f2(0.f)};
#pragma unroll
            for (int e = 0; e < 32; e += 2) t[e / 2 % 2] = tc::f2_add(t[e / 2 % 2], exps.of(tc::f2(x[e], x[e + 1])));
            float lo, hi;
            tc::f2_get(tc::f2_add(t[0], t[1]), lo, hi);
            sum = (lo + hi) * exp2_approx(-exps.rho);
        } else {
            sum = 0.f;
#pragma unroll
            for (int e = 0; e < 32; ++e) sum += __expf(x[e] - ref);
        }
        s = fmaf(s, __expf(m - ref), sum);
        m = top;
    }
    if (row < a.m) a.part[(size_t)part * a.m + row] = make_float2(m, s);
}

// What a drain warp's lane knows of its row; read before the row's sums are waited for.
struct RowArgs {
    int64_t token;
    float lse, g;
    __device__ RowArgs(const ProductArgs &a, int row, bool gradient) {
        const bool in = row < a.m;
        token = in ? a.tokens[row] : -1;
        lse = in && gradient ? a.lse[row] : 0.f;
        g = in && gradient ? a.g[row] : 0.f;
    }
};

// Where a result's 32 columns from c on come from: an accumulator, or the sums of
// several in registers (c known to the compiler).
struct InTmem {
    uint32_t at;
    __device__ void load(int c, float (&x)[32]) const { load_columns(at + c, x); }
};
struct InRegisters {
    const tc::F2 (&at)[64];
    __device__ void load(int c, float (&x)[32]) const {
#pragma unroll
        for (int e = 0; e < 32; e += 2) tc::f2_get(at[(c + e) / 2], x[e], x[e + 1]);
    }
};

// `f(c)` for c = 0, STEP .. below the limit, a step's code once only where the columns
// may be any.
template <int STEP, class F>
__device__ __forceinline__ void columns(const InTmem &, int limit, F f) {
#pragma unroll 1
    for (int c = 0; c < limit; c += STEP) f(c);
}
template <int STEP, class F>
__device__ __forceinline__ void columns(const InRegisters &, int limit, F f) {
#pragma unroll
    for (int c = 0; c < 128; c += STEP) {
        if (c >= limit) break;
        f(c);
    }
}

// `cols` columns of logits to D.
template <class From>
__device__ __forceinline__ void drain_logits(const From &from, const ProductArgs &a, const RowArgs &of, int row0, int lane, int col,
                                             int cols, uint32_t part) {
    const int64_t tok = of.token, at = tok - a.first - col;
    const int mine = at >= 0 && at < cols ? (int)at : -1;
    const float lse = of.lse == -INFINITY ? 0.f : of.lse;         // -inf: every logit of the row is
    const float g = tok >= a.vocab ? __int_as_float(0x7FC00000) : a.half ? scaled(of.g) : of.g;
    const bool live = tok >= 0, all_live = __all_sync(0xffffffffu, live), near = __all_sync(0xffffffffu, fabsf(lse) < kNear);
    const Exponentials exps(lse);
    const tc::F2 by = tc::f2(g * exp2_approx(-exps.rho));
    uint16_t *out = static_cast<uint16_t *>(a.out) + (size_t)row0 * a.ldo + col;
    const int limit = min(cols, a.n - col);
    columns<64>(from, limit, [&](int c) {
        uint32_t w[32];
#pragma unroll
        for (int h = 0; h < 64; h += 32) {
            float x[32];
            from.load(c + h, x);
            if (near) {
#pragma unroll
                for (int e = 0; e < 32; e += 2) tc::f2_get(tc::f2_mul(exps.of(tc::f2(x[e], x[e + 1])), by), x[e], x[e + 1]);
            } else {
#pragma unroll
                for (int e = 0; e < 32; ++e) x[e] = g * __expf(x[e] - lse);
            }
            const int j = mine - c - h;
            if (j >= 0 && j < 32) {
#pragma unroll
                for (int e = 0; e < 32; ++e)
                    if (e == j) {
                        x[e] -= g;
                        const float r = a.half ? __half2float(__float2half_rn(x[e])) : __bfloat162float(__float2bfloat16_rn(x[e]));
                        const float lost = x[e] - r;
                        a.lost[row0 + lane] = fabsf(lost) < INFINITY ? lost : 0.f;
                    }
            }
            if (!all_live) {
#pragma unroll
                for (int e = 0; e < 32; ++e)
                    if (!live) x[e] = 0.f;
            }
#pragma unroll
            for (int e = 0; e < 32; e += 2) w[(h + e) / 2] = pack2(x[e], x[e + 1], a.half);
        }
        stage_row(part, lane, w);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const int r = 4 * i + (lane >> 3), k = c + 8 * (lane & 7);
            // whole units up to the pitch: what lies past column n is not read
            if (row0 + r < a.m && k < limit)
                *reinterpret_cast<uint4 *>(out + (size_t)r * a.ldo + k) = staged(part, lane, i);
        }
    });
}

// What the one rounding of D took from the tokens' own entries goes back in here. Such an
// entry, about -g, is the largest of its row and of its token's column, and its error is that
// of a whole row of dX and dW: without this the results were off by up to 2.7 times
// what rounding them alone makes (one row), by 1.6 times with equal g; with it by 1.04 (reckoned
// in float64 over 40 seeds a size).
template <bool kRows>
struct Lost {
    const uint16_t *w = nullptr;
    const float *rest = nullptr;
    float by = 0.f;
    __device__ Lost(const ProductArgs &a, int row, bool first_split) {
        if (row >= a.m || !first_split) return;
        if constexpr (kRows) {
            const int64_t at = a.tokens[row] - a.first;
            if (a.tokens[row] < 0 || at < 0 || at >= a.window) return;
            by = a.lost[row];
            if (by != 0.f) w = a.w + at * a.ldw;
        } else {
            const int2 of = a.tally[row];
            if (of.y > 1) rest = a.rest + (size_t)of.x * a.rest_pitch;
            if (of.y != 1) return;
            by = a.lost[of.x];
            if (by != 0.f) w = a.w + of.x * a.ldw;
        }
    }
    // columns k .. k + 31 of a row of n; what is not finite has had its effect
    __device__ void add(float (&x)[32], int k, int n, bool half) const {
        if (w) {
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                uint32_t v[4] = {0, 0, 0, 0};
                if (k + 8 * i + 8 <= n) {
                    const uint4 u = *reinterpret_cast<const uint4 *>(w + k + 8 * i);
                    v[0] = u.x, v[1] = u.y, v[2] = u.z, v[3] = u.w;
                } else {
#pragma unroll
                    for (int e = 0; e < 8; ++e)
                        if (k + 8 * i + e < n) v[e / 2] |= (uint32_t)w[k + 8 * i + e] << (e & 1 ? 16 : 0);
                }
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const uint32_t raw = v[e / 2] >> (e & 1 ? 16 : 0) & 0xFFFFu;
                    const float y = half ? __half2float(__ushort_as_half((unsigned short)raw)) : __uint_as_float(raw << 16);
                    x[8 * i + e] += fabsf(y) < INFINITY ? by * y : 0.f;
                }
            }
        }
        if constexpr (!kRows) {
            if (!rest) return;
#pragma unroll
            for (int e = 0; e < 32; e += 4) {          // its rows are whole units
                if (k + e >= n) break;
                const float4 y = *reinterpret_cast<const float4 *>(rest + k + e);
                x[e] += y.x, x[e + 1] += y.y, x[e + 2] += y.z, x[e + 3] += y.w;
            }
        }
    }
};

// `cols` columns of dX or dW to the result.
template <bool kRows>
__device__ __forceinline__ void drain_result(uint32_t acc, const ProductArgs &a, const Lost<kRows> &lost, int row0, int lane,
                                             int col, int cols, uint32_t part) {
    const int limit = min(cols, a.n - col), rows = a.m - row0;
    const bool vec = ((uintptr_t)a.out & 15) == 0 && a.ldo % 8 == 0;
    const float by = !a.half ? 1.f : ldexpf(1.f, (!kRows ? *a.top : lane < rows ? exponent(a.g[row0 + lane]) : 0) - 14);
    uint16_t *out = static_cast<uint16_t *>(a.out) + (size_t)row0 * a.ldo + col;
#pragma unroll 1
    for (int c = 0; c < limit; c += 64) {
        uint32_t w[32];
#pragma unroll
        for (int h = 0; h < 64; h += 32) {
            float x[32];
            load_columns(acc + c + h, x);
            lost.add(x, col + c + h, a.n, a.half);
#pragma unroll
            for (int e = 0; e < 32; e += 2) w[(h + e) / 2] = pack2(x[e] * by, x[e + 1] * by, a.half);
        }
        stage_row(part, lane, w);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const int r = 4 * i + (lane >> 3), k = c + 8 * (lane & 7);
            if (r >= rows || k >= limit) continue;
            const uint4 u = staged(part, lane, i);
            uint16_t *to = out + (size_t)r * a.ldo + k;
            if (vec && k + 8 <= limit) {
                *reinterpret_cast<uint4 *>(to) = u;
            } else {
                const uint32_t v[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
                for (int e = 0; e < 8; ++e)
                    if (k + e < limit) to[e] = (uint16_t)(v[e / 2] >> (e & 1 ? 16 : 0));
            }
        }
    }
}

// The same to the float32 sums of a split or of several pieces; the last piece's, where
// there is one split, to the result.
template <bool kRows>
__device__ __forceinline__ void drain_sums(uint32_t acc, const ProductArgs &a, const Lost<kRows> &lost, int row0, int lane, int col,
                                           int cols, int split, uint32_t part) {
    const int top = !kRows && a.half ? *a.top : 0;
    const int limit = min(cols, a.n - col);
#pragma unroll 1
    for (int c = 0; c < limit; c += 32) {
        float x[32];
        load_columns(acc + c, x);
        lost.add(x, col + c, a.n, a.half);
        uint32_t w[32];
#pragma unroll
        for (int e = 0; e < 32; ++e) w[e] = __float_as_uint(x[e]);
        stage_row(part, lane, w);
        const int k = col + c + 4 * (lane & 7);
        if (c + 4 * (lane & 7) >= limit) continue;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const int r = row0 + 4 * i + (lane >> 3);
            if (r >= a.m) continue;
            const uint4 u = staged(part, lane, i);
            float y[4] = {__uint_as_float(u.x), __uint_as_float(u.y), __uint_as_float(u.z), __uint_as_float(u.w)};
            float4 *sum = reinterpret_cast<float4 *>(a.slab + ((size_t)split * a.m + r) * a.pitch + k);
            if (a.add) {
                const float4 o = *sum;
                y[0] += o.x, y[1] += o.y, y[2] += o.z, y[3] += o.w;
            }
            if (!a.last) {
                *sum = make_float4(y[0], y[1], y[2], y[3]);
                continue;
            }
            const float by = a.half ? ldexpf(1.f, (kRows ? exponent(a.g[r]) : top) - 14) : 1.f;
            uint16_t *to = static_cast<uint16_t *>(a.out) + (size_t)r * a.ldo + k;
            const uint32_t v[2] = {pack2(y[0] * by, y[1] * by, a.half), pack2(y[2] * by, y[3] * by, a.half)};
#pragma unroll
            for (int e = 0; e < 4; ++e)
                if (k + e < a.n) to[e] = (uint16_t)(v[e / 2] >> (e & 1 ? 16 : 0));
        }
    }
}

// kLong: sums over K are those of several accumulators.  (One alone is read straight from
// where it is: 4286 x 160 -> 36623 with both gradients 334 us, its logits by way of registers
// 348; 2048 x 512 -> 32000 with dX 156 and 164.)  Several logits go to D from the registers, so
// that the next tile has both accumulators: put back into the last, a step of 8192 x 4096 ->
// 32000 took 1.5 % longer.  dX and dW are put back: their epilogue from registers, its code
// unrolled, took 48 x 2048 -> 50001 with dX from 129 to 133 us.
// kStalled: for the self-test, the issuer stops after one tile.
template <Product kWhich, bool kLong, bool kStalled>
__global__ void __cluster_dims__(2, 1, 1) __launch_bounds__(kThreads, 1)
    tc_head_kernel(const __grid_constant__ CUtensorMap mapA, const __grid_constant__ CUtensorMap mapB, ProductArgs a) {
    constexpr uint32_t kPolls = tc::wait_polls(kStalled);
    constexpr bool kAmn = kWhich == kHead, kBmn = kWhich == kHead || kWhich == kHidden;
    extern __shared__ uint8_t smem_raw[];
    uint8_t *smem = (uint8_t *)(((uintptr_t)smem_raw + 1023) & ~(uintptr_t)1023);
    uint64_t *bars = (uint64_t *)(smem + kStages * kStage + kDrainWarps * kPart);
    uint32_t *tmem_slot = (uint32_t *)(bars + kBars);
    volatile int *abort_flag = (volatile int *)(tmem_slot + 1);
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int rank = (int)tc::cluster_rank();
    const int64_t pair = blockIdx.x / 2, npairs = gridDim.x / 2;
    const int64_t units = (int64_t)a.mt * a.nt * a.splits;

    auto full = [&](int s) { return tc::smem_u32(bars + s); };
    auto empty = [&](int s) { return tc::smem_u32(bars + kStages + s); };
    auto afull = [&](int b) { return tc::smem_u32(bars + 2 * kStages + b); };
    auto aempty = [&](int b) { return tc::smem_u32(bars + 2 * kStages + 2 + b); };
    const uint32_t closing = tc::smem_u32(bars + 2 * kStages + 4);
    auto tileA = [&](int s) { return tc::smem_u32(smem + s * kStage); };
    auto tileB = [&](int s) { return tc::smem_u32(smem + s * kStage + kTile); };

    if (threadIdx.x == 0) {
        for (int s = 0; s < kStages; ++s) {
            tc::mbar_init(full(s), 1);      // the even CTA's: bytes of both CTAs
            tc::mbar_init(empty(s), 1);
        }
        for (int b = 0; b < 2; ++b) {
            tc::mbar_init(afull(b), 1);
            tc::mbar_init(aempty(b), 2 * kDrainWarps);   // the even CTA's: both drains
        }
        tc::mbar_init(closing, 1);
        *abort_flag = 0;
        tc::fence_barrier_init();
    }
    if (warp == 1) {
        tc::tmem_alloc_pair(tc::smem_u32(tmem_slot), 512);
        tc::tmem_relinquish_pair();
    }
    if (warp == 0 && lane == 0) {
        tc::prefetch_tmap(&mapA);
        tc::prefetch_tmap(&mapB);
    }
    tc::tc_fence_before();
    __syncthreads();
    tc::cluster_sync();
    tc::tc_fence_after();
    const uint32_t tmem = *tmem_slot;
    // what the launch before this one wrote, if it may still be running
    tc::pdl_launch_dependents();
    tc::pdl_wait();

    if (warp == 0) {
        // ---------------- producer
        bool ok = true;
        const uint32_t full0 = tc::map_rank(full(0), 0);
        // of both CTAs; boxes of an operand along MN are 64 wide whatever the tile
        const int boxes = a.cols > 128 ? 2 : 1;
        // of a single tile's rows only those that there are: the others' places in shared
        // memory hold what they hold, and their sums are not kept
        const bool loadsA = kAmn || a.mt > 1 || 128 * rank < a.m;
        const uint32_t bytesA = kAmn ? 2 * kTile : a.rows * 128 * (a.mt > 1 || a.m > 128 ? 2 : 1);
        const uint32_t bytes = bytesA + 2 * (kBmn ? boxes * kBox : a.cols / 2 * 128);
        Slot<kStages> slot(1);
        int filled = 0;
        for (int64_t u = pair; u < units && ok; u += npairs) {
            const Unit unit(u, a);
            const int ra = unit.ri * 256 + 128 * rank, cb = unit.cj * a.cols + a.cols / 2 * rank;
            const int c1 = min(a.chunks, (unit.split + 1) * a.per);
            for (int c = unit.split * a.per; c < c1; ++c, slot.next()) {
                ok = tc::mbar_wait<kPolls>(empty(slot.s), slot.phase);
                if (!ok) break;
                if (tc::elect_one()) {
                    if (rank == 0) tc::mbar_expect_tx(full(slot.s), bytes);
                    const uint32_t bar = full0 + 8 * slot.s;
                    if (kAmn) {
#pragma unroll
                        for (int m = 0; m < 2; ++m)
                            tc::tma_load_2d_pair(tileA(slot.s) + m * kBox, &mapA, bar, ra + 64 * m, c * 64);
                    } else if (loadsA) {
                        tc::tma_load_2d_pair(tileA(slot.s), &mapA, bar, c * 64, ra);
                    }
                    if (kBmn) {
                        for (int m = 0; m < boxes; ++m)
                            tc::tma_load_2d_pair(tileB(slot.s) + m * kBox, &mapB, bar, cb + 64 * m, c * 64);
                    } else {
                        tc::tma_load_2d_pair(tileB(slot.s), &mapB, bar, c * 64, cb);
                    }
                }
                __syncwarp();
                ++filled;
            }
        }
        // do not leave before the MMAs have consumed the stages filled here:
        // no copy or commit is in flight afterwards
        for (int n = max(0, filled - kStages); n < filled && ok; ++n)
            ok = tc::mbar_wait<kPolls>(empty(n % kStages), (n / kStages) & 1);
        if (!ok) {
            *abort_flag = 1;
            tc::abandon_ring(full(0), kStages, filled, rank == 0);
        }
    } else if (warp == 1) {
        // ---------------- MMA issuer of the pair
        if (rank == 0) {
            bool ok = true;
            const uint64_t a0 = kAmn ? sdesc_mn(tileA(0)) : tc::sdesc_sw128(tileA(0));
            const uint64_t b0 = kBmn ? sdesc_mn(tileB(0)) : tc::sdesc_sw128(tileB(0));
            // 16 of K: 32 bytes along K, two 8-row atoms (2048 bytes) along MN
            constexpr uint64_t kA = kAmn ? 128 : 2, kB = kBmn ? 128 : 2;
            const uint32_t idesc = (a.half ? tc::idesc_f16_f32(256, a.cols) : tc::idesc_bf16_f32(256, a.cols)) |
                                   (kAmn ? 1u << 15 : 0) | (kBmn ? 1u << 16 : 0);
            Slot<kStages> slot(0);
            Slot<2> acc(1);
            for (int64_t u = pair; u < units && ok && !(kStalled && u != pair); u += npairs) {
                const Unit unit(u, a);
                const int first = unit.split * a.per, last = min(a.chunks, first + a.per);
                for (int c = first, c0 = first, c1 = first; c < last && ok; ++c, slot.next()) {
                    if (c == first || c == c1) {
                        // an accumulator's chunks of K begin
                        c0 = c;
                        c1 = kLong ? min(last, c + kSumChunks<kWhich>) : last;
                        ok = tc::mbar_wait<kPolls>(aempty(acc.s), acc.phase);
                        if (!ok) break;
                    }
                    ok = tc::mbar_wait<kPolls>(full(slot.s), slot.phase);
                    if (!ok) break;
                    tc::tc_fence_after();
                    if (tc::elect_one()) {
                        const uint64_t o = (uint64_t)(slot.s * (kStage >> 4));
#pragma unroll
                        for (int sub = 0; sub < 4; ++sub)
                            tc::mma_f16_pair(tmem + acc.s * 256, a0 + o + kA * sub, b0 + o + kB * sub, idesc, c > c0 || sub > 0);
                        tc::mma_commit_pair(empty(slot.s));
                        if (c + 1 == c1) tc::mma_commit_pair(afull(acc.s));
                    }
                    __syncwarp();
                    if (c + 1 == c1) acc.next();
                }
            }
            if (!tc::mma_done_pair<kPolls>(closing, tc::elect_one()) || !ok) *abort_flag = 1;
        }
    } else {
        // ---------------- drain
        const int q = warp & 3, half = (warp - 2) >> 2;   // lane quarter, 128-column half
        const uint32_t released = tc::map_rank(aempty(0), 0);
        const uint32_t part = tc::smem_u32(smem + kStages * kStage + (warp - 2) * kPart);
        bool ok = true;
        Slot<2> acc(0);
        const int cols = a.cols / 2;
        const uint32_t mine = tmem + ((uint32_t)(32 * q) << 16) + half * cols;
        auto filled = [&] {
            const bool in = __all_sync(0xffffffffu, tc::mbar_wait<kPolls>(afull(acc.s), acc.phase));
            if (in) tc::tc_fence_after();
            return in;
        };
        auto release = [&] {
            tc::tc_fence_before();
            __syncwarp();
            if (lane == 0) tc::mbar_arrive_cluster(released + 8 * acc.s);
            acc.next();
        };
        // a unit's sums, in the last of its accumulators
        auto summed = [&](int chunks, bool rows) {
            tc::F2 x[64];
#pragma unroll
            for (int e = 0; e < 64; ++e) x[e] = tc::f2(0.f);
            for (int c = 0;; c += kSumChunks<kWhich>) {
                if (!filled()) return false;
                const bool last = c + kSumChunks<kWhich> >= chunks;
#pragma unroll
                for (int h = 0; h < 128; h += 32) {
                    float v[32];
                    if (h >= cols || !rows) break;
                    load_columns(mine + acc.s * 256 + h, v);
#pragma unroll
                    for (int e = 0; e < 32; e += 2) x[(h + e) / 2] = tc::f2_add(x[(h + e) / 2], tc::f2(v[e], v[e + 1]));
                    if (!last) continue;
#pragma unroll
                    for (int i = 0; i < 32; i += 16) {
                        uint32_t w[16];
                        if (h + i >= cols) break;          // the other half's
#pragma unroll
                        for (int e = 0; e < 16; e += 2) {
                            float lo, hi;
                            tc::f2_get(x[(h + i + e) / 2], lo, hi);
                            w[e] = __float_as_uint(lo), w[e + 1] = __float_as_uint(hi);
                        }
                        tc::tmem_st16(mine + acc.s * 256 + h + i, w);
                    }
                }
                if (last) break;
                release();
            }
            tc::tmem_wait_st();
            return true;
        };
        for (int64_t u = pair; u < units && ok; u += npairs) {
            const Unit unit(u, a);
            const int row0 = unit.ri * 256 + 128 * rank + 32 * q, col = unit.cj * a.cols + half * cols;
            const bool rows = row0 < a.m;          // else nothing is kept of this warp's rows
            if constexpr (kWhich == kLoss || (kWhich == kLogits && kLong)) {
                const RowArgs of(a, row0 + lane, kWhich == kLogits);
                tc::F2 x[64];
#pragma unroll
                for (int e = 0; e < 64; ++e) x[e] = tc::f2(0.f);
                for (int c = 0; c < a.chunks && ok; c += kSumChunks<kWhich>) {
                    ok = filled();
                    if (!ok) break;
#pragma unroll
                    for (int h = 0; h < 128; h += 32) {
                        float v[32];
                        if (h >= cols || !rows) break;
                        load_columns(mine + acc.s * 256 + h, v);
#pragma unroll
                        for (int e = 0; e < 32; e += 2) x[(h + e) / 2] = tc::f2_add(x[(h + e) / 2], tc::f2(v[e], v[e + 1]));
                    }
                    release();
                }
                if (!ok || !rows)
                    ;
                else if (kWhich == kLoss)
                    reduce_loss(x, a, row0 + lane, of.token, col, cols, 2 * unit.cj + half);
                else
                    drain_logits(InRegisters{x}, a, of, row0, lane, col, cols, part);
            } else if constexpr (kWhich == kLogits) {
                const RowArgs of(a, row0 + lane, true);
                ok = filled();
                if (!ok) break;
                if (rows) drain_logits(InTmem{mine + acc.s * 256}, a, of, row0, lane, col, cols, part);
                release();
            } else {
                const Lost<kWhich == kHidden> lost(a, row0 + lane, unit.split == 0);
                ok = kLong ? summed(min(a.chunks, (unit.split + 1) * a.per) - unit.split * a.per, rows) : filled();
                if (!ok) break;
                if (!rows)
                    ;
                else if (a.slab)
                    drain_sums(mine + acc.s * 256, a, lost, row0, lane, col, cols, unit.split, part);
                else
                    drain_result(mine + acc.s * 256, a, lost, row0, lane, col, cols, part);
                release();
            }
        }
        if (!ok) *abort_flag = 1;
    }
    // neither CTA leaves while the other may still read its shared memory,
    // signal its barriers or hold TMEM of the pair
    tc::tc_fence_before();
    __syncwarp();
    __syncthreads();
    tc::cluster_sync();
    if (warp == 1) {
        tc::tc_fence_after();
        tc::tmem_dealloc_pair(tmem, 512);
    }
    if (threadIdx.x == 0 && *abort_flag) {
        *(volatile int *)a.failed = 1;
        __threadfence_system();
    }
}

template <Product kWhich, bool kLong, bool kStalled = false>
cudaError_t launch(const CUtensorMap &a, const CUtensorMap &b, const ProductArgs &args, cudaStream_t s, bool pdl) {
    static std::atomic<unsigned long long> done;
    auto *kernel = tc_head_kernel<kWhich, kLong, kStalled>;
    const cudaError_t e = set_max_dynamic_smem((const void *)kernel, kSmem, done);
    if (e != cudaSuccess) return e;
    const int64_t units = (int64_t)args.mt * args.nt * args.splits;
    return launch_k(kernel, dim3((unsigned)(2 * std::min<int64_t>(units, std::max(1, num_sms() / 2)))), dim3(kThreads),
                    (size_t)kSmem, s, pdl, a, b, args);
}

}  // namespace

cudaError_t launch_product(Product which, const CUtensorMap &a, const CUtensorMap &b, const ProductArgs &args,
                           cudaStream_t s, bool pdl, bool stalled) {
    if (stalled) return launch<kLoss, true, true>(a, b, args, s, pdl);
    auto of = [&](auto product) {
        constexpr Product kWhich = decltype(product)::value;
        return args.per > kSumChunks<kWhich> ? launch<kWhich, true>(a, b, args, s, pdl) : launch<kWhich, kWhich == kLoss>(a, b, args, s, pdl);
    };
    switch (which) {
        case kLoss: return of(std::integral_constant<Product, kLoss>());
        case kLogits: return of(std::integral_constant<Product, kLogits>());
        case kHidden: return of(std::integral_constant<Product, kHidden>());
        default: return of(std::integral_constant<Product, kHead>());
    }
}

}  // namespace head
}  // namespace jarq
