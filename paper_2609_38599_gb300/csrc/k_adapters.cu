// Low-rank adapters of many requests, added to a shared projection's outputs:
//   Y_t = Y0_t + s_i B_i (A_i x_t),   i = ids[t].
// Two kernels: the sums u_t = A_i x_t over the tokens' width, and their expansion by
// B_i with the addition.
//
// Few tokens: dot products, a block a token and a piece of its width (of its outputs);
// an adapter's bytes are read as wide as they lie.
//
// More tokens: first an order in which tokens of one adapter follow one another (a
// token's results do not depend on it: the sums of a row of an MMA are its own), then
// 16 or 32 tokens a warp on mma.sync, whose operands go straight from memory to
// registers: a sum over K does not depend on the order of K, so a lane takes 8
// neighbouring elements of a row (16 bytes) for its share of two MMAs, and the columns
// of the expansion are dealt out so that a lane's results are 8 neighbouring outputs.
// The work is bound by the tokens' and outputs' memory, far below what tensor cores
// could do.  The expansion multiplies u, split into two or three 16-bit parts, with B.
#include <algorithm>

#include "integer.cuh"
#include "rows.cuh"
#include "tc_common.cuh"

namespace jarq {
namespace {

using namespace rows;

constexpr int kMostAdapters = 8192, kMostRank = 128, kMostWidth = 1 << 20;
constexpr int kFew = 64;               // most tokens of the form without MMAs
constexpr int kFewPiece = 512;         // of a token's width, of one block
constexpr int kMostSplits = 16;        // of the width, of the form with MMAs

struct AdapterArgs {
    const void *X, *A, *B, *Y0;
    void *Y;
    const float *scale;
    const int32_t *ids;
    float *u;                 // [splits][n][rank] sums over pieces of the width
    int *order;               // [n] tokens by adapter, or null
    int64_t ldx, ldy0, ldy;
    int n, din, dout, rank, adapters, splits;
    bool vec_x, vec_y;        // rows of X and A, of Y0 and Y on 16-byte boundaries
};

// Elements k .. k + 7 of a row of d: zeros beyond it, which are not read.
template <class T>
__device__ __forceinline__ uint4 load8(const T *p, int k, int d, bool vec) {
    if (vec && k + 8 <= d) return *reinterpret_cast<const uint4 *>(p + k);
    alignas(16) T t[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) t[e] = k + e < d ? p[k + e] : T(0.f);
    return *reinterpret_cast<const uint4 *>(t);
}

__device__ __forceinline__ float warp_sum(float x) {
#pragma unroll
    for (int off = 16; off; off /= 2) x += __shfl_xor_sync(0xffffffffu, x, off);
    return x;
}
// The token's adapter: -1 for none, -2 where there is none of that number.
__device__ __forceinline__ int adapter_of(const AdapterArgs &a, int t) {
    const int i = a.ids[t];
    return i < 0 ? -1 : i >= a.adapters ? -2 : i;
}

// ---------------------------------------------------------------- few tokens
// Piece blockIdx.y of the width of token blockIdx.x: a warp has every 8th row of A.
template <class T>
__global__ void __launch_bounds__(256) few_sums_kernel(AdapterArgs a) {
    tc::pdl_launch_dependents();
    const int t = blockIdx.x, lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int i = adapter_of(a, t);
    if (i < 0) return;
    const T *x = static_cast<const T *>(a.X) + (size_t)t * a.ldx;
    const T *A = static_cast<const T *>(a.A) + (size_t)i * a.rank * a.din;
    const int k0 = blockIdx.y * kFewPiece + 8 * lane;
    float v[kFewPiece / 256][8];
#pragma unroll
    for (int h = 0; h < kFewPiece / 256; ++h) unpack(load8(x, k0 + 256 * h, a.din, a.vec_x), v[h], T());
    for (int j = warp; j < a.rank; j += 8) {
        float sum = 0.f;
#pragma unroll
        for (int h = 0; h < kFewPiece / 256; ++h) {
            float w[8];
            unpack(load8(A + (size_t)j * a.din, k0 + 256 * h, a.din, a.vec_x), w, T());
#pragma unroll
            for (int e = 0; e < 8; ++e) sum = fmaf(v[h][e], w[e], sum);
        }
        sum = warp_sum(sum);
        if (lane == 0) a.u[((size_t)blockIdx.y * a.n + t) * a.rank + j] = sum;
    }
}

// 256 outputs of token blockIdx.x, one a thread.
template <class T, class Out>
__global__ void __launch_bounds__(256) few_outputs_kernel(AdapterArgs a) {
    __shared__ float u[kMostRank], part[256];
    const int t = blockIdx.x, o = blockIdx.y * 256 + threadIdx.x;
    const int i = adapter_of(a, t);
    const float y0 = a.Y0 && o < a.dout ? to_float(static_cast<const Out *>(a.Y0)[(size_t)t * a.ldy0 + o]) : 0.f;
    float y = i == -2 ? __int_as_float(0x7FC00000) : y0;
    tc::pdl_wait();
    if (i >= 0) {
        // the sums over the width's pieces: 256 / rank threads have a rank's
        const int slices = 256 / a.rank, j = threadIdx.x % a.rank, s0 = threadIdx.x / a.rank;
        float sum = 0.f;
        if (s0 < slices)
            for (int s = s0; s < a.splits; s += slices) sum += a.u[((size_t)s * a.n + t) * a.rank + j];
        part[threadIdx.x] = sum;
        __syncthreads();
        if (threadIdx.x < a.rank) {
            sum = 0.f;
            for (int s = 0; s < slices; ++s) sum += part[s * a.rank + threadIdx.x];
            u[threadIdx.x] = sum * (a.scale ? a.scale[i] : 1.f);
        }
        __syncthreads();
        if (o < a.dout) {
            const T *b = static_cast<const T *>(a.B) + ((size_t)i * a.dout + o) * a.rank;
            const bool vec = ((uintptr_t)b & 15) == 0;
            float d = 0.f;
            for (int k = 0; k < a.rank; k += 8) {
                float w[8];
                unpack(load8(b, k, a.rank, vec), w, T());
#pragma unroll
                for (int e = 0; e < 8; ++e) d = fmaf(w[e], u[k + e], d);
            }
            y = y0 + d;
        }
    }
    if (o < a.dout) static_cast<Out *>(a.Y)[(size_t)t * a.ldy + o] = from_float<Out>(y);
}

// ---------------------------------------------------------------- more tokens
// Tokens by adapter, those without one last.  The order of an adapter's tokens is
// any; no result depends on it.
__global__ void __launch_bounds__(1024) order_kernel(AdapterArgs a) {
    tc::pdl_launch_dependents();
    extern __shared__ int bins[];              // adapters + 2
    __shared__ int sums[32];
    const int count = a.adapters + 2, lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    for (int i = threadIdx.x; i < count; i += 1024) bins[i] = 0;
    __syncthreads();
    auto bin = [&](int t) {
        const int i = adapter_of(a, t);
        return i < 0 ? a.adapters - 1 - i : i;
    };
    // one addition for the lanes of a warp that meet in a bin; the first place of these
    auto add = [&](int b, uint32_t among) {
        const uint32_t same = __match_any_sync(among, b);
        const int leader = __ffs(same) - 1;
        int at = 0;
        if (lane == leader) at = atomicAdd(&bins[b], __popc(same));
        return __shfl_sync(same, at, leader) + __popc(same & ((1u << lane) - 1));
    };
    // the first of a thread's tokens stay in registers between the two passes
    constexpr int kKeep = 8;
    int own_bin[kKeep];
#pragma unroll
    for (int i = 0; i < kKeep; ++i) {
        const int t = threadIdx.x + 1024 * i;
        own_bin[i] = t < a.n ? bin(t) : -1;
    }
#pragma unroll
    for (int i = 0; i < kKeep; ++i)
        if (own_bin[i] >= 0) add(own_bin[i], __activemask());
    for (int t = threadIdx.x + 1024 * kKeep; t < a.n; t += 1024) add(bin(t), __activemask());
    __syncthreads();
    // bins to their first places
    int base = 0;
    for (int i0 = 0; i0 < count; i0 += 1024) {
        const int i = i0 + threadIdx.x;
        const int own = i < count ? bins[i] : 0;
        int before = own;
#pragma unroll
        for (int off = 1; off < 32; off *= 2) {
            const int v = __shfl_up_sync(0xffffffffu, before, off);
            if (lane >= off) before += v;
        }
        if (lane == 31) sums[warp] = before;
        __syncthreads();
        int all = sums[lane], mine = all;
#pragma unroll
        for (int off = 1; off < 32; off *= 2) {
            const int v = __shfl_up_sync(0xffffffffu, mine, off);
            if (lane >= off) mine += v;
        }
        const int total = __shfl_sync(0xffffffffu, mine, 31);
        const int warps = __shfl_sync(0xffffffffu, mine - all, warp);
        if (i < count) bins[i] = base + warps + before - own;
        base += total;
        __syncthreads();
    }
#pragma unroll
    for (int i = 0; i < kKeep; ++i)
        if (own_bin[i] >= 0) a.order[add(own_bin[i], __activemask())] = threadIdx.x + 1024 * i;
    for (int t = threadIdx.x + 1024 * kKeep; t < a.n; t += 1024) a.order[add(bin(t), __activemask())] = t;
}

__device__ __forceinline__ void mma(float (&c)[4], const uint32_t (&x)[4], uint32_t b0, uint32_t b1, __half) {
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                 : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
                 : "r"(x[0]), "r"(x[1]), "r"(x[2]), "r"(x[3]), "r"(b0), "r"(b1));
}
__device__ __forceinline__ void mma(float (&c)[4], const uint32_t (&x)[4], uint32_t b0, uint32_t b1, __nv_bfloat16) {
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                 : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
                 : "r"(x[0]), "r"(x[1]), "r"(x[2]), "r"(x[3]), "r"(b0), "r"(b1));
}

// The adapters of a warp's tokens, one after the other: `f(adapter, lanes)` with the
// lanes whose token has it.  All lanes call it; `mine`: this lane's, -1 for none.
template <class F>
__device__ __forceinline__ void each_adapter(int mine, F f) {
    uint32_t left = __ballot_sync(0xffffffffu, mine >= 0);
    while (left) {
        const int i = __shfl_sync(0xffffffffu, mine, __ffs(left) - 1);
        const uint32_t its = __ballot_sync(0xffffffffu, mine == i);
        f(i, its);
        left &= ~its;
    }
}

// u of 16 MT tokens: the 8 warps of a block share a piece of the width; NT: eights of
// the rank (rounded up).
template <class T, int MT, int NT>
__global__ void __launch_bounds__(256) sums_kernel(AdapterArgs a) {
    constexpr int kTokens = 16 * MT, kCols = 8 * NT, kWarps = NT > 8 ? 4 : 8;
    __shared__ float part[kWarps][kTokens][kCols + 1];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, g = lane >> 2, c = lane & 3;
    const int at = blockIdx.x * kTokens;
    tc::pdl_launch_dependents();
    tc::pdl_wait();
    const int tok = lane < kTokens && at + lane < a.n ? a.order[at + lane] : -1;
    const int mine = tok >= 0 ? adapter_of(a, tok) : -1;
    const T *x[2 * MT];
#pragma unroll
    for (int m = 0; m < 2 * MT; ++m) {
        const int t = __shfl_sync(0xffffffffu, tok, 8 * m + g);
        x[m] = t >= 0 ? static_cast<const T *>(a.X) + (size_t)t * a.ldx : nullptr;
    }
    // this split's chunks of 32 of the width, dealt out to the warps
    const int chunks = (a.din + 31) / 32, per = (chunks + a.splits - 1) / a.splits;
    const int c0 = blockIdx.y * per, c1 = min(chunks, c0 + per);
    each_adapter(mine, [&](int i, uint32_t its) {
        const T *A = static_cast<const T *>(a.A) + (size_t)i * a.rank * a.din;
        float acc[MT][NT][4];
#pragma unroll
        for (int m = 0; m < MT; ++m)
#pragma unroll
            for (int j = 0; j < NT; ++j)
#pragma unroll
                for (int e = 0; e < 4; ++e) acc[m][j][e] = 0.f;
        if (warp < kWarps) {
#pragma unroll(NT <= 2 ? 4 : 2)
            for (int ch = c0 + warp; ch < c1; ch += kWarps) {
                const int k = ch * 32 + 8 * c;
                uint4 xv[2 * MT];
#pragma unroll
                for (int m = 0; m < 2 * MT; ++m) xv[m] = x[m] ? load8(x[m], k, a.din, a.vec_x) : make_uint4(0, 0, 0, 0);
                uint4 w[NT];
#pragma unroll
                for (int j = 0; j < NT; ++j)
                    w[j] = 8 * j + g < a.rank ? load8(A + (size_t)(8 * j + g) * a.din, k, a.din, a.vec_x) : make_uint4(0, 0, 0, 0);
#pragma unroll
                for (int m = 0; m < MT; ++m) {
                    const uint32_t lo[4] = {xv[2 * m].x, xv[2 * m + 1].x, xv[2 * m].y, xv[2 * m + 1].y};
                    const uint32_t hi[4] = {xv[2 * m].z, xv[2 * m + 1].z, xv[2 * m].w, xv[2 * m + 1].w};
#pragma unroll
                    for (int j = 0; j < NT; ++j) {
                        mma(acc[m][j], lo, w[j].x, w[j].y, T());
                        mma(acc[m][j], hi, w[j].z, w[j].w, T());
                    }
                }
            }
#pragma unroll
            for (int m = 0; m < MT; ++m)
#pragma unroll
                for (int j = 0; j < NT; ++j)
#pragma unroll
                    for (int e = 0; e < 4; ++e) part[warp][16 * m + g + 8 * (e / 2)][8 * j + 2 * c + e % 2] = acc[m][j][e];
        }
        __syncthreads();
        for (int e = threadIdx.x; e < kTokens * kCols; e += 256) {
            const int r = e / kCols, j = e % kCols;
            if (!(its >> r & 1) || j >= a.rank) continue;
            float sum = 0.f;
#pragma unroll
            for (int w = 0; w < kWarps; ++w) sum += part[w][r][j];
            a.u[((size_t)blockIdx.y * a.n + a.order[at + r]) * a.rank + j] = sum;
        }
        __syncthreads();
    });
}

// u in 16-bit parts: x = x_0 + x_1 (+ x_2) to 2^-22 (2^-24).
template <int PARTS, class T>
__device__ __forceinline__ void split(float lo, float hi, uint32_t (&out)[PARTS]) {
#pragma unroll
    for (int p = 0; p < PARTS; ++p) {
        alignas(4) T h[2] = {from_float<T>(lo), from_float<T>(hi)};
        out[p] = *reinterpret_cast<const uint32_t *>(h);
        lo -= to_float(h[0]);
        hi -= to_float(h[1]);
    }
}

// 16 neighbouring outputs of a token, from element o on: the sums d to what Y0 has
// there. `held`: Y0's, read before, where the outputs are whole 16 bytes.
template <class Out>
constexpr int kHeld16 = 16 / kUnit<Out>;
template <class Out>
__device__ __forceinline__ void put16(Out *y, const Out *y0, const uint4 (&held)[kHeld16<Out>], bool vec, int left,
                                      const float (&d)[16]) {
    constexpr int E = kUnit<Out>;
    if (vec && left >= 16) {
#pragma unroll
        for (int h = 0; h < kHeld16<Out>; ++h) {
            float v[E];
            unpack(held[h], v, Out());
#pragma unroll
            for (int e = 0; e < E; ++e) v[e] += d[E * h + e];
            *reinterpret_cast<uint4 *>(y + E * h) = pack(v, Out());
        }
    } else {
#pragma unroll
        for (int e = 0; e < 16; ++e)
            if (e < left) y[e] = from_float<Out>((y0 ? to_float(y0[e]) : 0.f) + d[e]);
    }
}

// Outputs of 16 MT tokens a block: each of its warps has 64 of every 256 columns, a
// lane 16 neighbours of a token; KS: sixteens of the rank.
template <class T, class Out, int MT, int KS, int PARTS>
__global__ void __launch_bounds__(128) outputs_kernel(AdapterArgs a, int columns) {
    constexpr int kTokens = 16 * MT;
    constexpr bool kHalf = std::is_same_v<T, __half>;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, g = lane >> 2, c = lane & 3;
    const int at = blockIdx.x * kTokens;
    tc::pdl_wait();
    const int tok = lane < kTokens && at + lane < a.n ? a.order[at + lane] : -1;
    const int mine = tok >= 0 ? adapter_of(a, tok) : -3;
    const int o0 = blockIdx.y * columns + 64 * warp, o1 = min(a.dout, (int)(blockIdx.y + 1) * columns);
    int t[2 * MT], id[2 * MT];
    uint32_t u[MT][KS][PARTS][4];
    float back[2 * MT];
#pragma unroll
    for (int m = 0; m < 2 * MT; ++m) {
        t[m] = __shfl_sync(0xffffffffu, tok, 8 * m + g);
        id[m] = __shfl_sync(0xffffffffu, mine, 8 * m + g);
        float v[KS][4], top = 0.f;
        const float by = id[m] >= 0 && a.scale ? a.scale[id[m]] : 1.f;
#pragma unroll
        for (int k = 0; k < KS; ++k) {
            const int j = 16 * k + 4 * c;
            float4 s = make_float4(0.f, 0.f, 0.f, 0.f);
            if (id[m] >= 0 && j < a.rank)
                for (int p = 0; p < a.splits; ++p) {
                    const float4 q = *reinterpret_cast<const float4 *>(a.u + ((size_t)p * a.n + t[m]) * a.rank + j);
                    s.x += q.x, s.y += q.y, s.z += q.z, s.w += q.w;
                }
            v[k][0] = s.x * by, v[k][1] = s.y * by, v[k][2] = s.z * by, v[k][3] = s.w * by;
#pragma unroll
            for (int e = 0; e < 4; ++e) top = fmaxf(top, fabsf(v[k][e]));
        }
        back[m] = 1.f;
        if (kHalf) {
            // into float16's range by a power of two
            top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 1));
            top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 2));
            const int e = (int)(__float_as_uint(top) >> 23) - 127;
            if (e > -100 && e < 100) {
                back[m] = ldexpf(1.f, e);
                const float down = ldexpf(1.f, -e);
#pragma unroll
                for (int k = 0; k < KS; ++k)
#pragma unroll
                    for (int q = 0; q < 4; ++q) v[k][q] *= down;
            }
        }
#pragma unroll
        for (int k = 0; k < KS; ++k) {
            uint32_t p0[PARTS], p1[PARTS];
            split<PARTS, T>(v[k][0], v[k][1], p0);
            split<PARTS, T>(v[k][2], v[k][3], p1);
#pragma unroll
            for (int p = 0; p < PARTS; ++p) {
                u[m / 2][k][p][m % 2] = p0[p];
                u[m / 2][k][p][2 + m % 2] = p1[p];
            }
        }
    }
    const Out *Y0 = static_cast<const Out *>(a.Y0);
    Out *Y = static_cast<Out *>(a.Y);
    // Y0's 16 of token t[m]
    auto hold = [&](int m, int o, uint4 (&held)[kHeld16<Out>]) {
#pragma unroll
        for (int h = 0; h < kHeld16<Out>; ++h)
            held[h] = Y0 && a.vec_y && o + 16 <= o1
                          ? *reinterpret_cast<const uint4 *>(Y0 + (size_t)t[m] * a.ldy0 + o + kUnit<Out> * h)
                          : make_uint4(0, 0, 0, 0);
    };
    auto put = [&](int m, int o, const uint4 (&held)[kHeld16<Out>], const float (&d)[16]) {
        put16<Out>(Y + (size_t)t[m] * a.ldy + o, Y0 ? Y0 + (size_t)t[m] * a.ldy0 + o : nullptr, held, a.vec_y, o1 - o, d);
    };
    each_adapter(mine, [&](int i, uint32_t its) {
        const T *B = static_cast<const T *>(a.B) + (size_t)i * a.dout * a.rank;
        const bool vec = ((uintptr_t)B & 7) == 0;
        for (int o = o0; o < o1; o += 256) {
            const int mo = o + 16 * c;             // this lane's outputs
            uint4 held[2 * MT][kHeld16<Out>];
#pragma unroll
            for (int m = 0; m < 2 * MT; ++m)
                if (id[m] == i) hold(m, mo, held[m]);
            float acc[MT][8][4];
#pragma unroll
            for (int m = 0; m < MT; ++m)
#pragma unroll
                for (int q = 0; q < 8; ++q)
#pragma unroll
                    for (int e = 0; e < 4; ++e) acc[m][q][e] = 0.f;
#pragma unroll
            for (int k = 0; k < KS; ++k) {
                const int j = 16 * k + 4 * c;
                uint2 b[8];
#pragma unroll
                for (int q = 0; q < 8; ++q) {
                    // column g of MMA q is output 16 (g / 2) + 2 q + g % 2: a lane's two
                    // of each of the eight are 16 neighbours
                    const int col = o + 16 * (g >> 1) + 2 * q + (g & 1);
                    b[q] = make_uint2(0, 0);
                    if (j < a.rank && col < o1) {
                        const T *p = B + (size_t)col * a.rank + j;
                        if (vec) {
                            b[q] = *reinterpret_cast<const uint2 *>(p);
                        } else {
                            alignas(8) T v[4] = {p[0], p[1], p[2], p[3]};
                            b[q] = *reinterpret_cast<const uint2 *>(v);
                        }
                    }
                }
#pragma unroll
                for (int q = 0; q < 8; ++q)
#pragma unroll
                    for (int m = 0; m < MT; ++m)
#pragma unroll
                        for (int p = 0; p < PARTS; ++p) mma(acc[m][q], u[m][k][p], b[q].x, b[q].y, T());
            }
#pragma unroll
            for (int m = 0; m < 2 * MT; ++m) {
                if (id[m] != i || mo >= o1) continue;
                float d[16];
#pragma unroll
                for (int q = 0; q < 8; ++q) {
                    d[2 * q] = acc[m / 2][q][2 * (m % 2)] * back[m];
                    d[2 * q + 1] = acc[m / 2][q][2 * (m % 2) + 1] * back[m];
                }
                put(m, mo, held[m], d);
            }
        }
    });
    // tokens without an adapter, and those of one that there is not
#pragma unroll
    for (int m = 0; m < 2 * MT; ++m) {
        if (id[m] != -1 && id[m] != -2) continue;
        float d[16];
#pragma unroll
        for (int e = 0; e < 16; ++e) d[e] = id[m] == -1 ? 0.f : __int_as_float(0x7FC00000);
        for (int o = o0 + 16 * c; o < o1; o += 256) {
            uint4 held[kHeld16<Out>];
            hold(m, o, held);
            put(m, o, held, d);
        }
    }
}

int ceil_div(int64_t a, int64_t b) { return (int)((a + b - 1) / b); }

int few_splits(int din) { return ceil_div(din, kFewPiece); }
// Splits of the width where there are few tiles of tokens.
int many_splits(int n, int din, int rank) {
    // as many blocks as run at one time
    const int tiles = ceil_div(n, 16), at_once = 152 * (rank <= 16 ? 4 : rank <= 64 ? 2 : 1);
    return std::max(1, std::min({at_once / tiles, ceil_div(din, 512), kMostSplits}));
}

template <class T, class Out>
cudaError_t launch_few(const AdapterArgs &a, cudaStream_t s) {
    few_sums_kernel<T><<<dim3(a.n, a.splits), 256, 0, s>>>(a);
    cudaError_t e = cudaGetLastError();
    if (e == cudaSuccess) e = launch_pdl(few_outputs_kernel<T, Out>, dim3(a.n, ceil_div(a.dout, 256)), dim3(256), 0, s, a);
    count_launches(2);
    return e;
}

template <class T, class Out, int MT, int KS>
cudaError_t launch_many_as(const AdapterArgs &a, cudaStream_t s) {
    constexpr int kParts = std::is_same_v<Out, float> && std::is_same_v<T, __nv_bfloat16> ? 3 : 2;
    order_kernel<<<1, 1024, (a.adapters + 2) * sizeof(int), s>>>(a);
    cudaError_t e = cudaGetLastError();
    const int tiles = ceil_div(a.n, 16 * MT);
    if (e == cudaSuccess)
        e = launch_pdl(sums_kernel<T, 1, 2 * KS>, dim3(ceil_div(a.n, 16), a.splits), dim3(256), 0, s, a);
    // columns of a block: enough blocks for the machine, in whole steps of 256
    const int columns = std::max(256, std::min(1024, round_up(ceil_div((int64_t)a.dout * tiles, 6 * 152), 256)));
    if (e == cudaSuccess)
        e = launch_pdl(outputs_kernel<T, Out, MT, KS, kParts>, dim3(tiles, ceil_div(a.dout, columns)), dim3(128), 0, s, a, columns);
    count_launches(3);
    return e;
}
template <class T, class Out>
cudaError_t launch_many(const AdapterArgs &a, cudaStream_t s) {
    if (a.rank <= 16) return launch_many_as<T, Out, 2, 1>(a, s);
    if (a.rank <= 32) return launch_many_as<T, Out, 2, 2>(a, s);
    if (a.rank <= 64) return launch_many_as<T, Out, 1, 4>(a, s);
    return launch_many_as<T, Out, 1, 8>(a, s);
}

bool is_aligned(const void *p, size_t b) { return ((uintptr_t)p & (b - 1)) == 0; }
bool usable(const void *p, size_t size) { return p && on_device(p) && is_aligned(p, size); }

}  // namespace
}  // namespace jarq

using namespace jarq;

extern "C" {

size_t jarq_adapters_workspace(int n, int din, int rank) {
    if (n < 1 || n > kMostIndex || din < 1 || din > kMostWidth || rank < 8 || rank > kMostRank || rank % 8) return 0;
    if (n <= kFew) return (size_t)few_splits(din) * n * rank * sizeof(float);
    return (size_t)many_splits(n, din, rank) * n * rank * sizeof(float) + (size_t)n * sizeof(int);
}

jarq_status jarq_apply_adapters(const void *X, jarq_dtype dtype, int64_t ldx, const void *A, const void *B,
                                const float *scale, int adapters, int rank, const int32_t *ids, int n,
                                int din, int dout, const void *Y0, int64_t ldy0, void *Y, int64_t ldy,
                                jarq_dtype ydtype, void *workspace, size_t workspace_bytes, void *stream) {
    if ((dtype != JARQ_F16 && dtype != JARQ_BF16) || (ydtype != dtype && ydtype != JARQ_F32)) return JARQ_ERR_ARG;
    if (n < 0 || n > kMostIndex || din < 1 || din > kMostWidth || dout < 1 || dout > kMostWidth || ldx < din || ldy < dout ||
        (Y0 && ldy0 < dout) || adapters < 0 || adapters > kMostAdapters || rank < 8 || rank > kMostRank || rank % 8 ||
        (Y0 == Y && Y && n > 1 && ldy0 != ldy))
        return JARQ_ERR_ARG;
    if (n == 0) return JARQ_OK;
    const size_t ysize = size_of(ydtype);
    if (!usable(X, 2) || !usable(ids, 4) || !usable(Y, ysize) || (Y0 && !usable(Y0, ysize)) || (scale && !usable(scale, 4)))
        return JARQ_ERR_ARG;
    if (adapters && (!usable(A, 2) || !usable(B, 2))) return JARQ_ERR_ARG;
    if (!usable(workspace, 16) || workspace_bytes < jarq_adapters_workspace(n, din, rank)) return JARQ_ERR_ARG;
    if (const jarq_status late = async_failure()) return late;
    cudaStream_t st = (cudaStream_t)stream;
    const bool few = n <= kFew;
    AdapterArgs a{X, A, B, Y0, Y, scale, ids, static_cast<float *>(workspace), nullptr, ldx, ldy0, ldy, n, din, dout, rank,
                  adapters, few ? few_splits(din) : many_splits(n, din, rank)};
    if (!few) a.order = reinterpret_cast<int *>(a.u + (size_t)a.splits * n * rank);
    a.vec_x = is_aligned(X, 16) && is_aligned(A, 16) && din % 8 == 0 && (n == 1 || ldx % 8 == 0);
    auto rows16 = [&](const void *p, int64_t ld) { return is_aligned(p, 16) && (n == 1 || ld * (int64_t)ysize % 16 == 0); };
    a.vec_y = rows16(Y, ldy) && (!Y0 || rows16(Y0, ldy0));
    ProfScope ps("adapters", st);
    const cudaError_t e = with_type(dtype, [&](auto type) {
        using T = decltype(type);
        if constexpr (std::is_same_v<T, float>) {
            return cudaErrorInvalidValue;
        } else if (ydtype == JARQ_F32) {
            return few ? launch_few<T, float>(a, st) : launch_many<T, float>(a, st);
        } else {
            return few ? launch_few<T, T>(a, st) : launch_many<T, T>(a, st);
        }
    });
    ps.done();
    if (e == cudaSuccess) return JARQ_OK;
    (void)cudaGetLastError();
    return JARQ_ERR_CUDA;
}

}  // extern "C"
