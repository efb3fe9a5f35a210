// Low-rank adapters of many requests, added to a shared projection's outputs:
//   Y_t = Y0_t + s_i B_i (A_i x_t),   i = ids[t].
//
// Few tokens: dot products, a cluster of CTAs a token, in one launch.
//
// More tokens: tiles of 16 of one adapter (order_kernel), then two kernels, the sums u_t =
// A_i x_t over the tokens' width and their expansion by B_i with the addition.  Bound by
// the tokens' and outputs' memory, far below what tensor cores could do, and an adapter's
// tile is too small to fill tcgen05's 128 rows: mma.sync, a warp 16 tokens.  A sum over K
// does not depend on the order of K, so a lane takes 8 neighbouring elements of a row for
// its share of two MMAs, and the columns of the expansion are dealt out so that a lane's
// results are 16 bytes of a token.  u is split into 16-bit parts for the expansion, two of
// float16 and three of bfloat16, and so kept to 2^-22 of a token's largest whatever the
// outputs' type: B's terms may cancel one another or Y0.
//
// On the device, cold: 8192 tokens 4096 -> 4096 of rank 16 in bfloat16, six adapters, 48.5
// to 49 us (201 MB; each launch alone under a profiler: order 9, sums 15 at 4.4 TB/s, outputs
// 25 at 5.2), of rank 64 94; 276 x 4236 -> 2009, rank 8, float32 outputs, rows on no boundary
// 23 us; 2392 x 992 -> 745, rank 64, 38 adapters in any order, float32 41 us.  With two parts of
// bfloat16 for three 0.5 us less, of rank 64 7.  States on the way, which
// differ in more than one thing each: operands straight into a lane's registers 74 to 103
// us, into places of each lane's own in shared memory 87, tiles of one adapter instead
// of two walked one after the other (the other blocks had ended) 61, whole lines 53.
#include <algorithm>

#include "integer.cuh"
#include "rows.cuh"
#include "tc_common.cuh"

namespace jarq {
namespace {

using namespace rows;

constexpr int kMostAdapters = 8192, kMostRank = 128, kMostWidth = 1 << 20, kMostTokens = 1 << 30;
constexpr int kFew = 64;               // most tokens of the form without MMAs
constexpr int kFewPiece = 512;         // of a token's width, of one block
constexpr int kMostSplits = 16;        // of the width, of the form with MMAs

struct AdapterArgs {
    const void *X, *A, *B, *Y0;
    void *Y;
    const float *scale;
    const int32_t *ids;
    float *u;                 // [splits][n][rank] sums over pieces of the width
    int *order;               // tokens by adapter (order_kernel), or null
    int64_t ldx, ldy0, ldy;
    int n, din, dout, rank, adapters, splits;
    bool vec_x, vec_y;        // rows of X and A, of Y0 and Y on 16-byte boundaries
};

// 16 bytes to shared memory, and the last copies but LEFT groups of them landed
__device__ __forceinline__ void copy_ahead(uint32_t to, const void *from) {
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(to), "l"(from) : "memory");
}
__device__ __forceinline__ void copies_made() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int LEFT>
__device__ __forceinline__ void copies_landed() {
    asm volatile("cp.async.wait_group %0;" ::"n"(LEFT) : "memory");
}

// Elements k .. k + 7 of a row of d: zeros beyond it, which are not read.  vec: the row
// and k are multiples of 16 bytes; otherwise whole words inside the row are read and
// shifted, and single elements at its ends.
template <class T>
__device__ __forceinline__ uint4 load8(const T *p, int k, int d, bool vec) {
    if (vec && k + 8 <= d) return *reinterpret_cast<const uint4 *>(p + k);
    if (!vec && k > 0 && k + 8 < d) {
        const uint32_t odd = (uint32_t)((uintptr_t)(p + k) & 2), sel = odd ? 0x5432 : 0x3210;
        const uint32_t *q = reinterpret_cast<const uint32_t *>(reinterpret_cast<uintptr_t>(p + k) & ~(uintptr_t)3);
        uint32_t w[5];
#pragma unroll
        for (int i = 0; i < 4; ++i) w[i] = q[i];
        w[4] = odd ? q[4] : 0;
        return make_uint4(__byte_perm(w[0], w[1], sel), __byte_perm(w[1], w[2], sel), __byte_perm(w[2], w[3], sel),
                          __byte_perm(w[3], w[4], sel));
    }
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
// The CTAs of a cluster share a token: pieces of its width, then, with the sums of all
// of them, pieces of its outputs.  Bound by latencies (first loads, cluster's join, B's
// loads) and, outside a graph, by the host: one token 4096 -> 11008 of rank 16 takes 5.9
// to 8.0 us on the device, by the machine, a call 20.  In two launches with the sums in memory
// between them it took 4.6 and 26.  48 tokens 11008 -> 4096 8.1 to 11.1 us, 8.4 in two on
// the machine of the 8.1.
__device__ __forceinline__ void cluster_arrive() { asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory"); }
__device__ __forceinline__ void cluster_wait() { asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory"); }
__device__ __forceinline__ float load_peer(const float *p, uint32_t rank) {
    float v;
    asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(v) : "r"(tc::map_rank(tc::smem_u32(p), rank)) : "memory");
    return v;
}

// kThreads: 512 where the CTAs leave SMs idle, with B on its way to L2 under the sums; a
// row's sum is the same.
template <class T, class Out, int kThreads>
__global__ void __launch_bounds__(kThreads) few_kernel(AdapterArgs a, int ctas) {
    constexpr int kWarps = kThreads / 32, kH = kFewPiece / 256;
    __shared__ float mine[kMostRank], u[kMostRank];
    const int t = blockIdx.x / ctas, part = blockIdx.x % ctas, lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int i = adapter_of(a, t);            // of all of the cluster
    const Out *y0 = static_cast<const Out *>(a.Y0) + (size_t)t * a.ldy0;
    Out *y = static_cast<Out *>(a.Y) + (size_t)t * a.ldy;
    const T *B = static_cast<const T *>(a.B) + (size_t)max(i, 0) * a.dout * a.rank;
    const int first = part * kThreads + threadIdx.x, step = ctas * kThreads;   // outputs
    if (i >= 0) {
        for (int o = first; kThreads == 512 && o < a.dout; o += step)
            for (int k = 0; k < a.rank; k += 64)
                asm volatile("prefetch.global.L2 [%0];" ::"l"(B + (size_t)o * a.rank + k) : "memory");
        const T *x = static_cast<const T *>(a.X) + (size_t)t * a.ldx;
        const T *A = static_cast<const T *>(a.A) + (size_t)i * a.rank * a.din;
        for (int k0 = part * kFewPiece; k0 < a.din || k0 == part * kFewPiece; k0 += ctas * kFewPiece) {
            const int k = k0 + 8 * lane;
            uint4 raw[kH];
#pragma unroll
            for (int h = 0; h < kH; ++h) raw[h] = load8(x, k + 256 * h, a.din, a.vec_x);
            // a warp has every kWarps-th row of A, two at a time
            for (int j = warp; j < a.rank; j += 2 * kWarps) {
                const bool two = j + kWarps < a.rank;
                uint4 w[2][kH];
#pragma unroll
                for (int r = 0; r < 2; ++r)
#pragma unroll
                    for (int h = 0; h < kH; ++h)
                        w[r][h] = r && !two ? make_uint4(0, 0, 0, 0)
                                            : load8(A + (size_t)(j + r * kWarps) * a.din, k + 256 * h, a.din, a.vec_x);
                float sum[2] = {0.f, 0.f};
#pragma unroll
                for (int h = 0; h < kH; ++h) {
                    float v[8];
                    unpack(raw[h], v, T());
#pragma unroll
                    for (int r = 0; r < 2; ++r) {
                        float q[8];
                        unpack(w[r][h], q, T());
#pragma unroll
                        for (int e = 0; e < 8; ++e) sum[r] = fmaf(v[e], q[e], sum[r]);
                    }
                }
#pragma unroll
                for (int r = 0; r < 2; ++r) {
                    const int row = j + r * kWarps;
                    sum[r] = warp_sum(sum[r]);
                    if (lane == 0 && (r == 0 || two)) mine[row] = (k0 == part * kFewPiece ? 0.f : mine[row]) + sum[r];
                }
            }
        }
    }
    __syncthreads();
    cluster_arrive();
    cluster_wait();
    if (i >= 0 && threadIdx.x < a.rank) {
        float sum = 0.f;
        for (int c = 0; c < ctas; ++c) sum += load_peer(mine + threadIdx.x, c);
        u[threadIdx.x] = sum * (a.scale ? a.scale[i] : 1.f);
    }
    __syncthreads();
    cluster_arrive();                          // no CTA leaves while another reads its sums
    const bool vec = ((uintptr_t)B & 15) == 0;
#pragma unroll 2
    for (int o = first; o < a.dout; o += step) {
        float v = a.Y0 ? to_float(y0[o]) : 0.f;
        if (i >= 0) {
            const T *b = B + (size_t)o * a.rank;
            float d = 0.f;
            for (int k = 0; k < a.rank; k += 16) {
                const bool two = k + 8 < a.rank;
                const uint4 raw[2] = {load8(b, k, a.rank, vec), two ? load8(b, k + 8, a.rank, vec) : make_uint4(0, 0, 0, 0)};
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    if (h && !two) break;
                    float w[8];
                    unpack(raw[h], w, T());
#pragma unroll
                    for (int e = 0; e < 8; ++e) d = fmaf(w[e], u[k + 8 * h + e], d);
                }
            }
            v += d;
        }
        y[o] = from_float<Out>(i == -2 ? __int_as_float(0x7FC00000) : v);
    }
    __syncwarp();
    cluster_wait();
}

// ---------------------------------------------------------------- more tokens
// Tokens by adapter, each adapter's from a multiple of 16 on, so that a tile of 16 has
// one adapter (a tile of two would take twice as long, and the others wait for it);
// places that are left hold -1.  order[0]: tiles; then from 16 on the tokens of each and
// its adapter, 17 a tile.  Tokens without an adapter are last.  The order of an adapter's tokens is any; no result depends on it.
int tiles_at_most(int n, int adapters) { return (int)std::min<int64_t>(n, ((int64_t)n + 15) / 16 + std::min(n, adapters + 2)); }

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
    // one addition for the lanes of a warp that meet in a bin; this lane's place
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
    for (int64_t t = threadIdx.x + 1024 * kKeep; t < a.n; t += 1024) add(bin((int)t), __activemask());
    __syncthreads();
    // bins to their first places
    int *order = a.order + 16;
    int base = 0;
    for (int i0 = 0; i0 < count; i0 += 1024) {
        const int i = i0 + threadIdx.x;
        const int tokens = i < count ? bins[i] : 0, own = (tokens + 15) & ~15;
        int before = own;
#pragma unroll
        for (int off = 1; off < 32; off *= 2) {
            const int v = __shfl_up_sync(0xffffffffu, before, off);
            if (lane >= off) before += v;
        }
        if (lane == 31) sums[warp] = before;
        __syncthreads();
        const int all = sums[lane];
        int upto = all;
#pragma unroll
        for (int off = 1; off < 32; off *= 2) {
            const int v = __shfl_up_sync(0xffffffffu, upto, off);
            if (lane >= off) upto += v;
        }
        const int total = __shfl_sync(0xffffffffu, upto, 31);
        const int warps = __shfl_sync(0xffffffffu, upto - all, warp);
        const int first = base + warps + before - own;
        if (i < count) bins[i] = first;
        for (int k = tokens; k < own; ++k) order[(first + k) / 16 * 17 + (first + k) % 16] = -1;
        for (int k = first / 16; k < (first + own) / 16; ++k) order[17 * k + 16] = i < a.adapters ? i : a.adapters - 1 - i;
        base += total;
        __syncthreads();
    }
    if (threadIdx.x == 0) a.order[0] = base / 16;
    auto put = [&](int at, int t) { order[at / 16 * 17 + at % 16] = t; };
#pragma unroll
    for (int i = 0; i < kKeep; ++i)
        if (own_bin[i] >= 0) put(add(own_bin[i], __activemask()), threadIdx.x + 1024 * i);
    for (int64_t t = threadIdx.x + 1024 * kKeep; t < a.n; t += 1024) put(add(bin((int)t), __activemask()), (int)t);
}

// A tile's tokens and their adapter.
struct Tile {
    int tok;             // of lanes 0 .. 15, -1 for none
    int adapter;         // -1: none, -2: there is none of that number, -3: no tile
    __device__ explicit Tile(const AdapterArgs &a) {
        const int lane = threadIdx.x & 31;
        const int v = lane < 17 ? a.order[16 + (size_t)blockIdx.x * 17 + lane] : -1;
        adapter = __shfl_sync(0xffffffffu, v, 16);
        tok = lane < 16 ? v : -1;
        if ((int)blockIdx.x >= a.order[0]) adapter = -3;
    }
};

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

// Rings.  A warp copies what it will multiply into shared memory of its own, some steps
// ahead, whole 128-byte lines at a time (a lane's own share of the lines, straight into
// registers or places of its own, is 64 of them: twice as much work for the L1, which
// was the bound).  Rows of a line's length lie one after the other with every odd one's
// halves exchanged, so that the two rows that eight lanes read are in different banks.
__device__ __forceinline__ uint32_t line_place(int row, int unit) { return row * 128 + ((unit ^ ((row & 1) << 2)) << 4); }
__device__ __forceinline__ uint4 shared16(uint32_t at) {
    uint4 v;
    asm volatile("ld.shared.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(at) : "memory");
    return v;
}
__device__ __forceinline__ uint2 shared8(uint32_t at) {
    uint2 v;
    asm volatile("ld.shared.v2.u32 {%0, %1}, [%2];" : "=r"(v.x), "=r"(v.y) : "r"(at) : "memory");
    return v;
}

// u of 16 tokens: a block's warps share a piece of the width, in chunks of 64.  NT: eights
// of the rank, rounded up.
constexpr int kSumWarps = 4;
__host__ __device__ constexpr int sum_stage(int nt) { return (16 + 8 * nt) * 128; }
__host__ __device__ constexpr int sum_stages(int nt) { return nt <= 4 ? 3 : 2; }
__host__ __device__ constexpr int sum_shared(int nt) {
    const int ring = kSumWarps * sum_stages(nt) * sum_stage(nt), part = kSumWarps * 16 * (8 * nt + 1) * 4;
    return ring > part ? ring : part;
}
// of an SM, by shared memory
constexpr int sum_blocks(int nt) { return 220 * 1024 / (sum_shared(nt) + 1024); }

template <class T, int NT>
__global__ void __launch_bounds__(32 * kSumWarps) sums_kernel(AdapterArgs a) {
    constexpr int kCols = 8 * NT, kStages = sum_stages(NT);
    extern __shared__ uint4 ring[];
    float(*part)[16][kCols + 1] = reinterpret_cast<float(*)[16][kCols + 1]>(ring);
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, g = lane >> 2, c = lane & 3;
    tc::pdl_launch_dependents();
    tc::pdl_wait();
    const Tile tile(a);
    if (tile.adapter < 0) return;
    // this split's chunks, dealt out to the warps
    const int chunks = (a.din + 63) / 64, per = (chunks + a.splits - 1) / a.splits;
    const int c0 = blockIdx.y * per, c1 = min(chunks, c0 + per), whole = a.vec_x ? min(c1, a.din / 64) : c0;
    const T *X = static_cast<const T *>(a.X), *A = static_cast<const T *>(a.A) + (size_t)tile.adapter * a.rank * a.din;
    float acc[NT][4];
#pragma unroll
    for (int j = 0; j < NT; ++j)
#pragma unroll
        for (int e = 0; e < 4; ++e) acc[j][e] = 0.f;
    auto multiply = [&](const uint4 (&xv)[2], int j, const uint4 &w) {
        const uint32_t lo[4] = {xv[0].x, xv[1].x, xv[0].y, xv[1].y}, hi[4] = {xv[0].z, xv[1].z, xv[0].w, xv[1].w};
        mma(acc[j], lo, w.x, w.y, T());
        mma(acc[j], hi, w.z, w.w, T());
    };
    const uint32_t room = tc::smem_u32(ring) + warp * kStages * sum_stage(NT);
    // four rows a copy: this lane has unit lane % 8 of rows 4 i + lane / 8
    const int unit = lane & 7, quarter = lane >> 3;
    const T *x[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int t = __shfl_sync(0xffffffffu, tile.tok, 4 * i + quarter);
        x[i] = X + (size_t)max(t, 0) * a.ldx + 8 * unit;             // sums past the tokens are not kept
    }
    auto ahead = [&](int ch, int s) {
        if (ch < whole) {
            const uint32_t to = room + s * sum_stage(NT);
#pragma unroll
            for (int i = 0; i < 4; ++i) copy_ahead(to + line_place(4 * i + quarter, unit), x[i] + ch * 64);
#pragma unroll
            for (int i = 0; i < 2 * NT; ++i)
                if (4 * i < a.rank)
                    copy_ahead(to + line_place(16 + 4 * i + quarter, unit), A + (size_t)(4 * i + quarter) * a.din + ch * 64 + 8 * unit);
        }
        copies_made();
    };
    int ch = c0 + warp;
#pragma unroll
    for (int s = 0; s + 1 < kStages; ++s) ahead(ch + s * kSumWarps, s);
    int s = 0;
#pragma unroll 1
    for (; ch < whole; ch += kSumWarps) {
        __syncwarp();                          // all lanes have read the stage that is filled next
        ahead(ch + (kStages - 1) * kSumWarps, s == 0 ? kStages - 1 : s - 1);
        copies_landed<kStages - 1>();
        __syncwarp();
        const uint32_t at = room + s * sum_stage(NT);
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const uint4 xv[2] = {shared16(at + line_place(g, 4 * h + c)), shared16(at + line_place(8 + g, 4 * h + c))};
#pragma unroll
            for (int j = 0; j < NT; ++j)
                if (8 * j < a.rank) multiply(xv, j, shared16(at + line_place(16 + 8 * j + g, 4 * h + c)));
        }
        s = s + 1 == kStages ? 0 : s + 1;
    }
    // a cut chunk, and rows that are not on 16-byte boundaries
    const int t0 = max(0, __shfl_sync(0xffffffffu, tile.tok, g)), t1 = max(0, __shfl_sync(0xffffffffu, tile.tok, 8 + g));
#pragma unroll 1
    for (int half = 2 * ch; half < 2 * c1; half += half & 1 ? 2 * kSumWarps - 1 : 1) {
        const int k = half * 32 + 8 * c;
        const uint4 xv[2] = {load8(X + (size_t)t0 * a.ldx, k, a.din, a.vec_x), load8(X + (size_t)t1 * a.ldx, k, a.din, a.vec_x)};
        uint4 w[NT];                           // all in flight; what lies past the rank is not kept
#pragma unroll
        for (int j = 0; j < NT; ++j) w[j] = load8(A + (size_t)((8 * j < a.rank ? 8 * j : 0) + g) * a.din, k, a.din, a.vec_x);
#pragma unroll
        for (int j = 0; j < NT; ++j) multiply(xv, j, w[j]);
    }
    copies_landed<0>();
    __syncthreads();                           // the rings' room takes the warps' sums
#pragma unroll
    for (int j = 0; j < NT; ++j)
#pragma unroll
        for (int e = 0; e < 4; ++e) part[warp][g + 8 * (e / 2)][8 * j + 2 * c + e % 2] = acc[j][e];
    __syncthreads();
    for (int e = threadIdx.x; e < 16 * kCols; e += 32 * kSumWarps) {
        const int r = e / kCols, j = e % kCols, t = a.order[16 + (size_t)blockIdx.x * 17 + r];
        if (t < 0 || j >= a.rank) continue;
        float sum = 0.f;
#pragma unroll
        for (int w = 0; w < kSumWarps; ++w) sum += part[w][r][j];
        a.u[((size_t)blockIdx.y * a.n + t) * a.rank + j] = sum;
    }
}

// u in 16-bit parts, x = x_0 + x_1 + ..: two of float16 keep it to 2^-22, of bfloat16 only to
// 2^-17, three to 2^-24.
template <int PARTS, class T>
__device__ __forceinline__ void split(float lo, float hi, uint32_t (&out)[PARTS]) {
#pragma unroll
    for (int p = 0; p < PARTS; ++p) {
        alignas(4) T h[2] = {from_float<T>(lo), from_float<T>(hi)};
        out[p] = *reinterpret_cast<const uint32_t *>(h);
        // (of an infinity nothing is left)
        lo = isinf(to_float(h[0])) ? 0.f : lo - to_float(h[0]);
        hi = isinf(to_float(h[1])) ? 0.f : hi - to_float(h[1]);
    }
}

// Outputs of 16 tokens a block: each of its warps has 64 of every 256 columns. KS:
// sixteens of the rank. A lane's results of a token are units of 16 bytes, which lie
// beside those of three other lanes.
template <class Out>
struct OutUnits {
    static constexpr int E = kUnit<Out>, count = 16 / E;     // of a token's 16 outputs of a lane
    // the first output of unit h of lanes c
    __device__ static int first(int h, int c) { return 4 * E * h + E * c; }
    // the output that column g of MMA q stands for: a lane's two of each of E / 2 MMAs
    // make up a unit
    __device__ static int of(int q, int g) { return 4 * E * (q / (E / 2)) + E * (g >> 1) + 2 * (q % (E / 2)) + (g & 1); }
};
// A step of a warp's ring: 64 outputs of Y0's 16 rows, then 64 rows of B, which are
// spread so that the four that 16 lanes read are in different banks.
template <class Out, int KS>
struct OutRing {
    static constexpr int E = kUnit<Out>, units = 64 / E, rows = 16 * 64 * (int)sizeof(Out);
    static constexpr int pitch = KS * 32 + (KS >= 4 ? 32 : 0), gap = KS == 2 ? 32 : 64;
    static constexpr int stage = rows + 64 * pitch + 8 * gap, stages = 2, bytes = 4 * stages * stage;
    static constexpr int blocks = 220 * 1024 / (bytes + 1024);   // of an SM
    __device__ static uint32_t y0(int row, int unit) { return row * 64 * (int)sizeof(Out) + ((unit ^ ((row & 1) << 2)) << 4); }
    __device__ static uint32_t b(int col) { return rows + col * pitch + (col >> 3) * gap; }
};

template <class T, class Out, int KS, int PARTS>
__global__ void __launch_bounds__(128) outputs_kernel(AdapterArgs a, int columns) {
    using Units = OutUnits<Out>;
    using Ring = OutRing<Out, KS>;
    __shared__ float4 joined[16][4 * KS + 1];
    constexpr int kStages = Ring::stages, E = Units::E;
    extern __shared__ uint4 ring[];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, g = lane >> 2, c = lane & 3;
    tc::pdl_wait();
    const Tile tile(a);
    if (tile.adapter == -3) return;
    const int o0 = blockIdx.y * columns + 64 * warp, o1 = min(a.dout, (int)(blockIdx.y + 1) * columns);
    int t[2];
    bool there[2];
    const Out *y0[2];
    Out *y[2];
#pragma unroll
    for (int m = 0; m < 2; ++m) {
        t[m] = __shfl_sync(0xffffffffu, tile.tok, 8 * m + g);
        there[m] = t[m] >= 0;
        t[m] = max(t[m], 0);
        y0[m] = static_cast<const Out *>(a.Y0) + (size_t)t[m] * a.ldy0;
        y[m] = static_cast<Out *>(a.Y) + (size_t)t[m] * a.ldy;
    }
    // unit h of token m from column o on: Y0's `held` and the sums d
    auto put_whole = [&](int m, int o, int h, const uint4 &held, const float *d) {
        float v[E];
        unpack(held, v, Out());
#pragma unroll
        for (int e = 0; e < E; ++e) v[e] += d[e];
        *reinterpret_cast<uint4 *>(y[m] + o + Units::first(h, c)) = pack(v, Out());
    };
    // 64 outputs from o on of token m of every lane, eight tokens in all, by way of 2 KB
    // of shared memory: then 32 lanes have neighbouring outputs of one token
    auto put_parts = [&](int m, int o, uint32_t stage, const float (&d)[16]) {
        __syncwarp();
#pragma unroll
        for (int h = 0; h < Units::count; ++h)
#pragma unroll
            for (int e = 0; e < E; ++e)
                asm volatile("st.shared.f32 [%0], %1;" ::"r"(stage + (g * 64 + Units::first(h, c) + e) * 4), "f"(d[E * h + e]) : "memory");
        __syncwarp();
        const Out *Y0 = static_cast<const Out *>(a.Y0);
        float v[8][2];
#pragma unroll
        for (int r = 0; r < 8; ++r) {
            const int at = __shfl_sync(0xffffffffu, tile.tok, 8 * m + r);
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                const int k = o + 32 * i + lane;
                v[r][i] = Y0 && at >= 0 && k < o1 ? to_float(Y0[(size_t)at * a.ldy0 + k]) : 0.f;
            }
        }
#pragma unroll
        for (int r = 0; r < 8; ++r) {
            const int at = __shfl_sync(0xffffffffu, tile.tok, 8 * m + r);
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                const int k = o + 32 * i + lane;
                float x;
                asm volatile("ld.shared.f32 %0, [%1];" : "=f"(x) : "r"(stage + (r * 64 + 32 * i + lane) * 4) : "memory");
                if (at >= 0 && k < o1) static_cast<Out *>(a.Y)[(size_t)at * a.ldy + k] = from_float<Out>(v[r][i] + x);
            }
        }
    };
    if (tile.adapter >= 0) {
        const T *B = static_cast<const T *>(a.B) + (size_t)tile.adapter * a.dout * a.rank;
        const bool fast = ((uintptr_t)B & 15) == 0, ringed = a.Y0 && a.vec_y;
        const uint32_t room = tc::smem_u32(ring) + warp * kStages * Ring::stage;
        auto ahead = [&](int o, int s) {
            if (fast && o + 64 <= o1) {
                const uint32_t to = room + s * Ring::stage;
                if (ringed) {
#pragma unroll
                    for (int i = 0; i < 16 * Ring::units / 32; ++i) {
                        const int row = (32 * i + lane) / Ring::units, unit = lane % Ring::units;
                        const int at = __shfl_sync(0xffffffffu, tile.tok, row);
                        if (at >= 0)
                            copy_ahead(to + Ring::y0(row, unit), static_cast<const Out *>(a.Y0) + (size_t)at * a.ldy0 + o + E * unit);
                    }
                }
                // 64 rows of B, one after the other in memory
                const T *from = B + (size_t)o * a.rank;
                if (a.rank == 16 * KS) {
#pragma unroll
                    for (int i = 0; i < 4 * KS; ++i) {
                        const int at = 32 * i + lane;
                        copy_ahead(to + Ring::b(at / (2 * KS)) + at % (2 * KS) * 16, from + 8 * at);
                    }
                } else {
                    const int units = a.rank / 8;
                    for (int at = lane; at < 64 * units; at += 32)
                        copy_ahead(to + Ring::b(at / units) + at % units * 16, from + 8 * at);
                }
            }
            copies_made();
        };
#pragma unroll
        for (int s = 0; s + 1 < kStages; ++s) ahead(o0 + 256 * s, s);
        // the tokens' sums, under the first copies: joined by all warps
        const float by = a.scale ? a.scale[tile.adapter] : 1.f;
        for (int e = threadIdx.x; e < 4 * a.rank; e += 128) {
            const int row = e / (a.rank / 4), j = e % (a.rank / 4) * 4, at = max(0, __shfl_sync(0xffffffffu, tile.tok, row));
            const float *from = a.u + (size_t)at * a.rank + j;
            float4 sum = make_float4(0.f, 0.f, 0.f, 0.f);
            constexpr int kBatch = 8;
            for (int p0 = 0; p0 < a.splits; p0 += kBatch) {
                float4 v[kBatch];
#pragma unroll
                for (int p = 0; p < kBatch; ++p)
                    v[p] = p0 + p < a.splits ? *reinterpret_cast<const float4 *>(from + (size_t)(p0 + p) * a.n * a.rank)
                                             : make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
                for (int p = 0; p < kBatch; ++p) sum.x += v[p].x, sum.y += v[p].y, sum.z += v[p].z, sum.w += v[p].w;
            }
            joined[row][j / 4] = make_float4(sum.x * by, sum.y * by, sum.z * by, sum.w * by);
        }
        __syncthreads();
        uint32_t u[KS][PARTS][4];
        float back[2];
#pragma unroll
        for (int m = 0; m < 2; ++m) {
            float v[KS][4], top = 0.f;
#pragma unroll
            for (int k = 0; k < KS; ++k) {
                const float4 s = 16 * k + 4 * c < a.rank ? joined[8 * m + g][4 * k + c] : make_float4(0.f, 0.f, 0.f, 0.f);
                v[k][0] = s.x, v[k][1] = s.y, v[k][2] = s.z, v[k][3] = s.w;
#pragma unroll
                for (int e = 0; e < 4; ++e) top = fmaxf(top, fabsf(v[k][e]) < INFINITY ? fabsf(v[k][e]) : 0.f);
            }
            // the largest of the finite sums to 1 .. 2 (less where it is no normal number) by a
            // power of two, whatever its size in float32: no part leaves the 16-bit type's range.
            // (Powers put together from their bits: 8192 tokens of rank 16 49.9 us for 48.7.)
            top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 1));
            top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 2));
            const int e = (int)(__float_as_uint(top) >> 23) - 127;
            const float down = ldexpf(1.f, -e);
            back[m] = ldexpf(1.f, e);
#pragma unroll
            for (int k = 0; k < KS; ++k)
#pragma unroll
                for (int q = 0; q < 4; ++q) v[k][q] *= down;
#pragma unroll
            for (int k = 0; k < KS; ++k) {
                uint32_t p0[PARTS], p1[PARTS];
                split<PARTS, T>(v[k][0], v[k][1], p0);
                split<PARTS, T>(v[k][2], v[k][3], p1);
#pragma unroll
                for (int p = 0; p < PARTS; ++p) {
                    u[k][p][m] = p0[p];
                    u[k][p][2 + m] = p1[p];
                }
            }
        }
        auto multiply = [&](float (&acc)[8][4], int k, int q, uint2 b) {
#pragma unroll
            for (int p = 0; p < PARTS; ++p) mma(acc[q], u[k][p], b.x, b.y, T());
        };
        auto sums_of = [&](const float (&acc)[8][4], int m, float (&d)[16]) {
#pragma unroll
            for (int q = 0; q < 8; ++q) {
                d[2 * q] = acc[q][2 * m] * back[m];
                d[2 * q + 1] = acc[q][2 * m + 1] * back[m];
            }
        };
        int o = o0, s = 0;
#pragma unroll 1
        for (; fast && o + 64 <= o1; o += 256) {
            __syncwarp();                      // all lanes have read the stage that is filled next
            ahead(o + 256 * (kStages - 1), s == 0 ? kStages - 1 : s - 1);
            copies_landed<kStages - 1>();
            __syncwarp();
            const uint32_t at = room + s * Ring::stage;
            float acc[8][4] = {};
#pragma unroll
            for (int k = 0; k < KS; ++k)
#pragma unroll
                for (int q = 0; q < 8; ++q)
                    multiply(acc, k, q, 16 * k + 4 * c < a.rank ? shared8(at + Ring::b(Units::of(q, g)) + 32 * k + 8 * c) : make_uint2(0, 0));
#pragma unroll
            for (int m = 0; m < 2; ++m) {
                float d[16];
                sums_of(acc, m, d);
                if (!a.vec_y) {
                    put_parts(m, o, at, d);
                    continue;
                }
                if (!there[m]) continue;
#pragma unroll
                for (int h = 0; h < Units::count; ++h)
                    put_whole(m, o, h, ringed ? shared16(at + Ring::y0(8 * m + g, 4 * h + c)) : make_uint4(0, 0, 0, 0), d + E * h);
            }
            s = s + 1 == kStages ? 0 : s + 1;
        }
        copies_landed<0>();
        // cut columns, and rows that are not on 16-byte boundaries
#pragma unroll 1
        for (; o < o1; o += 256) {
            float acc[8][4] = {};
#pragma unroll
            for (int k = 0; k < KS; ++k) {
                const int j = 16 * k + 4 * c;
                uint2 v[8];                        // all in flight
#pragma unroll
                for (int q = 0; q < 8; ++q) {
                    const int col = o + Units::of(q, g);
                    const T *p = B + (size_t)col * a.rank + j;
                    v[q] = make_uint2(0, 0);
                    if (j < a.rank && col < o1) {
                        if (fast) {
                            v[q] = *reinterpret_cast<const uint2 *>(p);
                        } else {
                            const uint16_t *h = reinterpret_cast<const uint16_t *>(p);
                            v[q] = make_uint2(h[0] | (uint32_t)h[1] << 16, h[2] | (uint32_t)h[3] << 16);
                        }
                    }
                }
#pragma unroll
                for (int q = 0; q < 8; ++q) multiply(acc, k, q, v[q]);
            }
#pragma unroll
            for (int m = 0; m < 2; ++m) {
                float d[16];
                sums_of(acc, m, d);
                put_parts(m, o, room, d);
            }
        }
        return;
    }
    // tokens without an adapter, and those of one that there is not: a row a warp
    const float add = tile.adapter == -1 ? -0.f : __int_as_float(0x7FC00000);      // x + -0 is x, -0 too
    const int first = blockIdx.y * columns;
#pragma unroll 1
    for (int r = warp; r < 16; r += 4) {
        const int at = __shfl_sync(0xffffffffu, tile.tok, r);
        if (at < 0) continue;
        const Out *from = static_cast<const Out *>(a.Y0) + (size_t)at * a.ldy0;
        Out *to = static_cast<Out *>(a.Y) + (size_t)at * a.ldy;
        int k = first;
        if (a.vec_y) {
            constexpr int kBatch = 4;              // units in flight
#pragma unroll 1
            for (; k + E <= o1; k += kBatch * 32 * E) {
                uint4 v[kBatch];
#pragma unroll
                for (int i = 0; i < kBatch; ++i) {
                    const int j = k + (32 * i + lane) * E;
                    v[i] = a.Y0 && j + E <= o1 ? *reinterpret_cast<const uint4 *>(from + j) : make_uint4(0, 0, 0, 0);
                }
#pragma unroll
                for (int i = 0; i < kBatch; ++i) {
                    const int j = k + (32 * i + lane) * E;
                    if (j + E > o1) continue;
                    float x[E];
                    unpack(v[i], x, Out());
#pragma unroll
                    for (int e = 0; e < E; ++e) x[e] += add;
                    *reinterpret_cast<uint4 *>(to + j) = pack(x, Out());
                }
            }
            k = o1 - (o1 - first) % E;
        }
        constexpr int kBatch = 8;
#pragma unroll 1
        for (; k < o1; k += kBatch * 32) {
            float v[kBatch];
#pragma unroll
            for (int i = 0; i < kBatch; ++i) v[i] = a.Y0 && k + 32 * i + lane < o1 ? to_float(from[k + 32 * i + lane]) : 0.f;
#pragma unroll
            for (int i = 0; i < kBatch; ++i)
                if (k + 32 * i + lane < o1) to[k + 32 * i + lane] = from_float<Out>(v[i] + add);
        }
    }
}

int ceil_div(int64_t a, int64_t b) { return (int)((a + b - 1) / b); }

// Splits of the width where there are few tiles of tokens: as many blocks as run at
// one time, each at least 256 of it.
int many_splits(int n, int din, int rank) {
    const int tiles = ceil_div(n, 16), at_once = 152 * sum_blocks(rank <= 16 ? 2 : rank <= 32 ? 4 : rank <= 64 ? 8 : 16);
    return std::max(1, std::min({at_once / tiles, ceil_div(din, 256), kMostSplits}));
}

template <class T, class Out>
cudaError_t launch_few(const AdapterArgs &a, cudaStream_t s) {
    // CTAs of a token by its width and outputs alone, so that its sums do not depend on
    // the batch
    int ctas = 1;
    while (ctas < 8 && ctas * kFewPiece < std::max(a.din, a.dout)) ctas *= 2;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)(a.n * ctas));
    const bool wide = a.n * ctas <= 152;
    cfg.blockDim = dim3(wide ? 512 : 256);
    cfg.stream = s;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = ctas;
    attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    count_launches(1);
    return wide ? cudaLaunchKernelEx(&cfg, few_kernel<T, Out, 512>, a, ctas) : cudaLaunchKernelEx(&cfg, few_kernel<T, Out, 256>, a, ctas);
}

template <class T, class Out, int KS>
cudaError_t launch_many_as(const AdapterArgs &a, cudaStream_t s) {
    constexpr int kParts = std::is_same_v<T, __nv_bfloat16> ? 3 : 2;
    static std::atomic<unsigned long long> done[2];
    auto *sums = sums_kernel<T, 2 * KS>;
    auto *outputs = outputs_kernel<T, Out, KS, kParts>;
    const int tiles = tiles_at_most(a.n, a.adapters);
    // Columns of a block, in whole steps of 256: up to four blocks after one another,
    // which do not all take as long (8192 tokens, 4096 -> 4096: 48 us; as many blocks as
    // run at one time 65, twice as many 60).
    const int columns =
        std::max(512, round_up(ceil_div(a.dout, std::max(1, 4 * 152 * OutRing<Out, KS>::blocks / tiles)), 256));
    order_kernel<<<1, 1024, (a.adapters + 2) * sizeof(int), s>>>(a);
    cudaError_t e = cudaGetLastError();
    if (e == cudaSuccess) e = set_max_dynamic_smem((const void *)sums, sum_shared(2 * KS), done[0]);
    if (e == cudaSuccess) e = launch_pdl(sums, dim3(tiles, a.splits), dim3(32 * kSumWarps), sum_shared(2 * KS), s, a);
    if (e == cudaSuccess) e = set_max_dynamic_smem((const void *)outputs, OutRing<Out, KS>::bytes, done[1]);
    if (e == cudaSuccess)
        e = launch_pdl(outputs, dim3(tiles, ceil_div(a.dout, columns)), dim3(128), OutRing<Out, KS>::bytes, s, a, columns);
    count_launches(3);
    return e;
}
template <class T, class Out>
cudaError_t launch_many(const AdapterArgs &a, cudaStream_t s) {
    if (a.rank <= 16) return launch_many_as<T, Out, 1>(a, s);
    if (a.rank <= 32) return launch_many_as<T, Out, 2>(a, s);
    if (a.rank <= 64) return launch_many_as<T, Out, 4>(a, s);
    return launch_many_as<T, Out, 8>(a, s);
}

bool is_aligned(const void *p, size_t b) { return ((uintptr_t)p & (b - 1)) == 0; }
bool usable(const void *p, size_t size) { return p && on_device(p) && is_aligned(p, size); }

}  // namespace
}  // namespace jarq

using namespace jarq;

extern "C" {

size_t jarq_adapters_workspace(int n, int din, int rank, int adapters) {
    if (n < 1 || adapters < 0 || adapters > kMostAdapters || n > kMostTokens || din < 1 || din > kMostWidth || rank < 8 || rank > kMostRank || rank % 8) return 0;
    if (n <= kFew) return 0;
    return (size_t)many_splits(n, din, rank) * n * rank * sizeof(float) + ((size_t)tiles_at_most(n, adapters) * 17 + 16) * sizeof(int);
}

jarq_status jarq_apply_adapters(const void *X, jarq_dtype dtype, int64_t ldx, const void *A, const void *B,
                                const float *scale, int adapters, int rank, const int32_t *ids, int n,
                                int din, int dout, const void *Y0, int64_t ldy0, void *Y, int64_t ldy,
                                jarq_dtype ydtype, void *workspace, size_t workspace_bytes, void *stream) {
    if ((dtype != JARQ_F16 && dtype != JARQ_BF16) || (ydtype != dtype && ydtype != JARQ_F32)) return JARQ_ERR_ARG;
    if (n < 0 || n > kMostTokens || din < 1 || din > kMostWidth || dout < 1 || dout > kMostWidth || ldx < din || ldy < dout ||
        (Y0 && ldy0 < dout) || adapters < 0 || adapters > kMostAdapters || rank < 8 || rank > kMostRank || rank % 8 ||
        (Y0 == Y && Y && n > 1 && ldy0 != ldy))
        return JARQ_ERR_ARG;
    if (n == 0) return JARQ_OK;
    const size_t ysize = size_of(ydtype);
    if (!usable(X, 2) || !usable(ids, 4) || !usable(Y, ysize) || (Y0 && !usable(Y0, ysize)) || (scale && !usable(scale, 4)))
        return JARQ_ERR_ARG;
    if (adapters && (!usable(A, 2) || !usable(B, 2))) return JARQ_ERR_ARG;
    const size_t need = jarq_adapters_workspace(n, din, rank, adapters);
    if (need && (!usable(workspace, 16) || workspace_bytes < need)) return JARQ_ERR_ARG;
    if (const jarq_status late = async_failure()) return late;
    cudaStream_t st = (cudaStream_t)stream;
    const bool few = n <= kFew;
    AdapterArgs a{X, A, B, Y0, Y, scale, ids, static_cast<float *>(workspace), nullptr, ldx, ldy0, ldy, n, din, dout, rank,
                  adapters, few ? 1 : many_splits(n, din, rank)};
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
