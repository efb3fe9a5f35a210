// The integer product's tensor-core form, for more than a few tokens.
//
// GB300's 8-bit integer tensor rate is a small fraction of its fp16 rate, so
// int8 codes become fp16 on the way into shared memory (exactly: |c| <= 128) and
// the product runs on fp16 MMAs.  Their sums are integers of at most
// 128 128 1024 = 2^24 over 1024 of K, exact in the float32 accumulator; after
// that many, or after each group, they leave it: with one scale a channel for
// an int32 sum, with groups for a float32 sum of the terms ws_i sum_i.
//
// A pair of CTAs (cta_group::2): 256 channels x NT tokens, channels on the lanes
// of TMEM, so that a thread of the epilogue has one channel and its group's
// scale in a register.  Per 128 of K each CTA converts its own 128 channels and
// half of the tokens.
//   warp 0        MMA issuer (of the pair's even CTA); warp 1: TMEM
//   warps 4..11   loaders: 16 codes at a time from global memory to registers, a
//                 step or two ahead, then converted and written to the ring in
//                 the 128-byte swizzle of a K-major operand
//   warps 12..19  drain: lane quarter w % 4, half of the columns
// A cluster of 2 S CTAs splits K over S pairs where there are few tiles; the
// partial sums are joined through distributed shared memory.
#include "integer.cuh"
#include "rows.cuh"
#include "tc_common.cuh"

namespace jarq {
namespace {

using namespace rows;

constexpr int kThreads = 640, kLoaders = 256, kDrain = 256;
constexpr int kStepK = 128;                   // K of a stage: two swizzled atoms of 64
constexpr int kAtomA = 128 * 128;             // bytes: 128 channels x 64 of K, fp16
constexpr int kExact = 16;                    // atoms (1024 of K) with an exact sum

__host__ __device__ constexpr int atom_b(int nt) { return nt / 2 * 128; }
__host__ __device__ constexpr int stage_bytes(int nt) { return 2 * (kAtomA + atom_b(nt)); }
__host__ __device__ constexpr int stages(int nt) { return nt == 256 ? 3 : nt == 128 ? 4 : 5; }
__host__ __device__ constexpr int smem_bytes(int nt) { return 1024 + stages(nt) * stage_bytes(nt) + 256; }
// steps that a loader holds in registers
__host__ __device__ constexpr int ahead(int nt) { return nt == 256 ? 1 : 2; }

__device__ __forceinline__ bool wait_cluster(uint32_t bar, uint32_t parity) {
#pragma unroll 1
    for (uint32_t i = 0; i < tc::kWaitIters; ++i) {
        uint32_t ok;
        asm volatile(
            "{\n .reg .pred p;\n mbarrier.try_wait.parity.acquire.cluster.shared::cta.b64 p, [%1], %2;\n"
            " selp.u32 %0, 1, 0, p;\n}\n"
            : "=r"(ok)
            : "r"(bar), "r"(parity)
            : "memory");
        if (ok) return true;
    }
    return false;
}
__device__ __forceinline__ void arrive_cluster(uint32_t bar) {
    asm volatile("mbarrier.arrive.release.cluster.shared::cluster.b64 _, [%0];" ::"r"(bar) : "memory");
}
__device__ __forceinline__ void fence_to_async() { asm volatile("fence.proxy.async.shared::cta;" ::: "memory"); }
__device__ __forceinline__ void cluster_barrier() {
    __syncwarp();
    asm volatile("barrier.cluster.arrive.release.aligned;\n barrier.cluster.wait.acquire.aligned;" ::: "memory");
}
__device__ __forceinline__ uint32_t load_remote(uint32_t addr) {
    uint32_t v;
    asm volatile("ld.shared::cluster.u32 %0, [%1];" : "=r"(v) : "r"(addr) : "memory");
    return v;
}
template <int R>
__device__ __forceinline__ void registers_down() {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(R));
}
template <int R>
__device__ __forceinline__ void registers_up() {
    asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(R));
}

// Two codes of w as fp16: c + 128 in the low bits of 1024 + (c + 128), less 1152.
__device__ __forceinline__ uint32_t to_half2(uint32_t w, uint32_t sel) {
    const uint32_t h = __byte_perm(w, 0x64646464u, sel);
    const __half2 d = __hsub2(*reinterpret_cast<const __half2 *>(&h), __half2half2(__ushort_as_half(0x6480)));
    return *reinterpret_cast<const uint32_t *>(&d);
}
__device__ __forceinline__ void convert16(const uint4 &raw, uint4 &lo, uint4 &hi) {
    const uint32_t a = raw.x ^ 0x80808080u, b = raw.y ^ 0x80808080u, c = raw.z ^ 0x80808080u, d = raw.w ^ 0x80808080u;
    lo = make_uint4(to_half2(a, 0x4140), to_half2(a, 0x4342), to_half2(b, 0x4140), to_half2(b, 0x4342));
    hi = make_uint4(to_half2(c, 0x4140), to_half2(c, 0x4342), to_half2(d, 0x4140), to_half2(d, 0x4342));
}
__device__ __forceinline__ void store_shared(uint32_t addr, const uint4 &v) {
    asm volatile("st.shared.v4.u32 [%0], {%1, %2, %3, %4};" ::"r"(addr), "r"(v.x), "r"(v.y), "r"(v.z), "r"(v.w) : "memory");
}

// NT: tokens of a tile.  GROUPS: group scales.  VEC: 16-byte aligned rows.
template <int NT, bool GROUPS, bool VEC>
__global__ void __launch_bounds__(kThreads, 1) tc_integer_kernel(ProductArgs a, int split, int *failed) {
    constexpr int kStages = stages(NT), kStage = stage_bytes(NT), kAtomB = atom_b(NT);
    constexpr int kRowsB = NT / 2;
    constexpr int kCols = NT / 2;               // columns of a drain warp
    constexpr uint32_t kIdesc = tc::idesc_f16_f32(256, NT);
    constexpr uint32_t kTmem = 2 * NT;
    extern __shared__ uint8_t smem_raw[];
    uint8_t *smem = (uint8_t *)(((uintptr_t)smem_raw + 1023) & ~(uintptr_t)1023);
    uint64_t *bars = (uint64_t *)(smem + kStages * kStage);
    uint32_t *tmem_slot = (uint32_t *)(bars + 2 * kStages + 5);
    volatile int *abort_flag = (volatile int *)(tmem_slot + 1);
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int crank = (int)tc::cluster_rank(), rank = crank & 1, part = crank >> 1;
    const uint32_t even = crank & ~1;
    const int nclusters = gridDim.x / (2 * split), cluster = blockIdx.x / (2 * split);
    const int mt = (a.dout + 255) / 256, ntiles = mt * ((a.n + NT - 1) / NT);
    // this pair's part of K
    const int steps = (a.din + kStepK - 1) / kStepK, per = (steps + split - 1) / split;
    const int step0 = min(steps, part * per), nsteps = min(steps, step0 + per) - step0;
    const int natoms = max(0, min((a.din + 63) / 64 - 2 * step0, 2 * nsteps));
    const int ua = GROUPS ? a.g / 64 : kExact;               // atoms of an accumulator
    const int nunits = (natoms + ua - 1) / ua;

    auto full = [&](int s) { return tc::smem_u32(bars + s); };
    auto empty = [&](int s) { return tc::smem_u32(bars + kStages + s); };
    auto afull = [&](int b) { return tc::smem_u32(bars + 2 * kStages + b); };
    auto aempty = [&](int b) { return tc::smem_u32(bars + 2 * kStages + 2 + b); };
    const uint32_t closing = tc::smem_u32(bars + 2 * kStages + 4);
    const uint32_t ring = tc::smem_u32(smem);

    if (threadIdx.x == 0) {
        for (int s = 0; s < kStages; ++s) {
            tc::mbar_init(full(s), 2 * kLoaders / 32);       // the even CTA's: both CTAs' loaders
            tc::mbar_init(empty(s), 1);
        }
        for (int b = 0; b < 2; ++b) {
            tc::mbar_init(afull(b), 1);
            tc::mbar_init(aempty(b), 2 * kDrain / 32);       // the even CTA's: both drains
        }
        tc::mbar_init(closing, 1);
        *abort_flag = 0;
        tc::fence_barrier_init();
    }
    if (warp == 1) {
        tc::tmem_alloc_pair(tc::smem_u32(tmem_slot), kTmem);
        tc::tmem_relinquish_pair();
    }
    tc::tc_fence_before();
    __syncthreads();
    tc::cluster_sync();
    tc::tc_fence_after();
    const uint32_t tmem = *tmem_slot;

    if (warp < 4) {
        if constexpr (NT == 256) registers_down<40>();
        // ---------------- MMA issuer of the pair
        if (warp == 0 && rank == 0) {
            bool ok = true;
            const uint64_t ad0 = tc::sdesc_sw128(ring), bd0 = tc::sdesc_sw128(ring + 2 * kAtomA);
            int s = 0, ph = 0, pc = 0;
            for (int tile = cluster; tile < ntiles && ok; tile += nclusters) {
                int left = 0;                                // atoms left in the accumulator
                for (int at = 0; at < natoms && ok; ++at) {
                    if ((at & 1) == 0) ok = wait_cluster(full(s), ph);
                    const bool first = left == 0;
                    if (first) {
                        left = min(ua, natoms - at);
                        ok = tc::mbar_wait(aempty(pc & 1), ((pc >> 1) & 1) ^ 1) && ok;
                    }
                    if (!ok) break;
                    tc::tc_fence_after();
                    const bool last = --left == 0, done = (at & 1) || at + 1 == natoms;
                    if (tc::elect_one()) {
                        const uint64_t ad = ad0 + (uint64_t)((s * kStage + (at & 1) * kAtomA) >> 4);
                        const uint64_t bd = bd0 + (uint64_t)((s * kStage + (at & 1) * kAtomB) >> 4);
#pragma unroll
                        for (int sub = 0; sub < 4; ++sub)
                            tc::mma_f16_pair(tmem + (pc & 1) * NT, ad + 2 * sub, bd + 2 * sub, kIdesc, !first || sub > 0);
                        if (done) tc::mma_commit_pair(empty(s), 3 << even);
                        if (last) tc::mma_commit_pair(afull(pc & 1), 3 << even);
                    }
                    __syncwarp();
                    if (last) ++pc;
                    if (done && ++s == kStages) {
                        s = 0;
                        ph ^= 1;
                    }
                }
            }
            if (tc::elect_one()) tc::mma_commit_pair(closing, 1 << even);
            if (!tc::mbar_wait(closing, 0) || !ok) *abort_flag = 1;
        }
    } else if (warp < 12) {
        if constexpr (NT == 256) registers_down<72>();
        // ---------------- loaders
        constexpr int kUB = (kRowsB + 31) / 32;              // units of the tokens a thread
        constexpr int kU = 4 + kUB, kAhead = ahead(NT);
        const int t = threadIdx.x - 128, c = t & 7, r0 = t >> 3;
        const bool has_b = kRowsB >= 32 || r0 < kRowsB;
        // 16 codes become two 16-byte chunks of a 128-byte row; threads of the
        // second atom write theirs in the other order, so that eight lanes of a
        // row always cover all banks
        const int atom = c >> 2, j0 = 2 * (c & 3) + atom;
        const uint32_t sw0 = (uint32_t)(r0 * 128 + ((j0 ^ (r0 & 7)) << 4)), sw1 = (uint32_t)(r0 * 128 + (((j0 ^ 1) ^ (r0 & 7)) << 4));
        const uint32_t toA = ring + atom * kAtomA, toB = ring + 2 * kAtomA + atom * kAtomB;
        const uint32_t full0 = tc::map_rank(full(0), even);
        bool ok = true;
        int s = 0, ph = 1;
        for (int tile = cluster; tile < ntiles && ok; tile += nclusters) {
            const int o = tile % mt * 256 + 128 * rank + r0, tk = tile / mt * NT + kRowsB * rank + r0;
            const int8_t *pa = a.C + (size_t)o * a.ldc, *pb = a.X + (size_t)tk * a.ldx;
            const size_t sa = (size_t)32 * a.ldc, sb = (size_t)32 * a.ldx;
            uint4 held[kAhead][kU];
            if (tile == cluster) tc::pdl_wait();
            auto fetch = [&](uint4 (&h)[kU], int i, int step) {
                const int k = (step0 + step) * kStepK + c * 16;
                const bool in = step < nsteps && (i < 4 ? o + 32 * i < a.dout : has_b && tk + 32 * (i - 4) < a.n);
                h[i] = in ? load_codes<VEC>(i < 4 ? pa + i * sa : pb + (i - 4) * sb, k, a.din) : make_uint4(0, 0, 0, 0);
            };
#pragma unroll
            for (int p = 0; p < kAhead; ++p)
#pragma unroll
                for (int i = 0; i < kU; ++i) fetch(held[p], i, p);
            for (int step = 0; step < nsteps && ok; step += kAhead) {
#pragma unroll
                for (int p = 0; p < kAhead; ++p) {
                    if (step + p >= nsteps) break;
                    ok = tc::mbar_wait(empty(s), ph);
                    if (!ok) break;
                    const uint32_t da = toA + s * kStage, db = toB + s * kStage;
#pragma unroll
                    for (int i = 0; i < kU; ++i) {
                        uint4 lo, hi;
                        convert16(held[p][i], lo, hi);
                        fetch(held[p], i, step + p + kAhead);
                        if (i < 4 || has_b) {
                            const uint32_t d = i < 4 ? da + i * 32 * 128 : db + (i - 4) * 32 * 128;
                            store_shared(d + sw0, atom ? hi : lo);
                            store_shared(d + sw1, atom ? lo : hi);
                        }
                    }
                    fence_to_async();
                    __syncwarp();
                    if (lane == 0) arrive_cluster(full0 + 8 * s);
                    if (++s == kStages) {
                        s = 0;
                        ph ^= 1;
                    }
                }
            }
        }
        if (!ok) *abort_flag = 1;
    } else {
        if constexpr (NT == 256) registers_up<144>();
        // ---------------- drain
        tc::pdl_wait();                                      // the tokens' scales
        const int w = warp - 12, q = w & 3, col0 = (w >> 2) * kCols;
        const int lrow = 32 * q + lane;
        const uint32_t released = tc::map_rank(aempty(0), even);
        const uint32_t taddr = tmem + ((uint32_t)(32 * q) << 16) + col0;
        bool ok = true;
        int pc = 0;
        for (int tile = cluster; tile < ntiles && ok; tile += nclusters) {
            const int o = tile % mt * 256 + 128 * rank + lrow, t0 = tile / mt * NT;
            const bool live = o < a.dout;
            uint32_t acc[kCols];                             // int32, or float32 with groups
#pragma unroll
            for (int e = 0; e < kCols; ++e) acc[e] = 0;
            const float *wp = a.ws + (live ? (size_t)o * a.G : 0) + (GROUPS ? 2 * step0 / ua : 0);
            for (int u = 0; u < nunits; ++u, ++pc) {
                const int b = pc & 1;
                const float wsc = GROUPS ? wp[u] : 0.f;
                ok = __all_sync(0xffffffffu, tc::mbar_wait(afull(b), (pc >> 1) & 1));
                if (!ok) break;
                tc::tc_fence_after();
#pragma unroll
                for (int cc = 0; cc < kCols; cc += 16) {
                    uint32_t v[16];
                    tc::tmem_ld16(taddr + b * NT + cc, v);
                    tc::tmem_wait_ld();
                    if (cc + 16 == kCols) {
                        tc::tc_fence_before();
                        __syncwarp();
                        if (lane == 0) tc::mbar_arrive_cluster(released + 8 * b);
                    }
#pragma unroll
                    for (int e = 0; e < 16; ++e) {
                        if (GROUPS)
                            acc[cc + e] = __float_as_uint(fmaf(__uint_as_float(v[e]), wsc, __uint_as_float(acc[cc + e])));
                        else
                            acc[cc + e] += (uint32_t)__float2int_rn(__uint_as_float(v[e]));
                    }
                }
            }
            if (!ok) break;
            const float wch = GROUPS ? 1.f : wp[0], bias = a.bias && live ? a.bias[o] : 0.f;
            if (split > 1) {
                // every MMA of the pair is done: its ring takes the partial sums
                const uint32_t mine = ring + (uint32_t)(col0 * 128 + lrow) * 4;
#pragma unroll
                for (int e = 0; e < kCols; ++e)
                    asm volatile("st.shared.u32 [%0], %1;" ::"r"(mine + e * 512), "r"(acc[e]) : "memory");
                break;                                       // joined below: one tile a cluster
            }
            if (live) {
                const int cols = min(kCols, a.n - t0 - col0);
                with_type_device(a.dtype, [&](auto type) {
                    using T = decltype(type);
                    T *y = static_cast<T *>(a.Y) + (size_t)(t0 + col0) * a.ldy + o;
#pragma unroll
                    for (int e = 0; e < kCols; ++e)
                        if (e < cols) {
                            const float v = GROUPS ? __uint_as_float(acc[e]) : (float)(int)acc[e] * wch;
                            y[(size_t)e * a.ldy] = from_float<T>(fmaf(v, a.xs[t0 + col0 + e], bias));
                        }
                });
            }
        }
        if (!ok) *abort_flag = 1;
    }
    if (split > 1) {
        // join: pair `part` finishes columns part NT / split .. of its 128 channels
        cluster_barrier();
        if (warp >= 12 && cluster < ntiles) {
            const int t = threadIdx.x - 384, lrow = t & 127, half = t >> 7;
            const int o = cluster % mt * 256 + 128 * rank + lrow, t0 = cluster / mt * NT;
            const int cols = NT / split;
            const float bias = a.bias && o < a.dout ? a.bias[o] : 0.f, wch = !GROUPS && o < a.dout ? a.ws[o] : 1.f;
            for (int e = half; e < cols; e += 2) {
                const int col = part * cols + e;
                if (o >= a.dout || t0 + col >= a.n) continue;
                const uint32_t at = ring + (uint32_t)(col * 128 + lrow) * 4;
                float f = 0.f;
                int i = 0;
                for (int p = 0; p < split; ++p) {
                    const uint32_t v = load_remote(tc::map_rank(at, 2 * p + rank));
                    f += __uint_as_float(v);
                    i += (int)v;
                }
                const float v = GROUPS ? f : (float)i * wch;
                with_type_device(a.dtype, [&](auto type) {
                    using T = decltype(type);
                    static_cast<T *>(a.Y)[(size_t)(t0 + col) * a.ldy + o] = from_float<T>(fmaf(v, a.xs[t0 + col], bias));
                });
            }
        }
    }
    // neither CTA leaves while another may still read its shared memory, signal
    // its barriers or hold TMEM of the pair
    tc::tc_fence_before();
    __syncwarp();
    __syncthreads();
    tc::cluster_sync();
    if (warp == 1) {
        tc::tc_fence_after();
        tc::tmem_dealloc_pair(tmem, kTmem);
    }
    if (threadIdx.x == 0 && *abort_flag) {
        *(volatile int *)failed = 1;
        __threadfence_system();
    }
}

template <int NT, bool GROUPS, bool VEC>
cudaError_t launch(const ProductArgs &a, int split, int *failed, cudaStream_t s, bool pdl) {
    static std::atomic<unsigned long long> done;
    auto *kernel = tc_integer_kernel<NT, GROUPS, VEC>;
    const cudaError_t e = set_max_dynamic_smem((const void *)kernel, smem_bytes(NT), done);
    if (e != cudaSuccess) return e;
    const int64_t tiles = (int64_t)((a.dout + 255) / 256) * ((a.n + NT - 1) / NT);
    const int64_t clusters = split > 1 ? tiles : std::min<int64_t>(tiles, num_sms() / 2);
    if (tiles > 0x3FFFFFFF / (2 * split)) return cudaErrorInvalidValue;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)(clusters * 2 * split));
    cfg.blockDim = dim3(kThreads);
    cfg.dynamicSmemBytes = smem_bytes(NT);
    cfg.stream = s;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = 2 * split;
    attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
    attr[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[1].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = pdl ? 2 : 1;
    return cudaLaunchKernelEx(&cfg, kernel, a, split, failed);
}

template <int NT>
cudaError_t launch_nt(const ProductArgs &a, int split, int *failed, cudaStream_t s, bool pdl) {
    const bool vec = vector_rows(a);
    if (a.g) return vec ? launch<NT, true, true>(a, split, failed, s, pdl) : launch<NT, true, false>(a, split, failed, s, pdl);
    return vec ? launch<NT, false, true>(a, split, failed, s, pdl) : launch<NT, false, false>(a, split, failed, s, pdl);
}

}  // namespace

cudaError_t launch_tc_integer(const ProductArgs &a, int *failed, cudaStream_t s, bool pdl) {
    // The tile's tokens and the split of K that leave the fewest steps in a
    // row, a step of 128 of K being about as long as given (cycles)
    constexpr struct {
        int nt, cycles;
    } kinds[] = {{32, 400}, {64, 450}, {128, 650}, {256, 1100}};
    const int mt = (a.dout + 255) / 256, steps = (a.din + kStepK - 1) / kStepK, pairs = std::max(1, num_sms() / 2);
    int nt = 0, split = 1;
    double best = 0;
    for (const auto &k : kinds)
        for (int sp = 1; sp <= 4; sp *= 2) {
            if (sp > 1 && sp > steps) break;
            const int64_t tiles = (int64_t)mt * ((a.n + k.nt - 1) / k.nt);
            if (sp > 1 && tiles * sp > pairs) break;
            const double t = (double)((tiles * sp + pairs - 1) / pairs) * ((steps + sp - 1) / sp) * k.cycles + (sp > 1 ? 2000 : 0);
            if (nt == 0 || t < best) {
                best = t;
                nt = k.nt;
                split = sp;
            }
        }
    switch (nt) {
        case 32: return launch_nt<32>(a, split, failed, s, pdl);
        case 64: return launch_nt<64>(a, split, failed, s, pdl);
        case 128: return launch_nt<128>(a, split, failed, s, pdl);
        default: return launch_nt<256>(a, split, failed, s, pdl);
    }
}

}  // namespace jarq
