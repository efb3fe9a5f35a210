// The integer product's tensor-core form, for more than a few tokens.
//
// GB300's 8-bit integer tensor rate is a small fraction of its fp16 rate (a library's
// products of 8192^3: 155 TOP/s in int8, 1823 TFLOP/s in fp16), so int8 codes become
// fp16 inside the SM (exactly: |c| <= 128) and the product runs on fp16 MMAs.  Their
// sums are integers of at most 128 128 1024 = 2^24 over 1024 of K, exact in the float32 accumulator; after that many, or after each
// group, they leave it: with one scale a channel for an int32 sum, with groups for
// a float32 sum of the terms ws_i sum_i.
//
// 128 channels on the lanes of TMEM x NT tokens, so that a thread of the epilogue
// has one channel and its group's scale in a register; for more than 64 tokens a
// pair of CTAs (cta_group::2) has 256 channels, and each CTA converts its own 128
// and half of the tokens.  Per 128 of K the channels go to TMEM as the A operand
// and the tokens to shared memory as the B operand; the linear layer's own tokens
// are quantized to integers in fp16 and need no conversion here.  (With both operands in shared
// memory 192 bytes are moved there per cycle of the MMAs, and the kernel took 1.6
// times as long; with A in TMEM it is 128.)  Tiles of 256 tokens are two
// accumulators of 128, one read while the other's MMAs run; smaller tiles
// alternate two.
//   warp 0        MMA issuer (of a pair's even CTA)
//   warps 0, 1, 3 of a pair's odd CTA pass on that a stage is full, where tokens are
//                 converted.  (Shared memory written for the other CTA's MMAs takes a
//                 release at cluster scope, which holds a warp for some 1300 cycles:
//                 done by the converters it doubled the time, by one warp it set the
//                 pace.  TMEM alone is ordered by the tcgen05 fences and an arrival.)
//   warp 1        TMEM allocation
//   warp 2        TMA producer: codes as they are into a ring of their own
//   warp 3        TMA producer of tokens that are fp16
//   warps 4..7    convert channels: a thread has one channel's row
//   warps 8..11   convert tokens, and half of the channels' K where tokens are few;
//                 with fp16 tokens, every other stage's channels
//   warps 12..19  drain: lane quarter w % 4, half of the columns (with kBrief one
//                 part of a tile)
//   warps 20..27  only where rows are not on 16-byte boundaries: fill the ring in
//                 the producer's place
// A cluster splits K over its CTAs or pairs where there are few tiles; the
// partial sums are joined through distributed shared memory.
//
// Measured from a graph, the quantization of float16 tokens included where tokens
// x K -> channels is given:
//   8192 x 11008 -> 4096, one scale    430 us (the product 384: 1.92 PFLOP/s)
//   4096 x 4096 -> 14336, groups of 128 297 us (1.62 PFLOP/s)
//   2048 x 4096 -> 4096, groups of 64   71 us, of 128 55, one scale 54 (with three sets
//                                       of inputs in turn 74, 57, 56)
//   64 x 4096 -> 4096 9.9 us from L2, 11.6 cold; 24 x 11008 -> 4096 (45 MB, cold) 18.5 us
//   int8 tokens given, the product alone: 8192 x 11008 -> 4096 608 us (converted in
//                                       every tile, and their stages relayed)
// A large product with one scale runs near the rate of a library's product in
// bfloat16.  With groups a sum leaves the accumulator eight (sixteen) times as often
// as with one scale, and what a scheduler's two drain warps do then (wake, read TMEM,
// hand back, add) is the bound: at 79 (groups of 64) and 309 us (128) of the sizes
// above, 61 and 271 were left without seven in eight additions and the scales' loads.
// Few tokens: the latency of a cluster's chain (first copies, conversion, MMAs,
// join), then reading the codes.  Rows off 16-byte boundaries are bound by the
// filling warps' loads (333 x 1001 -> 1343: 14.2 us, 1008 aligned 8.2; 4096 x 4001 -> 4096
// 236 us, 4096 x 4096 -> 4096 106, where every tile of tokens fills the channels again).
//
// Tried and dropped: four accumulators of 64 columns (the issuer's own instructions
// take 1620 of 1024 cycles a stage), the issue loop rolled (619 us for 430), two sets
// of converters for small tiles and conversion two units at a time (no gain, 5 %
// slower); in the drain, with groups: the next columns' loads under the additions (92
// us for 78, since the accumulator is held longer), scales loaded ahead or four at a
// time (81, 80), scalar additions (79; of 128: 325 for 309).
#include "integer.cuh"
#include "rows.cuh"
#include "tc_common.cuh"
#include "turns.cuh"

namespace jarq {
namespace {

using namespace rows;

constexpr int kDrain = 256, kFill = 256;
constexpr int kStepK = 128;                   // K of a stage: two atoms of 64
constexpr int kExact = 16;                    // atoms (1024 of K) with an exact sum
constexpr int kStages = 4;
constexpr int kMostParts = 4;                  // of K, over a cluster
constexpr int kColsA = 64;                    // TMEM columns of a stage's channels (two fp16 each)
constexpr int kTmem = 512;                    // accumulators of up to 128, then stages of channels

// columns of an accumulator, and how many a tile has
__host__ __device__ constexpr int acc_cols(int nt) { return nt < 128 ? nt : 128; }
__host__ __device__ constexpr int acc_parts(int nt) { return nt / acc_cols(nt); }
// Accumulators that take turns, and stages of channels.  With groups of 64 in tiles
// of 256 tokens (`brief`) an accumulator's MMAs take 256 cycles, less than the way of
// another's sums to the drain's registers and of the word back: there a third one
// takes the room of two stages of channels, which with groups of 128 costs more than
// it gives (2048 x 4096 -> 4096, groups of 64: 78 -> 71 us; 4096 x 4096 -> 14336, of
// 128: 297 -> 315; with channels handed on 64 of K at a time 73 and 350).
__host__ __device__ constexpr int accs(bool brief) { return brief ? 3 : 2; }
__host__ __device__ constexpr int channel_stages(bool brief) { return (kTmem - 128 * accs(brief)) / kColsA; }
// CTAs of a tile: a pair for many tokens
__host__ __device__ constexpr int ctas(int nt) { return nt > 64 ? 2 : 1; }
// a CTA's tokens
__host__ __device__ constexpr int own_tokens(int nt) { return nt / ctas(nt); }
// a stage of tokens x 128 of K, fp16
__host__ __device__ constexpr int stage_bytes(int nt) { return own_tokens(nt) * kStepK * 2; }
// the ring of codes as they are: 128 channels and the tokens x 128 of K
// (the channels alone where tokens are fp16)
__host__ __device__ constexpr int raw_bytes(int nt, bool half) { return (128 + (half ? 0 : own_tokens(nt))) * kStepK; }
__host__ __device__ constexpr int raw_stages(int nt, bool half) {
    return half ? (nt == 256 ? 4 : nt == 32 ? 11 : 9) : nt == 32 ? 8 : 6;
}
// columns of a drain warp that are written out at a time, and the room for those
// of all: 128 channels x two halves, float32
__host__ __device__ constexpr int out_cols(int nt) { return nt == 256 ? 32 : 16; }
__host__ __device__ constexpr int out_bytes(int nt) { return 2 * out_cols(nt) * 128 * 4; }
__host__ __device__ constexpr int ring_bytes(int nt, bool half) {
    return kStages * stage_bytes(nt) + raw_stages(nt, half) * raw_bytes(nt, half);
}
__host__ __device__ constexpr int smem_bytes(int nt, bool half) { return 1024 + ring_bytes(nt, half) + out_bytes(nt) + nt * 4 + 512; }
constexpr bool rings_fit(bool half) {
    for (int nt = 32; nt <= (half ? 256 : 128); nt *= 2)
        if (smem_bytes(nt, half) > 227 * 1024 || 8 * (4 * kStages + 3 * 3 + 2 * raw_stages(nt, half) + 1) + 8 > 512)
            return false;
    return true;
}
static_assert(rings_fit(false) && rings_fit(true), "rings and barriers must fit an SM's shared memory");

// A block's threads, and registers a thread of each role where the drain needs
// more than an even share.  The roles' sum may not pass what the block is launched
// with, or they would wait for registers that never come: ptxas compiles for the
// `launch` registers that the launch bounds leave, and the build checks its count.
template <int NT, bool VEC, bool HALF>
struct Block {
    // 256 tokens, fp16 only: a stage takes four converting warps 600 of the 1024
    // cycles of its MMAs, and the drain can hold a whole part besides its sums
    static constexpr bool lean = NT == 256;
    static_assert(!lean || (VEC && HALF), "tiles of 256 tokens: fp16 tokens and aligned channels");
    static constexpr int convert = lean ? 128 : 256;
    static constexpr int threads = 128 + convert + kDrain + (VEC ? 0 : kFill);
    static constexpr bool splits = lean || (NT == 128 && !VEC);
    static constexpr int launch = lean ? 128 : VEC ? 96 : 72;
    static constexpr int few = 48, conv = lean ? 64 : 56, drain = lean ? 200 : 112, fill = 56;
    static_assert(!splits || 128 * few + convert * conv + kDrain * drain + (VEC ? 0 : kFill * fill) <= launch * threads,
                  "the roles' registers must fit the block's");
};

template <uint32_t kPolls>
__device__ __forceinline__ bool wait_cluster(uint32_t bar, uint32_t parity) {
#pragma unroll 1
    for (uint32_t i = 0; i < kPolls; ++i) {
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
__device__ __forceinline__ uint4 load_shared(uint32_t addr) {
    uint4 v;
    asm volatile("ld.shared.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(addr) : "memory");
    return v;
}
__device__ __forceinline__ void store_shared(uint32_t addr, const uint4 &v) {
    asm volatile("st.shared.v4.u32 [%0], {%1, %2, %3, %4};" ::"r"(addr), "r"(v.x), "r"(v.y), "r"(v.z), "r"(v.w) : "memory");
}
// D (+)= A B^T, A in TMEM; of a pair in the TMEM of both CTAs (128 rows each)
__device__ __forceinline__ void mma_tmem(uint32_t d, uint32_t a, uint64_t bdesc, uint32_t idesc, uint32_t accumulate) {
    asm volatile(
        "{\n .reg .pred p;\n setp.ne.b32 p, %4, 0;\n"
        " tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n}\n" ::"r"(d),
        "r"(a), "l"(bdesc), "r"(idesc), "r"(accumulate)
        : "memory");
}
__device__ __forceinline__ void mma_tmem_pair(uint32_t d, uint32_t a, uint64_t bdesc, uint32_t idesc, uint32_t accumulate) {
    asm volatile(
        "{\n .reg .pred p;\n setp.ne.b32 p, %4, 0;\n"
        " tcgen05.mma.cta_group::2.kind::f16 [%0], [%1], %2, %3, p;\n}\n" ::"r"(d),
        "r"(a), "l"(bdesc), "r"(idesc), "r"(accumulate)
        : "memory");
}

// Two codes of w as fp16: c + 128 in the low bits of 1024 + (c + 128), less 1152.
__device__ __forceinline__ uint32_t to_half2(uint32_t w, uint32_t sel) {
    const uint32_t h = __byte_perm(w, 0x64646464u, sel);
    const __half2 d = __hsub2(*reinterpret_cast<const __half2 *>(&h), __half2half2(__ushort_as_half(0x6480)));
    return *reinterpret_cast<const uint32_t *>(&d);
}
// 16 codes as fp16, two a word
__device__ __forceinline__ void convert16(const uint4 &raw, uint32_t *h) {
    const uint32_t w[4] = {raw.x ^ 0x80808080u, raw.y ^ 0x80808080u, raw.z ^ 0x80808080u, raw.w ^ 0x80808080u};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        h[2 * i] = to_half2(w[i], 0x4140);
        h[2 * i + 1] = to_half2(w[i], 0x4342);
    }
}

// Chunks first .. last - 1 (16 of K each, multiples of four) of a stage's 128
// channels: from the raw ring, a thread a channel, to the TMEM lanes of quarter q.
__device__ __forceinline__ void convert_channels(uint32_t raw, uint32_t tmem, int q, int lane, int first, int last) {
    const int r = 32 * q + lane, sw = r & 7;
    const uint32_t src = raw + (uint32_t)(r * kStepK), to = tmem + ((uint32_t)(32 * q) << 16);
#pragma unroll 1
    for (int c = first; c < last; c += 4) {
        uint4 v[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) v[j] = load_shared(src + (((c + j) ^ sw) << 4));
#pragma unroll
        for (int j = 0; j < 4; j += 2) {
            uint32_t h[16];
            convert16(v[j], h);
            convert16(v[j + 1], h + 8);
            tc::tmem_st16(to + 8 * (c + j), h);
        }
    }
}

// The drain warps meet; all of them go on only if `ok` in each.
__device__ __forceinline__ void drain_barrier() { asm volatile("bar.sync 1, %0;" ::"n"(kDrain) : "memory"); }
__device__ __forceinline__ bool all_drain_warps(bool ok) {
    uint32_t r;
    asm volatile(
        "{\n .reg .pred p, q;\n setp.ne.u32 q, %1, 0;\n bar.red.and.pred p, 1, %2, q;\n selp.u32 %0, 1, 0, p;\n}\n"
        : "=r"(r)
        : "r"((uint32_t)ok), "n"(kDrain)
        : "memory");
    return r != 0;
}

// Whether eight channels of a token, the first a multiple of eight, are whole 16 bytes of Y.
__device__ __forceinline__ bool vector_out(const ProductArgs &a) {
    return (((uintptr_t)a.Y | (size_t)a.ldy * (a.dtype == JARQ_F32 ? 4 : 2)) & 15) == 0;
}
// Channel j of drain thread t in write_out: eight in a row, or four 32 apart.
__device__ __forceinline__ int out_channel(bool vector, int t, int j) {
    return vector ? 8 * (t & 15) + j : (t & 31) + 32 * (j & 3);
}

// 2 kOut tokens x 128 channels of staged sums (float32, or int32 without groups),
// scaled, to Y: rows r < kOut are tokens first + r, the others kCols further on.
// Threads t of 256; o: the first channel; xs: of token first.
template <bool GROUPS, int kOut, int kCols>
__device__ __forceinline__ void write_out(const ProductArgs &a, uint32_t staged, const float *xs, int t, int first, int o,
                                          bool vector, const float (&scale)[8], const float (&bias)[8]) {
    auto token = [&](int r) { return r < kOut ? r : r - kOut + kCols; };
    auto value = [&](uint32_t raw, float x, int j) {
        return fmaf(GROUPS ? __uint_as_float(raw) : (float)(int)raw * scale[j], x, bias[j]);
    };
    const size_t size = a.dtype == JARQ_F32 ? 4 : 2;
    if (vector) {
        const int oc = o + 8 * (t & 15);
#pragma unroll
        for (int r = t >> 4; r < 2 * kOut; r += 16) {
            const int c = token(r), tk = first + c;
            if (tk >= a.n || oc >= a.dout) continue;
            const uint32_t at = staged + (uint32_t)(r * 128 + 8 * (t & 15)) * 4;
            const uint4 lo = load_shared(at), hi = load_shared(at + 16);
            const uint32_t raw[8] = {lo.x, lo.y, lo.z, lo.w, hi.x, hi.y, hi.z, hi.w};
            const float x = xs[c];
            float y[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) y[j] = value(raw[j], x, j);
            char *p = static_cast<char *>(a.Y) + ((size_t)tk * a.ldy + oc) * size;
            if (oc + 8 > a.dout) {
#pragma unroll 1
                for (int j = 0; oc + j < a.dout; ++j)
                    with_type_device(a.dtype, [&](auto type) {
                        using T = decltype(type);
                        float v = y[0];
#pragma unroll
                        for (int i = 1; i < 8; ++i) v = i == j ? y[i] : v;
                        reinterpret_cast<T *>(p)[j] = from_float<T>(v);
                    });
            } else if (a.dtype == JARQ_F32) {
                reinterpret_cast<float4 *>(p)[0] = make_float4(y[0], y[1], y[2], y[3]);
                reinterpret_cast<float4 *>(p)[1] = make_float4(y[4], y[5], y[6], y[7]);
            } else {
                *reinterpret_cast<uint4 *>(p) = a.dtype == JARQ_F16 ? pack(y, __half()) : pack(y, __nv_bfloat16());
            }
        }
        return;
    }
    with_type_device(a.dtype, [&](auto type) {
        using T = decltype(type);
#pragma unroll 1
        for (int r = t >> 5; r < 2 * kOut; r += 8) {
            const int c = token(r), tk = first + c;
            if (tk >= a.n) continue;
            const float x = xs[c];
            T *p = static_cast<T *>(a.Y) + (size_t)tk * a.ldy + o;
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const int ch = (t & 31) + 32 * j;
                uint32_t raw;
                asm volatile("ld.shared.u32 %0, [%1];" : "=r"(raw) : "r"(staged + (uint32_t)(r * 128 + ch) * 4) : "memory");
                if (o + ch < a.dout) p[ch] = from_float<T>(value(raw, x, j));
            }
        }
    });
}

// NT: tokens of a tile.  GROUPS: group scales.  VEC: rows of codes on 16-byte
// boundaries.  HALF: tokens are integers in fp16, rows on 16-byte boundaries.
// kBrief: groups of 64, NT 256.
// kStalled: for the self-test, the issuer stops after one accumulator.
template <int NT, bool GROUPS, bool VEC, bool HALF, bool kBrief, bool kStalled>
__global__ void __launch_bounds__(Block<NT, VEC, HALF>::threads, 1)
    tc_integer_kernel(const __grid_constant__ CUtensorMap mapC, const __grid_constant__ CUtensorMap mapX, ProductArgs a,
                      int split, int *failed) {
    constexpr uint32_t kPolls = tc::wait_polls(kStalled);
    using B = Block<NT, VEC, HALF>;
    constexpr int kDrain0 = 4 + B::convert / 32, kFill0 = kDrain0 + kDrain / 32;   // first warps
    constexpr int kStage = stage_bytes(NT), kRaws = raw_stages(NT, HALF), kRaw = raw_bytes(NT, HALF);
    constexpr int kAcc = acc_cols(NT), kParts = acc_parts(NT);
    constexpr bool kPair = ctas(NT) == 2;
    constexpr int kChannels = 128 * ctas(NT);   // of a tile
    constexpr int kRowsB = kAcc / ctas(NT);     // this CTA's tokens of an accumulator
    constexpr int kAtomB = kRowsB * 128, kHalfB = 2 * kAtomB;
    // Columns of a drain warp in an accumulator, and how many of a unit's it reads:
    // half of each, or all of one, where the two warps of a scheduler so take turns
    // at reading TMEM and at adding
    constexpr int kCols = kBrief ? kAcc : kAcc / 2, kReads = kBrief ? 1 : kParts;
    constexpr bool kShare = !kPair && !HALF;    // the tokens' converters have time for channels
    // warps that convert a stage, and those of a pair's odd CTA that pass it on
    constexpr int kConverters = HALF ? 4 : B::convert / 32, kRelays = 3;
    constexpr int kAccs = accs(kBrief), kStagesA = channel_stages(kBrief);
    constexpr bool kApart = kStagesA != kStages;   // channels have barriers of their own
    static_assert(!kBrief || (GROUPS && B::lean), "converted tokens share their barriers with the channels");
    constexpr int kBarsA = kApart ? 2 * kStagesA : 0;
    using Accs = Turn<kAccs, kParts, kBrief>;
    constexpr int kReports = Accs::kReports;
    constexpr int kBars = 2 * kStages + kReports + kAccs + 2 * kRaws + kBarsA + 1;
    constexpr uint32_t kIdesc = tc::idesc_f16_f32(kChannels, kAcc);
    extern __shared__ uint8_t smem_raw[];
    uint8_t *smem = (uint8_t *)(((uintptr_t)smem_raw + 1023) & ~(uintptr_t)1023);
    float *sxs = (float *)(smem + ring_bytes(NT, HALF) + out_bytes(NT));   // the tile's token scales
    uint64_t *bars = (uint64_t *)(sxs + NT);
    uint32_t *tmem_slot = (uint32_t *)(bars + kBars);
    volatile int *abort_flag = (volatile int *)(tmem_slot + 1);
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int crank = (int)tc::cluster_rank(), rank = kPair ? crank & 1 : 0, part = crank / ctas(NT);
    const uint32_t even = crank - rank;
    const int nclusters = gridDim.x / (ctas(NT) * split), cluster = blockIdx.x / (ctas(NT) * split);
    const int mt = (a.dout + kChannels - 1) / kChannels, ntiles = mt * ((a.n + NT - 1) / NT);
    // this pair's part of K
    const int steps = (a.din + kStepK - 1) / kStepK, per = (steps + split - 1) / split;
    const int step0 = min(steps, part * per), nsteps = min(steps, step0 + per) - step0;
    const int natoms = max(0, min((a.din + 63) / 64 - 2 * step0, 2 * nsteps));
    const int ua = GROUPS ? a.g / 64 : kExact;               // atoms of an accumulator
    const int nunits = (natoms + ua - 1) / ua;

    auto full = [&](int s) { return tc::smem_u32(bars + s); };
    auto empty = [&](int s) { return tc::smem_u32(bars + kStages + s); };
    auto afull = [&](int b) { return tc::smem_u32(bars + 2 * kStages + b); };
    auto aempty = [&](int b) { return tc::smem_u32(bars + 2 * kStages + kReports + b); };
    auto raw_full = [&](int s) { return tc::smem_u32(bars + 2 * kStages + kReports + kAccs + s); };
    auto raw_empty = [&](int s) { return tc::smem_u32(bars + 2 * kStages + kReports + kAccs + kRaws + s); };
    auto full_a = [&](int s) { return kApart ? tc::smem_u32(bars + kBars - 1 - kBarsA + s) : full(s); };
    auto empty_a = [&](int s) { return kApart ? tc::smem_u32(bars + kBars - 1 - kBarsA + kStagesA + s) : empty(s); };
    const uint32_t closing = tc::smem_u32(bars + kBars - 1);
    const uint32_t ring = tc::smem_u32(smem), raws = ring + kStages * kStage, staged = ring + ring_bytes(NT, HALF);

    if (threadIdx.x == 0) {
        for (int s = 0; s < kStages; ++s) {
            // own converters and the other CTA's relay; with fp16 tokens, in the
            // issuer's CTA only, both CTAs' converters and the tokens' bytes
            tc::mbar_init(full(s), kApart ? 1 : HALF ? ctas(NT) * kConverters + 1 : kConverters + (kPair && rank == 0));
            tc::mbar_init(empty(s), 1);
        }
        for (int s = 0; s < kBarsA / 2; ++s) {
            tc::mbar_init(full_a(s), ctas(NT) * kConverters);
            tc::mbar_init(empty_a(s), 1);
        }
        for (int b = 0; b < kReports; ++b) tc::mbar_init(afull(b), 1);
        for (int b = 0; b < kAccs; ++b)
            tc::mbar_init(aempty(b), ctas(NT) * kDrain / 32 * kReads / kParts);   // the even CTA's: both drains
        for (int s = 0; s < kRaws; ++s) {
            tc::mbar_init(raw_full(s), VEC ? 1 : kFill / 32);
            tc::mbar_init(raw_empty(s), kConverters);
        }
        tc::mbar_init(closing, 1);
        *abort_flag = 0;
        tc::fence_barrier_init();
    }
    if (warp == 1) {
        if (kPair) {
            tc::tmem_alloc_pair(tc::smem_u32(tmem_slot), kTmem);
            tc::tmem_relinquish_pair();
        } else {
            tc::tmem_alloc(tc::smem_u32(tmem_slot), kTmem);
            tc::tmem_relinquish();
        }
    }
    tc::tc_fence_before();
    __syncthreads();
    if (kPair) tc::cluster_sync();
    tc::tc_fence_after();
    const uint32_t tmem = *tmem_slot, tmem_a = tmem + kAccs * 128;

    if (warp < 4) {
        if constexpr (B::splits) registers_down<B::few>();
        if (warp == 0 && rank == 0) {
            // ---------------- MMA issuer of the pair
            bool ok = true;
            const uint64_t bd0 = tc::sdesc_sw128(ring);
            const uint16_t both = (uint16_t)(3 << even);
            const int us = GROUPS ? max(1, ua / 2) : kExact / 2;     // stages of an accumulator
            Slot<kStages> in(0);
            Slot<kStagesA> chan(0);
            Accs turn(1);
            int unit = 0;                                    // over all tiles
            // `count` atoms from atom `at` of a stage into every part's accumulator
            auto mma = [&](uint32_t d, uint32_t ad, uint64_t bd, uint32_t add) {
                if (kPair)
                    mma_tmem_pair(d, ad, bd, kIdesc, add);
                else
                    mma_tmem(d, ad, bd, kIdesc, add);
            };
            auto commit = [&](uint32_t bar) {
                if (kPair)
                    tc::mma_commit_pair(bar, both);
                else
                    tc::mma_commit(bar);
            };
            auto issue = [&](int at, int count, bool first, bool last, bool done) {
#pragma unroll
                for (int h = 0; h < kParts; ++h) {
                    const int b = turn.acc(h);
                    if (first) {
                        ok = tc::mbar_wait<kPolls>(aempty(b), turn.parity(h));
                        if (!ok) return;
                        tc::tc_fence_after();
                    }
                    if (tc::elect_one()) {
                        const uint32_t d = tmem + b * kAcc;
                        const uint32_t ad = tmem_a + chan.s * kColsA + at * 32;
                        const uint64_t bd = bd0 + (uint32_t)((in.s * kStage + h * kHalfB + at * kAtomB) >> 4);
#pragma unroll
                        for (int sub = 0; sub < 4; ++sub) mma(d, ad + 8 * sub, bd + 2 * sub, !first || sub > 0);
                        if (count == 2) {
#pragma unroll
                            for (int sub = 0; sub < 4; ++sub)
                                mma(d, ad + 32 + 8 * sub, bd + (kAtomB >> 4) + 2 * sub, 1);
                        }
                        if (last) commit(afull(turn.report(h)));
                        if (done && h == kParts - 1) {
                            commit(empty(in.s));
                            if (kApart) commit(empty_a(chan.s));
                        }
                    }
                    __syncwarp();
                }
                unit += last;
                if (last) turn.next();
            };
            for (int tile = cluster; tile < ntiles && ok; tile += nclusters)
                for (int step = 0, in_unit = 0; step < nsteps && ok; ++step, in.next(), chan.next()) {
                    if (kStalled && unit > 0) break;
                    ok = kPair && !HALF ? wait_cluster<kPolls>(full(in.s), in.phase) : tc::mbar_wait<kPolls>(full(in.s), in.phase);
                    if (kApart) ok = tc::mbar_wait<kPolls>(full_a(chan.s), chan.phase) && ok;
                    if (!ok) break;
                    tc::tc_fence_after();
                    const int atoms = min(2, natoms - 2 * step);
                    if (GROUPS && ua == 1) {
                        issue(0, 1, true, true, atoms == 1);
                        if (ok && atoms == 2) issue(1, 1, true, true, true);
                    } else {
                        const bool last = in_unit + 1 == us || step + 1 == nsteps;
                        issue(0, atoms, in_unit == 0, last, true);
                        in_unit = last ? 0 : in_unit + 1;
                    }
                }
            if (tc::elect_one()) {
                if (kPair)
                    tc::mma_commit_pair(closing, 1 << even);
                else
                    tc::mma_commit(closing);
            }
            if (!tc::mbar_wait<kPolls>(closing, 0) || !ok) *abort_flag = 1;
        } else if (kPair && !HALF && rank == 1 && warp != 2) {
            // ---------------- relays of the odd CTA: its stages are full, in turn
            const uint32_t full0 = tc::map_rank(full(0), even);
            const int me = warp == 3 ? 2 : warp;
            bool ok = true;
            int turn = 0;
            Slot<kStages> in(0);
            for (int tile = cluster; tile < ntiles && ok; tile += nclusters)
                for (int step = 0; step < nsteps && ok; ++step, in.next()) {
                    if (turn == me) {
                        ok = tc::mbar_wait<kPolls>(full(in.s), in.phase);
                        tc::tc_fence_after();
                        tc::tc_fence_before();
                        if (ok && lane == 0) arrive_cluster(full0 + 8 * in.s);
                        __syncwarp();
                    }
                    turn = turn == kRelays - 1 ? 0 : turn + 1;
                }
            if (!ok) *abort_flag = 1;
        } else if (VEC && warp == 2) {
            // ---------------- producer of the raw ring
            if (!HALF) tc::pdl_wait();
            bool ok = true;
            Slot<kRaws> out(1);
            int filled = 0;
            for (int tile = cluster; tile < ntiles && ok; tile += nclusters) {
                const int o = tile % mt * kChannels + 128 * rank, tk = tile / mt * NT + kRowsB * rank;
                for (int step = 0; step < nsteps; ++step, out.next()) {
                    ok = tc::mbar_wait<kPolls>(raw_empty(out.s), out.phase);
                    if (!ok) break;
                    if (tc::elect_one()) {
                        const uint32_t at = raws + out.s * kRaw, bar = raw_full(out.s);
                        const int k = (step0 + step) * kStepK;
                        tc::mbar_expect_tx(bar, kRaw);
                        tc::tma_load_2d(at, &mapC, bar, k, o);
                        if (!HALF) {
#pragma unroll
                            for (int h = 0; h < kParts; ++h)
                                tc::tma_load_2d(at + (128 + h * kRowsB) * kStepK, &mapX, bar, k, tk + h * kAcc);
                        }
                    }
                    __syncwarp();
                    ++filled;
                }
            }
            // no copy is in flight when the CTA ends
            for (int n = max(0, filled - kRaws); n < filled && ok; ++n)
                ok = tc::mbar_wait<kPolls>(raw_empty(n % kRaws), (n / kRaws) & 1);
            if (!ok) {
                *abort_flag = 1;
                tc::abandon_ring(raw_full(0), kRaws, filled, true);
            }
        } else if (HALF && warp == 3) {
            // ---------------- producer of the tokens, onto the issuer's barriers
            tc::pdl_wait();
            const uint32_t full0 = kPair ? tc::map_rank(full(0), even) : full(0);
            bool ok = true;
            Slot<kStages> out(1);
            int filled = 0;
            for (int tile = cluster; tile < ntiles && ok; tile += nclusters) {
                const int tk = tile / mt * NT + kRowsB * rank;
                for (int step = 0; step < nsteps; ++step, out.next()) {
                    ok = tc::mbar_wait<kPolls>(empty(out.s), out.phase);
                    if (!ok) break;
                    if (tc::elect_one()) {
                        const uint32_t bar = full0 + 8 * out.s;
                        const int k = (step0 + step) * kStepK;
                        if (rank == 0) tc::mbar_expect_tx(bar, ctas(NT) * kStage);
#pragma unroll
                        for (int h = 0; h < kParts; ++h)
#pragma unroll
                            for (int at = 0; at < 2; ++at) {
                                const uint32_t dst = ring + out.s * kStage + h * kHalfB + at * kAtomB;
                                if (kPair)
                                    tc::tma_load_2d_pair(dst, &mapX, bar, k + 64 * at, tk + h * kAcc);
                                else
                                    tc::tma_load_2d(dst, &mapX, bar, k + 64 * at, tk + h * kAcc);
                            }
                    }
                    __syncwarp();
                    ++filled;
                }
            }
            for (int n = max(0, filled - kStages); n < filled && ok; ++n)
                ok = tc::mbar_wait<kPolls>(empty(n % kStages), (n / kStages) & 1);
            if (!ok) {
                *abort_flag = 1;
                tc::abandon_ring(full(0), kStages, filled, rank == 0);
            }
        }
    } else if (warp < 8 || (HALF && warp < kDrain0)) {
        if constexpr (B::splits) registers_down<B::conv>();
        // ---------------- channels: raw ring -> fp16 -> TMEM
        const uint32_t full0 = tc::map_rank(full_a(0), even);
        bool ok = true, turn = warp >= 8;
        Slot<kRaws> in(0);
        Slot<kStagesA> out(1);
        for (int tile = cluster; tile < ntiles && ok; tile += nclusters)
            for (int step = 0; step < nsteps; ++step, in.next(), out.next()) {
                if (HALF && B::convert == 256 && (turn = !turn, !turn)) continue;     // the other four warps' stage
                ok = tc::mbar_wait<kPolls>(raw_full(in.s), in.phase);
                ok = tc::mbar_wait<kPolls>(empty_a(out.s), out.phase) && ok;
                ok = __all_sync(0xffffffffu, ok);
                if (!ok) break;
                tc::tc_fence_after();
                convert_channels(raws + in.s * kRaw, tmem_a + out.s * kColsA, warp & 3, lane, 0, kShare ? 4 : 8);
                tc::tmem_wait_st();
                tc::tc_fence_before();
                __syncwarp();
                if (lane == 0) {
                    if (kPair && HALF)
                        tc::mbar_arrive_cluster(full0 + 8 * out.s);
                    else
                        tc::mbar_arrive(full_a(out.s));
                    tc::mbar_arrive(raw_empty(in.s));
                }
            }
        if (!ok) *abort_flag = 1;
    } else if (warp < kDrain0) {
        if constexpr (B::splits) registers_down<B::conv>();
        // ---------------- tokens: raw ring -> fp16 -> K-major tiles, 128-byte swizzle
        constexpr int kU = own_tokens(NT) / 16;              // 16 rows at a time
        constexpr int kBatch = kU < 4 ? kU : 4;              // loads in flight
        const int t = threadIdx.x - 256, c = t & 7, r0 = t >> 3, sw = r0 & 7;
        // 16 codes become two 16-byte chunks of a 128-byte row; threads of the
        // second atom write theirs in the other order, so that eight lanes of a
        // row always cover all banks
        const int atom = c >> 2, j0 = 2 * (c & 3) + atom;
        const uint32_t to = ring + atom * kAtomB + r0 * 128;
        const uint32_t sw0 = (uint32_t)((j0 ^ sw) << 4), sw1 = (uint32_t)(((j0 ^ 1) ^ sw) << 4);
        const uint32_t from = raws + (uint32_t)((128 + r0) * kStepK + ((c ^ sw) << 4));
        bool ok = true;
        Slot<kRaws> in(0);
        Slot<kStages> out(1);
        for (int tile = cluster; tile < ntiles && ok; tile += nclusters)
            for (int step = 0; step < nsteps; ++step, in.next(), out.next()) {
                ok = tc::mbar_wait<kPolls>(raw_full(in.s), in.phase);
                ok = tc::mbar_wait<kPolls>(empty(out.s), out.phase) && ok;
                ok = __all_sync(0xffffffffu, ok);
                if (!ok) break;
                if (kShare) {
                    tc::tc_fence_after();
                    convert_channels(raws + in.s * kRaw, tmem_a + out.s * kColsA, warp & 3, lane, 4, 8);
                }
                const uint32_t src = from + in.s * kRaw, dst = to + out.s * kStage;
                uint4 raw[kBatch];
#pragma unroll 1
                for (int i = 0; i < kU; i += kBatch) {
#pragma unroll
                    for (int j = 0; j < kBatch; ++j) raw[j] = load_shared(src + (i + j) * 16 * kStepK);
#pragma unroll
                    for (int j = 0; j < kBatch; ++j) {
                        uint32_t h[8];
                        convert16(raw[j], h);
                        // row 16 (i + j) + r0 of the stage: part 16 (i + j) / kRowsB
                        const uint32_t d = dst + 16 * (i + j) / kRowsB * kHalfB + 16 * (i + j) % kRowsB * 128;
                        const uint4 lo = make_uint4(h[0], h[1], h[2], h[3]), hi = make_uint4(h[4], h[5], h[6], h[7]);
                        store_shared(d + sw0, atom ? hi : lo);
                        store_shared(d + sw1, atom ? lo : hi);
                    }
                }
                fence_to_async();
                if (kShare) {
                    tc::tmem_wait_st();
                    tc::tc_fence_before();
                }
                __syncwarp();
                if (lane == 0) {
                    tc::mbar_arrive(full(out.s));
                    tc::mbar_arrive(raw_empty(in.s));
                }
            }
        if (!ok) *abort_flag = 1;
    } else if (warp < kFill0) {
        if constexpr (B::splits) registers_up<B::drain>();
        // ---------------- drain
        tc::pdl_wait();                                      // the tokens' scales
        float *factors = (float *)(smem + ring_bytes(NT, HALF));   // scale and bias; then staged outputs
        const int t = threadIdx.x - 32 * kDrain0, w = warp - kDrain0, q = w & 3, col0 = (w >> 2) * kCols, mine = kBrief ? w >> 2 : 0;
        const int lrow = 32 * q + lane;
        const uint32_t released = tc::map_rank(aempty(0), even);
        const uint32_t taddr = tmem + ((uint32_t)(32 * q) << 16) + (kBrief ? 0 : col0);
        bool ok = true;
        Accs turn(0);
        for (int tile = cluster; tile < ntiles && ok; tile += nclusters) {
            const int o = tile % mt * kChannels + 128 * rank + lrow, t0 = tile / mt * NT;
            const bool live = o < a.dout;
            // what the outputs are scaled with, under the products
            if (t < NT) sxs[t] = t0 + t < a.n ? a.xs[t0 + t] : 0.f;
            if (t < 128) {
                const int ch = tile % mt * kChannels + 128 * rank + t;
                factors[t] = !GROUPS && ch < a.dout ? a.ws[ch] : 1.f;
                factors[128 + t] = a.bias && ch < a.dout ? a.bias[ch] : 0.f;
            }
            uint32_t acc[kReads][kCols];                    // int32, or float32 with groups
#pragma unroll
            for (int h = 0; h < kReads; ++h)
#pragma unroll
                for (int e = 0; e < kCols; ++e) acc[h][e] = 0;
            const float *wp = a.ws + (live ? (size_t)o * a.G : 0) + (GROUPS ? 2 * step0 / ua : 0);
            for (int u = 0; u < nunits && ok; ++u, turn.next()) {
                const float wsc = GROUPS ? wp[u] : 0.f;
#pragma unroll
                for (int h = 0; h < kReads; ++h) {
                    const int b = turn.acc(h + mine);
                    ok = __all_sync(0xffffffffu, tc::mbar_wait<kPolls>(afull(turn.report(h + mine)), turn.report_parity(h + mine))) && ok;
                    if (!ok) break;
                    tc::tc_fence_after();
                    const uint32_t at = taddr + b * kAcc;
                    // the accumulator is handed back once it is in registers: at
                    // once where they allow, else with its last columns
                    constexpr int kHeld = kBrief ? 32 : B::lean ? kCols : 16;
                    uint32_t v[kHeld < kCols ? 2 : 1][kHeld];
                    auto load = [&](int cc) {
#pragma unroll
                        for (int i = 0; i < kHeld; i += 16)
                            tc::tmem_ld16(at + cc + i, *reinterpret_cast<uint32_t(*)[16]>(&v[cc / kHeld & (kHeld < kCols)][i]));
                    };
                    load(0);
#pragma unroll
                    for (int cc = 0; cc < kCols; cc += kHeld) {
                        tc::tmem_wait_ld();
                        if (cc + kHeld < kCols) {
                            load(cc + kHeld);
                        } else {
                            tc::tc_fence_before();
                            __syncwarp();
                            if (lane == 0) {
                                if (kPair)
                                    tc::mbar_arrive_cluster(released + 8 * b);
                                else
                                    tc::mbar_arrive(aempty(b));
                            }
                        }
                        uint32_t *x = v[cc / kHeld & (kHeld < kCols)];
#pragma unroll
                        for (int e = 0; e < kHeld; e += 2) {
                            uint32_t *s = &acc[h][cc + e];
                            if (GROUPS) {
                                const tc::F2 v2 = tc::f2(__uint_as_float(x[e]), __uint_as_float(x[e + 1]));
                                float lo, hi;
                                tc::f2_get(tc::f2_fma(v2, tc::f2(wsc), tc::f2(__uint_as_float(s[0]), __uint_as_float(s[1]))), lo, hi);
                                s[0] = __float_as_uint(lo);
                                s[1] = __float_as_uint(hi);
                            } else {
                                // (the integer by additions that bring it to the low bits: of
                                // all 256 of K at a time 468, of 10 in 16 values with 1024 of K
                                // 472 us for 8192 x 11008 x 4096, against 458)
                                s[0] += (uint32_t)__float2int_rn(__uint_as_float(x[e]));
                                s[1] += (uint32_t)__float2int_rn(__uint_as_float(x[e + 1]));
                            }
                        }
                    }
                }
            }
            // all drain warps or none go on: the rest meets at barriers
            ok = all_drain_warps(ok);
            if (!ok) break;
            if (split > 1) {
                // every MMA of the pair is done: its ring takes the partial sums
#pragma unroll
                for (int h = 0; h < kReads; ++h)
#pragma unroll
                    for (int e = 0; e < kCols; ++e)
                        asm volatile("st.shared.u32 [%0], %1;" ::"r"(ring + (uint32_t)((h * kAcc + col0 + e) * 128 + lrow) * 4),
                                     "r"(acc[h][e])
                                     : "memory");
                break;                                       // joined below: one tile a cluster
            }
            // Out through shared memory, a few columns of each warp at a time: a
            // thread scales eight channels of a token.  (Each value scaled and stored
            // from its register, code without a loop, took 16000 cycles a tile.)
            constexpr int kOut = out_cols(NT);
            const bool vector = vector_out(a);
            float scale[8], bias[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                scale[j] = factors[out_channel(vector, t, j)];
                bias[j] = factors[128 + out_channel(vector, t, j)];
            }
            drain_barrier();
#pragma unroll
            for (int h = 0; h < kReads; ++h)
#pragma unroll
                for (int c0 = 0; c0 < kCols; c0 += kOut) {
#pragma unroll
                    for (int e = 0; e < kOut; ++e)
                        asm volatile("st.shared.u32 [%0], %1;" ::"r"(staged + (uint32_t)(((w >> 2) * kOut + e) * 128 + lrow) * 4),
                                     "r"(acc[h][c0 + e])
                                     : "memory");
                    drain_barrier();
                    write_out<GROUPS, kOut, kCols>(a, staged, sxs + h * kAcc + c0, t, t0 + h * kAcc + c0, tile % mt * kChannels + 128 * rank,
                                                   vector, scale, bias);
                    drain_barrier();
                }
        }
        if (!ok) *abort_flag = 1;
    } else {
        if constexpr (B::splits) registers_down<B::fill>();
        // ---------------- rows that TMA cannot read, into the raw ring
        if (!HALF) tc::pdl_wait();
        constexpr int kRows = 128 + (HALF ? 0 : own_tokens(NT)), kU = (kRows + 31) / 32;   // 32 rows at a time: channels, tokens
        constexpr int kBatch = 4;
        const int t = threadIdx.x - 32 * kFill0, c = t & 7, r0 = t >> 3;
        const uint32_t to = raws + (uint32_t)(r0 * kStepK + ((c ^ (r0 & 7)) << 4));
        bool ok = true;
        Slot<kRaws> out(1);
        for (int tile = cluster; tile < ntiles && ok; tile += nclusters) {
            const int o = tile % mt * kChannels + 128 * rank + r0, tk = tile / mt * NT + kRowsB * rank;
            // row r0 + 32 i of the stage, null where there is none
            auto row_of = [&](int i) -> const int8_t * {
                if (i < 4) return o + 32 * i < a.dout ? a.C + (size_t)(o + 32 * i) * a.ldc : nullptr;
                const int j = r0 + 32 * (i - 4), r = tk + j / kRowsB * kAcc + j % kRowsB;
                return j < own_tokens(NT) && r < a.n ? static_cast<const int8_t *>(a.X) + (size_t)r * a.ldx : nullptr;
            };
            for (int step = 0; step < nsteps; ++step, out.next()) {
                const int k = (step0 + step) * kStepK + c * 16;
                ok = tc::mbar_wait<kPolls>(raw_empty(out.s), out.phase);
                if (!ok) break;
                const uint32_t dst = to + out.s * kRaw;
#pragma unroll 1
                for (int i0 = 0; i0 < kU; i0 += kBatch) {
                    uint4 v[kBatch];
                    if (k >= 4 && k + 20 <= a.din) {
                        // inside the rows: whole words, all in flight
                        uint32_t w[kBatch][5], sel[kBatch];
#pragma unroll
                        for (int j = 0; j < kBatch; ++j) {
                            const int8_t *row = row_of(i0 + j);
                            sel[j] = row ? (uint32_t)((uintptr_t)(row + k) & 3) : 4;
#pragma unroll
                            for (int e = 0; e < 5; ++e)
                                w[j][e] = row ? reinterpret_cast<const uint32_t *>(row + k - sel[j])[e] : 0;
                        }
#pragma unroll
                        for (int j = 0; j < kBatch; ++j) {
                            const uint32_t p = 0x3210u + 0x1111u * (sel[j] & 3);
                            v[j] = make_uint4(__byte_perm(w[j][0], w[j][1], p), __byte_perm(w[j][1], w[j][2], p),
                                              __byte_perm(w[j][2], w[j][3], p), __byte_perm(w[j][3], w[j][4], p));
                        }
                    } else {
#pragma unroll
                        for (int j = 0; j < kBatch; ++j) {
                            const int8_t *row = row_of(i0 + j);
                            v[j] = row ? load_codes<false>(row, k, a.din) : make_uint4(0, 0, 0, 0);
                        }
                    }
#pragma unroll
                    for (int j = 0; j < kBatch; ++j)
                        if (r0 + 32 * (i0 + j) < kRows) store_shared(dst + (i0 + j) * 32 * kStepK, v[j]);
                }
                __syncwarp();
                if (lane == 0) tc::mbar_arrive(raw_full(out.s));
            }
        }
        if (!ok) *abort_flag = 1;
    }
    if (split > 1) {
        // join: part `part` of K finishes columns part cols .. of its 128 channels
        cluster_barrier();
        if (warp >= kDrain0 && warp < kFill0 && cluster < ntiles) {
            const int t = threadIdx.x - 32 * kDrain0, lrow = t & 127, half = t >> 7;
            const int o = cluster % mt * kChannels + 128 * rank + lrow, t0 = cluster / mt * NT;
            const int cols = (NT + split - 1) / split;       // columns past NT are skipped
            const float bias = a.bias && o < a.dout ? a.bias[o] : 0.f, wch = !GROUPS && o < a.dout ? a.ws[o] : 1.f;
            constexpr int kAtOnce = 4;                       // columns in flight
#pragma unroll 1
            for (int e0 = half; e0 < cols; e0 += 2 * kAtOnce) {
                uint32_t v[kAtOnce][kMostParts];
#pragma unroll
                for (int j = 0; j < kAtOnce; ++j) {
                    const int col = part * cols + e0 + 2 * j;
                    const uint32_t at = ring + (uint32_t)(col * 128 + lrow) * 4;
#pragma unroll
                    for (int p = 0; p < kMostParts; ++p)
                        v[j][p] = p < split && e0 + 2 * j < cols ? load_remote(tc::map_rank(at, ctas(NT) * p + rank)) : 0;
                }
#pragma unroll
                for (int j = 0; j < kAtOnce; ++j) {
                    const int col = part * cols + e0 + 2 * j;
                    if (e0 + 2 * j >= cols || col >= NT || o >= a.dout || t0 + col >= a.n) continue;
                    float f = 0.f;
                    int i = 0;
#pragma unroll
                    for (int p = 0; p < kMostParts; ++p) {
                        f += __uint_as_float(v[j][p]);
                        i += (int)v[j][p];
                    }
                    const float y = fmaf(GROUPS ? f : (float)i * wch, a.xs[t0 + col], bias);
                    with_type_device(a.dtype, [&](auto type) {
                        using T = decltype(type);
                        static_cast<T *>(a.Y)[(size_t)(t0 + col) * a.ldy + o] = from_float<T>(y);
                    });
                }
            }
        }
    }
    // neither CTA leaves while another may still read its shared memory, signal
    // its barriers or hold TMEM of the pair
    tc::tc_fence_before();
    __syncwarp();
    __syncthreads();
    if (kPair || split > 1) tc::cluster_sync();
    if (warp == 1) {
        tc::tc_fence_after();
        if (kPair)
            tc::tmem_dealloc_pair(tmem, kTmem);
        else
            tc::tmem_dealloc(tmem, kTmem);
    }
    if (threadIdx.x == 0 && *abort_flag) {
        *(volatile int *)failed = 1;
        __threadfence_system();
    }
}

template <int NT, bool GROUPS, bool VEC, bool HALF, bool kBrief = false, bool kStalled = false>
cudaError_t launch(const ProductArgs &a, int split, int *failed, cudaStream_t s, bool pdl) {
    static std::atomic<unsigned long long> done;
    auto *kernel = tc_integer_kernel<NT, GROUPS, VEC, HALF, kBrief, kStalled>;
    cudaError_t e = set_max_dynamic_smem((const void *)kernel, smem_bytes(NT, HALF), done);
    if (e != cudaSuccess) return e;
    CUtensorMap mapC = {}, mapX = {};
    auto pitch = [](int64_t ld, int rows) { return (uint64_t)(rows > 1 ? ld : (ld + 15) / 16 * 16); };
    constexpr int rows = acc_cols(NT) / ctas(NT);
    if (VEC) e = make_tmap_codes(&mapC, a.C, a.dout, a.din, pitch(a.ldc, a.dout), 128);
    if (e == cudaSuccess && HALF)
        e = make_tmap_half(&mapX, a.X, a.n, a.din, pitch(a.ldx, a.n), rows);
    else if (e == cudaSuccess && VEC)
        e = make_tmap_codes(&mapX, static_cast<const int8_t *>(a.X), a.n, a.din, pitch(a.ldx, a.n), rows);
    if (e != cudaSuccess) return e;
    const int64_t tiles = (int64_t)((a.dout + 128 * ctas(NT) - 1) / (128 * ctas(NT))) * ((a.n + NT - 1) / NT);
    const int64_t clusters = split > 1 ? tiles : std::min<int64_t>(tiles, num_sms() / ctas(NT));
    if (tiles > 0x3FFFFFFF / (2 * split)) return cudaErrorInvalidValue;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)(clusters * ctas(NT) * split));
    cfg.blockDim = dim3(Block<NT, VEC, HALF>::threads);
    cfg.dynamicSmemBytes = smem_bytes(NT, HALF);
    cfg.stream = s;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = ctas(NT) * split;
    attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
    attr[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[1].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = pdl ? 2 : 1;
    return cudaLaunchKernelEx(&cfg, kernel, mapC, mapX, a, split, failed);
}

template <int NT, bool VEC, bool HALF>
cudaError_t launch_scales(const ProductArgs &a, int split, int *failed, cudaStream_t s, bool pdl) {
    if constexpr (NT == 256)
        if (a.g == 64) return launch<NT, true, VEC, HALF, true>(a, split, failed, s, pdl);
    return a.g ? launch<NT, true, VEC, HALF>(a, split, failed, s, pdl) : launch<NT, false, VEC, HALF>(a, split, failed, s, pdl);
}
template <int NT>
cudaError_t launch_nt(const ProductArgs &a, int split, int *failed, cudaStream_t s, bool pdl) {
    if constexpr (NT == 256) return launch_scales<256, true, true>(a, split, failed, s, pdl);
    else if (a.half)
        return vector_codes(a) ? launch_scales<NT, true, true>(a, split, failed, s, pdl)
                               : launch_scales<NT, false, true>(a, split, failed, s, pdl);
    else
        return vector_rows(a) ? launch_scales<NT, true, false>(a, split, failed, s, pdl)
                              : launch_scales<NT, false, false>(a, split, failed, s, pdl);
}

}  // namespace

cudaError_t launch_tc_integer_stalled(const ProductArgs &a, int *failed, cudaStream_t s) {
    return launch<256, false, true, true, false, true>(a, 1, failed, s, false);
}

cudaError_t launch_tc_integer(const ProductArgs &a, int *failed, cudaStream_t s, bool pdl) {
    // The tile's tokens and the split of K that take the least time: waves of
    // clusters, each so many steps of 128 of K and what a tile costs besides
    // (cycles, fitted to 28 layers of 8 to 8000 tokens; within 3 % of the best of
    // all choices).  Of clusters of four CTAs 36 run at a time, of six 23, of eight 15
    // (occupancy calculator, 152 SMs: a cluster's SMs lie in one GPC).
    constexpr struct {
        int nt, step, tile;
    } kinds[] = {{32, 530, 5000}, {64, 530, 7500}, {128, 530, 10000}, {256, 940, 17000}};
    constexpr int resident[] = {0, 152, 76, 48, 36, 0, 23, 0, 15};
    const bool vec = a.half ? vector_codes(a) : vector_rows(a);
    const int steps = (a.din + kStepK - 1) / kStepK, sms = num_sms();
    int nt = 0, split = 1;
    double best = 0;
    for (const auto &k : kinds) {
        if (k.nt == 256 && !(vec && a.half)) continue;
        for (int sp = 1; sp <= std::min(kMostParts, steps); ++sp) {
            const int channels = 128 * ctas(k.nt), at_once = std::max(1, resident[ctas(k.nt) * sp] * sms / 152);
            const int64_t tiles = (int64_t)((a.dout + channels - 1) / channels) * ((a.n + k.nt - 1) / k.nt);
            if (sp > 1 && tiles > at_once) break;
            const double waves = (double)((tiles + at_once - 1) / at_once);
            const double t = waves * ((steps + sp - 1) / sp) * k.step * (vec ? 1 : 2) + waves * k.tile + (sp > 1 ? 500 : 0);
            if (nt == 0 || t < best) {
                best = t;
                nt = k.nt;
                split = sp;
            }
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
