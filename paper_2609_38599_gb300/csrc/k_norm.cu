// Root-mean-square norm of rows with the residual's addition, its outputs in the
// rows' type and in 8-bit integers, and its gradient.
//
//   h = round(x + r),  rstd = (mean_k h_k^2 + eps)^(-1/2),  v = h gain,
//   y = round(v rstd),  a = max_k |v_k|,  scale = (a / 127) rstd,  q = rint(v (127 / a)).
// rstd is one number a row, so it goes into the row's scale and the integers do
// not depend on the order of the sum behind it.  With u = dy gain and z = h rstd,
//   dx = dh + rstd (u - z mean_k u_k z_k),   dgain = sum_t dy z.
// (z is of unit size whatever the row's; rstd^2 and dy h are not, and leave float32's
// range for rows of 1e19 and more or less than its inverse.)
//
// One pass over memory.  More than a row an SM: blocks go from row to row with the next
// rows on their way into shared memory.  Few rows: a block a row, which holds it in
// registers from the loads to the outputs, and the gains' gradient by columns beside it.
// Threads of a row and the order of its sums go by its width and by whether the rows lie on
// 16-byte boundaries, so that a row's outputs do not depend on the batch.  Rows are read 16 bytes at a time where every
// array's rows lie on 16-byte boundaries, else an element at a time, neighbouring threads
// reading neighbouring elements.
//
// Bound by memory, near the issue slots (70 % of them in the forward): on the device, cold
//   8192 x 4096 bfloat16, residual, integers     40 us (235 MB, 5.8 TB/s)
//   its gradient, with a residual's and gains'   53 us (268 MB, 5.1 TB/s; 47 and the join of
//                                                the blocks' parts, 7.5 MB, in a launch of its own)
//   one row of 4096, residual                    3.4 us (a launch and three latencies)
//   48 x 11008 float16, gradient                 6.0 us
//   7653 x 997 float16, residual, values         26 us (rows on no boundary: an element a lane)
// A block of one row each, and of several without a ring, took 65 us and 204.  Two elements
// an instruction throughout: 41 and 57.
#include <math.h>

#include <algorithm>
#include <type_traits>

#include "integer.cuh"
#include "quantize.cuh"
#include "rows.cuh"

namespace jarq {
namespace {

using namespace rows;

constexpr int kMostGradBlocks = 608;       // four for each of 152 SMs
constexpr int kFewGradRows = 152;          // most rows of the gradient's form for few

// Elements that a thread reads at a time, how often it does so and keeps them, and
// so the longest row that P threads hold.  (1024 threads have 64 registers each.)
template <class T, bool VEC, int P>
struct Shape {
    static constexpr int E = VEC ? kUnit<T> : 1, held = !VEC ? 8 : P == 1024 ? 16 / E : 4, row = P * E * held;
};

// Elements k .. k + E - 1 of a row of d.
template <int E, class T>
__device__ __forceinline__ void load(const T *p, int k, int d, float (&v)[E]) {
    if constexpr (E == 1) {
        v[0] = to_float(p[k]);
    } else if (k + E <= d) {
        if constexpr (E == kUnit<T>) {
            unpack(*reinterpret_cast<const uint4 *>(p + k), v, T());
        } else {                            // float32 beside a 16-bit type
            static_assert(E == 2 * kUnit<T>, "two units of float32");
            const float4 lo = reinterpret_cast<const float4 *>(p + k)[0], hi = reinterpret_cast<const float4 *>(p + k)[1];
            v[0] = lo.x, v[1] = lo.y, v[2] = lo.z, v[3] = lo.w;
            v[4] = hi.x, v[5] = hi.y, v[6] = hi.z, v[7] = hi.w;
        }
    } else {
#pragma unroll
        for (int e = 0; e < E; ++e) v[e] = k + e < d ? to_float(p[k + e]) : 0.f;
    }
}
template <int E, class T>
__device__ __forceinline__ void store(T *p, int k, int d, const float (&v)[E]) {
    if constexpr (E == 1) {
        p[k] = from_float<T>(v[0]);
    } else if (k + E <= d) {
        *reinterpret_cast<uint4 *>(p + k) = pack(v, T());
    } else {
#pragma unroll
        for (int e = 0; e < E; ++e)
            if (k + e < d) p[k + e] = from_float<T>(v[e]);
    }
}
template <int E>
__device__ __forceinline__ void store_codes(int8_t *p, int k, int d, const int (&q)[E]) {
    if constexpr (E == 1) {
        p[k] = (int8_t)q[0];
    } else if (k + E <= d) {
        uint32_t w[E / 4];
#pragma unroll
        for (int i = 0; i < E / 4; ++i)
            w[i] = __byte_perm(__byte_perm(q[4 * i], q[4 * i + 1], 0x0040), __byte_perm(q[4 * i + 2], q[4 * i + 3], 0x0040), 0x5410);
        if constexpr (E == 8)
            *reinterpret_cast<uint2 *>(p + k) = make_uint2(w[0], w[1]);
        else
            *reinterpret_cast<uint32_t *>(p + k) = w[0];
    } else {
#pragma unroll
        for (int e = 0; e < E; ++e)
            if (k + e < d) p[k + e] = (int8_t)q[e];
    }
}
// The gains of elements k ..: 1 where there are none, float32 or of the rows' type.
template <int E, class T>
__device__ __forceinline__ void load_gain(const void *gain, bool wide, int k, int d, float (&g)[E]) {
    if (!gain) {
#pragma unroll
        for (int e = 0; e < E; ++e) g[e] = 1.f;
    } else if (wide) {
        load<E>(static_cast<const float *>(gain), k, d, g);
    } else {
        load<E>(static_cast<const T *>(gain), k, d, g);
    }
}

__device__ __forceinline__ float warp_sum(float x) {
#pragma unroll
    for (int off = 16; off; off /= 2) x += __shfl_xor_sync(0xffffffffu, x, off);
    return x;
}
// The sum over a row's P threads, in all of them, the same bits in each.
// `part`: P / 32 floats; two sums in a row need two of them.
template <int P>
__device__ __forceinline__ float row_sum(float x, float *part) {
    x = warp_sum(x);
    if constexpr (P > 32) {
        if ((threadIdx.x & 31) == 0) part[threadIdx.x >> 5] = x;
        __syncthreads();
        x = warp_sum((threadIdx.x & 31) < P / 32 ? part[threadIdx.x & 31] : 0.f);
    }
    return x;
}

// 1 / sqrt(mean + eps) of a sum of squares over a row; `again(by)` is the sum of (by h)^2
// over the row, which is read once more where sum or eps leave what float32 holds in full
// (an infinity in the row stays one, and rstd is 0).
template <class F>
__device__ __forceinline__ float inverse_rms(float sum, int d, float eps, F again) {
    const float mean = sum / (float)d + eps;
    if (isinf(mean)) return 0x1p-80f / sqrtf(again(0x1p-80f) / (float)d + eps * 0x1p-80f * 0x1p-80f);
    if (mean < 0x1p-100f) return 0x1p64f / sqrtf(again(0x1p64f) / (float)d + eps * 0x1p64f * 0x1p64f);
    return 1.f / sqrtf(mean);
}

struct NormArgs {
    const void *X, *R, *gain;
    void *H, *Y;
    int8_t *Q;
    float *scale, *rstd;
    int64_t ldx, ldr, ldh, ldy, ldq;
    int n, d;
    float eps;
    bool wide_gain;
};

// T: element type; VEC: rows on 16-byte boundaries; P: threads of a row (a block of
// 256 has several rows where P is 32).
template <class T, bool VEC, int P>
__global__ void __launch_bounds__(P == 32 ? 256 : P) norm_kernel(NormArgs a) {
    constexpr int E = Shape<T, VEC, P>::E, kHeld = Shape<T, VEC, P>::held;
    __shared__ float sums[2][32];
    __shared__ uint32_t tops[32];
    const int t = P == 32 ? threadIdx.x & 31 : threadIdx.x;
    const int64_t r = P == 32 ? (int64_t)blockIdx.x * 8 + (threadIdx.x >> 5) : blockIdx.x;
    if (r >= a.n) return;
    const T *x = static_cast<const T *>(a.X) + r * a.ldx, *res = static_cast<const T *>(a.R) + r * a.ldr;
    T *h = static_cast<T *>(a.H) + r * a.ldh, *y = static_cast<T *>(a.Y) + r * a.ldy;
    int8_t *q = a.Q + r * a.ldq;
    // what a later pass over the row reads
    const T *again = a.R ? h : x;

    auto read = [&](int k, float (&v)[E]) {
        load<E>(x, k, a.d, v);
        if (a.R) {
            float o[E];
            load<E>(res, k, a.d, o);
#pragma unroll
            for (int e = 0; e < E; ++e) v[e] = to_float(from_float<T>(v[e] + o[e]));
            store<E>(h, k, a.d, v);
        }
    };
    float held[kHeld][E];
    float sum = 0.f;
    uint32_t top = 0;
    auto take = [&](int k, float (&v)[E]) {
        float g[E];
        load_gain<E, T>(a.gain, a.wide_gain, k, a.d, g);
#pragma unroll
        for (int e = 0; e < E; ++e) {
            sum = fmaf(v[e], v[e], sum);
            v[e] = __fmul_rn(v[e], g[e]);
            top = max(top, __float_as_uint(v[e]) & 0x7FFFFFFFu);
        }
    };
#pragma unroll
    for (int i = 0; i < kHeld; ++i)
        if ((t + i * P) * E < a.d) read((t + i * P) * E, held[i]);
#pragma unroll
    for (int i = 0; i < kHeld; ++i)
        if ((t + i * P) * E < a.d) take((t + i * P) * E, held[i]);
    for (int64_t k = (int64_t)(t + kHeld * P) * E; k < a.d; k += P * E) {
        float v[E];
        read((int)k, v);
        take((int)k, v);
    }
    sum = warp_sum(sum);
    top = __reduce_max_sync(0xffffffffu, top);
    if constexpr (P > 32) {
        if ((threadIdx.x & 31) == 0) {
            sums[0][threadIdx.x >> 5] = sum;
            tops[threadIdx.x >> 5] = top;
        }
        __syncthreads();
        const int w = threadIdx.x & 31;
        sum = warp_sum(w < P / 32 ? sums[0][w] : 0.f);
        top = __reduce_max_sync(0xffffffffu, w < P / 32 ? tops[w] : 0u);
    }
    const float rstd = inverse_rms(sum, a.d, a.eps, [&](float by) {
        float part = 0.f;
        for (int64_t k = (int64_t)t * E; k < a.d; k += P * E) {
            float v[E];
            load<E>(again, (int)k, a.d, v);
#pragma unroll
            for (int e = 0; e < E; ++e) part = fmaf(v[e] * by, v[e] * by, part);
        }
        return row_sum<P>(part, sums[1]);
    });
    const quant::RowScale by(top);
    if (t == 0) {
        if (a.rstd) a.rstd[r] = rstd;
        if (a.scale) a.scale[r] = __fmul_rn(by.scale, rstd);
    }
    auto put = [&](int k, const float (&v)[E]) {
        if (a.Y) {
            float o[E];
#pragma unroll
            for (int e = 0; e < E; ++e) o[e] = v[e] * rstd;
            store<E>(y, k, a.d, o);
        }
        if (a.Q) {
            int c[E];
#pragma unroll
            for (int e = 0; e < E; ++e) c[e] = by.bad ? 0 : __float2int_rn(__fmul_rn(v[e], by.inv));
            store_codes<E>(q, k, a.d, c);
        }
    };
#pragma unroll
    for (int i = 0; i < kHeld; ++i)
        if ((t + i * P) * E < a.d) put((t + i * P) * E, held[i]);
    for (int64_t k = (int64_t)(t + kHeld * P) * E; k < a.d; k += P * E) {
        float v[E], g[E];
        load<E>(again, (int)k, a.d, v);
        load_gain<E, T>(a.gain, a.wide_gain, (int)k, a.d, g);
#pragma unroll
        for (int e = 0; e < E; ++e) v[e] = __fmul_rn(v[e], g[e]);
        put((int)k, v);
    }
}

struct GradArgs {
    const void *H, *gain, *dY, *dH;
    void *dX;
    const float *rstd;
    float *part;               // [blocks][d] sums of the gains' gradient, or null
    int64_t ldh, ldy, lds, ldx;
    int n, d;
    bool wide_gain;
};

// A block goes from row to row; a thread has the same columns of each, and so their
// part of the gains' gradient in registers.  GAIN: it is wanted, and a row fits
// what the threads hold.
template <class T, bool VEC, int P, bool GAIN>
__global__ void __launch_bounds__(P) norm_grad_kernel(GradArgs a) {
    constexpr int E = Shape<T, VEC, P>::E, kHeld = Shape<T, VEC, P>::held;
    __shared__ float part[2][32];
    tc::pdl_launch_dependents();
    const int t = threadIdx.x;
    float acc[GAIN ? kHeld : 1][E];
    if constexpr (GAIN)
#pragma unroll
        for (int i = 0; i < kHeld; ++i)
#pragma unroll
            for (int e = 0; e < E; ++e) acc[i][e] = 0.f;
    int turn = 0;
    for (int64_t r = blockIdx.x; r < a.n; r += gridDim.x, turn ^= 1) {
        const T *h = static_cast<const T *>(a.H) + r * a.ldh, *dy = static_cast<const T *>(a.dY) + r * a.ldy;
        const T *dh = static_cast<const T *>(a.dH) + r * a.lds;
        T *dx = static_cast<T *>(a.dX) + r * a.ldx;
        const float rstd = a.rstd[r];
        float hv[kHeld][E], u[kHeld][E], dot = 0.f;
#pragma unroll
        for (int i = 0; i < kHeld; ++i) {
            const int k = (t + i * P) * E;
            if (k >= a.d) continue;
            load<E>(h, k, a.d, hv[i]);
            load<E>(dy, k, a.d, u[i]);
        }
#pragma unroll
        for (int i = 0; i < kHeld; ++i) {
            const int k = (t + i * P) * E;
            if (k >= a.d) continue;
            float g[E];
            load_gain<E, T>(a.gain, a.wide_gain, k, a.d, g);
#pragma unroll
            for (int e = 0; e < E; ++e) {
                hv[i][e] *= rstd;
                if constexpr (GAIN) acc[i][e] = fmaf(u[i][e], hv[i][e], acc[i][e]);
                u[i][e] = __fmul_rn(u[i][e], g[e]);
                dot = fmaf(u[i][e], hv[i][e], dot);
            }
        }
        if constexpr (!GAIN)
            for (int64_t k = (int64_t)(t + kHeld * P) * E; k < a.d; k += P * E) {
                float v[E], w[E], g[E];
                load<E>(h, (int)k, a.d, v);
                load<E>(dy, (int)k, a.d, w);
                load_gain<E, T>(a.gain, a.wide_gain, (int)k, a.d, g);
#pragma unroll
                for (int e = 0; e < E; ++e)
                    dot = fmaf(__fmul_rn(w[e], g[e]), __fmul_rn(v[e], rstd), dot);
            }
        if (!a.dX) continue;
        // the launch before this one may be reading dY still, where dX is dY
        if (!GAIN && turn == 0) tc::pdl_wait();
        // the two rows of `part` take turns: one is written while the other may still be read
        const float along = row_sum<P>(dot, part[turn]) / (float)a.d;
        // of z and u
        auto put = [&](int k, const float (&v)[E], const float (&w)[E]) {
            float o[E], s[E];
            if (a.dH) load<E>(dh, k, a.d, s);
#pragma unroll
            for (int e = 0; e < E; ++e) {
                const float x = fmaf(-v[e], along, w[e]);
                o[e] = a.dH ? fmaf(x, rstd, s[e]) : x * rstd;
            }
            store<E>(dx, k, a.d, o);
        };
#pragma unroll
        for (int i = 0; i < kHeld; ++i) {
            const int k = (t + i * P) * E;
            if (k < a.d) put(k, hv[i], u[i]);
        }
        if constexpr (!GAIN)
            for (int64_t k = (int64_t)(t + kHeld * P) * E; k < a.d; k += P * E) {
                float v[E], w[E], g[E];
                load<E>(h, (int)k, a.d, v);
                load<E>(dy, (int)k, a.d, w);
                load_gain<E, T>(a.gain, a.wide_gain, (int)k, a.d, g);
#pragma unroll
                for (int e = 0; e < E; ++e) {
                    v[e] = __fmul_rn(v[e], rstd);
                    w[e] = __fmul_rn(w[e], g[e]);
                }
                put((int)k, v, w);
            }
    }
    if constexpr (GAIN) {
        float *to = a.part + (size_t)blockIdx.x * a.d;
#pragma unroll
        for (int i = 0; i < kHeld; ++i)
#pragma unroll
            for (int e = 0; e < E; ++e)
                if ((t + i * P) * E + e < a.d) to[(t + i * P) * E + e] = acc[i][e];
    }
}

// The gains' gradient by columns, 32 a block, in parts of `rows_each` rows: of rows too
// long to be held, with gain_join_kernel after it, and of few rows in one part.
template <class T>
__global__ void __launch_bounds__(256) gain_columns_kernel(GradArgs a, int rows_each) {
    __shared__ float part[8][32];
    tc::pdl_launch_dependents();
    const int lane = threadIdx.x & 31, w = threadIdx.x >> 5;
    const int64_t k = (int64_t)blockIdx.x * 32 + lane;
    const int64_t r0 = (int64_t)blockIdx.y * rows_each, r1 = min((int64_t)a.n, r0 + rows_each);
    float acc = 0.f;
    if (k < a.d) {
        constexpr int kBatch = 8;                  // rows in flight
        for (int64_t b = r0 + w; b < r1; b += 8 * kBatch) {
            float y[kBatch], h[kBatch], s[kBatch];
#pragma unroll
            for (int j = 0; j < kBatch; ++j) {
                const int64_t r = b + 8 * j;
                const bool in = r < r1;
                y[j] = in ? to_float(static_cast<const T *>(a.dY)[r * a.ldy + k]) : 0.f;
                h[j] = in ? to_float(static_cast<const T *>(a.H)[r * a.ldh + k]) : 0.f;
                s[j] = in ? a.rstd[r] : 0.f;
            }
#pragma unroll
            for (int j = 0; j < kBatch; ++j) acc = fmaf(y[j], h[j] * s[j], acc);
        }
    }
    part[w][lane] = acc;
    __syncthreads();
    if (w == 0 && k < a.d) {
#pragma unroll
        for (int i = 1; i < 8; ++i) acc += part[i][lane];
        a.part[(size_t)blockIdx.y * a.d + k] = acc;
    }
}

// dgain[k] = sum of its parts, always in the same order.
__global__ void __launch_bounds__(1024) gain_join_kernel(const float *parts, int count, int d, float *dgain) {
    __shared__ float part[32][33];
    const int lane = threadIdx.x & 31, w = threadIdx.x >> 5;
    const int64_t k = (int64_t)blockIdx.x * 32 + lane;
    tc::pdl_wait();
    float acc = 0.f;
    if (k < d)
        for (int i0 = w; i0 < count; i0 += 32 * 8) {
            float v[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) v[j] = i0 + 32 * j < count ? parts[(size_t)(i0 + 32 * j) * d + k] : 0.f;
#pragma unroll
            for (int j = 0; j < 8; ++j) acc += v[j];
        }
    part[w][lane] = acc;
    __syncthreads();
    acc = warp_sum(part[lane][w]);                 // column w of the block's 32
    const int64_t c = (int64_t)blockIdx.x * 32 + w;
    if (lane == 0 && c < d) dgain[c] = acc;
}

// ---------------------------------------------------------------- many rows
// A block goes from row to row.  A thread has the same units of each, which it copies
// into its own places of a ring in shared memory rows ahead: they are read by no other
// thread, so that a copy needs no barrier, and what a row waits for is its sum alone.
// The gains stay in registers.  P: threads, HELD: units of 16 bytes of a thread.
constexpr int kMostShared = 220 * 1024;
template <int P, int HELD, int ARRAYS>
struct Ring {
    static constexpr int stage = P * HELD * ARRAYS * 16;
    static constexpr int stages = 3 * stage <= kMostShared ? 3 : 2, bytes = stages * stage;
    // blocks of an SM, by threads and by shared memory
    static constexpr int resident = 768 / P < 1 ? 1 : 768 / P < kMostShared / bytes ? 768 / P : kMostShared / bytes;
    __device__ static uint4 *at(uint4 *ring, int s, int array, int i) {
        return ring + ((s * ARRAYS + array) * HELD + i) * P + threadIdx.x;
    }
};
// 16 bytes, or the `bytes` that are left of a row and zeros
__device__ __forceinline__ void copy_ahead(uint4 *to, const void *from, int bytes) {
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(tc::smem_u32(to)), "l"(from), "r"(bytes) : "memory");
}
__device__ __forceinline__ void copies_made() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int LEFT>
__device__ __forceinline__ void copies_landed() {
    asm volatile("cp.async.wait_group %0;" ::"n"(LEFT) : "memory");
}
template <class R, class T, int HELD, int P>
__device__ __forceinline__ void copy_row(uint4 *ring, int s, int array, const T *row, int d) {
    constexpr int E = kUnit<T>;
#pragma unroll
    for (int i = 0; i < HELD; ++i) {
        const int k = (threadIdx.x + i * P) * E;
        if (k < d) copy_ahead(R::at(ring, s, array, i), row + k, min(E, d - k) * (int)sizeof(T));
    }
}

template <class T, int P, int HELD, bool RES>
__global__ void __launch_bounds__(P, Ring<P, HELD, 1 + RES>::resident) norm_rows_kernel(NormArgs a) {
    using R = Ring<P, HELD, 1 + RES>;
    constexpr int E = kUnit<T>;
    extern __shared__ uint4 ring[];
    __shared__ float sums[2][32], again[32];
    __shared__ uint32_t tops[2][32];
    const int t = threadIdx.x, w = t & 31;
    const T *X = static_cast<const T *>(a.X), *S = static_cast<const T *>(a.R);
    float g[HELD][E];
#pragma unroll
    for (int i = 0; i < HELD; ++i)
        if ((t + i * P) * E < a.d) load_gain<E, T>(a.gain, a.wide_gain, (t + i * P) * E, a.d, g[i]);
    auto ahead = [&](int64_t r, int s) {
        if (r < a.n) {
            copy_row<R, T, HELD, P>(ring, s, 0, X + r * a.ldx, a.d);
            if (RES) copy_row<R, T, HELD, P>(ring, s, 1, S + r * a.ldr, a.d);
        }
        copies_made();
    };
    for (int s = 0; s + 1 < R::stages; ++s) ahead(blockIdx.x + (int64_t)s * gridDim.x, s);
    int s = 0, turn = 0;
    for (int64_t r = blockIdx.x; r < a.n; r += gridDim.x, turn ^= 1) {
        ahead(r + (int64_t)(R::stages - 1) * gridDim.x, s == 0 ? R::stages - 1 : s - 1);
        copies_landed<R::stages - 1>();
        T *h = static_cast<T *>(a.H) + r * a.ldh;
        float v[HELD][E], sum = 0.f;
        uint32_t top = 0;
#pragma unroll
        for (int i = 0; i < HELD; ++i) {
            const int k = (t + i * P) * E;
            if (k >= a.d) continue;
            unpack(*R::at(ring, s, 0, i), v[i], T());
            if (RES) {
                float o[E];
                unpack(*R::at(ring, s, 1, i), o, T());
#pragma unroll
                for (int e = 0; e < E; ++e) v[i][e] += o[e];
                const uint4 raw = pack(v[i], T());
                if (k + E <= a.d) {
                    *reinterpret_cast<uint4 *>(h + k) = raw;
                    unpack(raw, v[i], T());
                } else {
                    unpack(raw, v[i], T());
                    store<E>(h, k, a.d, v[i]);
                }
            }
#pragma unroll
            for (int e = 0; e < E; ++e) {
                sum = fmaf(v[i][e], v[i][e], sum);
                v[i][e] = __fmul_rn(v[i][e], g[i][e]);
                top = max(top, __float_as_uint(v[i][e]) & 0x7FFFFFFFu);
            }
        }
        sum = warp_sum(sum);
        top = __reduce_max_sync(0xffffffffu, top);
        if (w == 0) {
            sums[turn][t >> 5] = sum;
            tops[turn][t >> 5] = top;
        }
        __syncthreads();
        sum = warp_sum(w < P / 32 ? sums[turn][w] : 0.f);
        top = __reduce_max_sync(0xffffffffu, w < P / 32 ? tops[turn][w] : 0u);
        const float rstd = inverse_rms(sum, a.d, a.eps, [&](float by) {
            // the row is still in the ring
            float part = 0.f;
#pragma unroll
            for (int i = 0; i < HELD; ++i) {
                if ((t + i * P) * E >= a.d) continue;
                float x[E], o[E];
                unpack(*R::at(ring, s, 0, i), x, T());
                if (RES) unpack(*R::at(ring, s, 1, i), o, T());
#pragma unroll
                for (int e = 0; e < E; ++e) {
                    if (RES) x[e] = to_float(from_float<T>(x[e] + o[e]));
                    part = fmaf(x[e] * by, x[e] * by, part);
                }
            }
            part = row_sum<P>(part, again);
            __syncthreads();                       // `again` is free for the next row
            return part;
        });
        const quant::RowScale by(top);
        if (t == 0) {
            if (a.rstd) a.rstd[r] = rstd;
            if (a.scale) a.scale[r] = __fmul_rn(by.scale, rstd);
        }
#pragma unroll
        for (int i = 0; i < HELD; ++i) {
            const int k = (t + i * P) * E;
            if (k >= a.d) continue;
            if (a.Y) {
                float o[E];
#pragma unroll
                for (int e = 0; e < E; ++e) o[e] = v[i][e] * rstd;
                store<E>(static_cast<T *>(a.Y) + r * a.ldy, k, a.d, o);
            }
            if (a.Q) {
                int c[E];
#pragma unroll
                for (int e = 0; e < E; ++e) c[e] = by.bad ? 0 : __float2int_rn(__fmul_rn(v[i][e], by.inv));
                store_codes<E>(a.Q + r * a.ldq, k, a.d, c);
            }
        }
        s = s + 1 == R::stages ? 0 : s + 1;
    }
}

template <class T, int P, int HELD, bool STREAM>
__global__ void __launch_bounds__(P, Ring<P, HELD, 2 + STREAM>::resident) norm_grad_rows_kernel(GradArgs a) {
    using R = Ring<P, HELD, 2 + STREAM>;
    constexpr int E = kUnit<T>;
    extern __shared__ uint4 ring[];
    __shared__ float part[2][32];
    tc::pdl_launch_dependents();
    const int t = threadIdx.x;
    const T *H = static_cast<const T *>(a.H), *Y = static_cast<const T *>(a.dY), *D = static_cast<const T *>(a.dH);
    float g[HELD][E], acc[HELD][E];
#pragma unroll
    for (int i = 0; i < HELD; ++i) {
        if ((t + i * P) * E < a.d) load_gain<E, T>(a.gain, a.wide_gain, (t + i * P) * E, a.d, g[i]);
#pragma unroll
        for (int e = 0; e < E; ++e) acc[i][e] = 0.f;
    }
    auto ahead = [&](int64_t r, int s) {
        if (r < a.n) {
            copy_row<R, T, HELD, P>(ring, s, 0, H + r * a.ldh, a.d);
            copy_row<R, T, HELD, P>(ring, s, 1, Y + r * a.ldy, a.d);
            if (STREAM) copy_row<R, T, HELD, P>(ring, s, 2, D + r * a.lds, a.d);
        }
        copies_made();
    };
    for (int s = 0; s + 1 < R::stages; ++s) ahead(blockIdx.x + (int64_t)s * gridDim.x, s);
    int s = 0, turn = 0;
    float next = a.rstd[blockIdx.x];
    for (int64_t r = blockIdx.x; r < a.n; r += gridDim.x, turn ^= 1) {
        ahead(r + (int64_t)(R::stages - 1) * gridDim.x, s == 0 ? R::stages - 1 : s - 1);
        const float rstd = next;
        if (r + gridDim.x < a.n) next = a.rstd[r + gridDim.x];
        copies_landed<R::stages - 1>();
        float dot = 0.f;
#pragma unroll
        for (int i = 0; i < HELD; ++i) {
            if ((t + i * P) * E >= a.d) continue;
            float h[E], u[E];
            unpack(*R::at(ring, s, 0, i), h, T());
            unpack(*R::at(ring, s, 1, i), u, T());
#pragma unroll
            for (int e = 0; e < E; ++e) {
                const float z = __fmul_rn(h[e], rstd);
                acc[i][e] = fmaf(u[e], z, acc[i][e]);
                // as norm_grad_kernel adds it, so that a row's gradient does not depend on the batch
                dot = fmaf(__fmul_rn(u[e], g[i][e]), z, dot);
            }
        }
        if (a.dX) {
            const float along = row_sum<P>(dot, part[turn]) / (float)a.d;
            T *dx = static_cast<T *>(a.dX) + r * a.ldx;
#pragma unroll
            for (int i = 0; i < HELD; ++i) {
                const int k = (t + i * P) * E;
                if (k >= a.d) continue;
                float h[E], u[E], o[E];
                unpack(*R::at(ring, s, 0, i), h, T());
                unpack(*R::at(ring, s, 1, i), u, T());
                if (STREAM) unpack(*R::at(ring, s, 2, i), o, T());
#pragma unroll
                for (int e = 0; e < E; ++e) {
                    const float x = fmaf(-__fmul_rn(h[e], rstd), along, __fmul_rn(u[e], g[i][e]));
                    o[e] = STREAM ? fmaf(x, rstd, o[e]) : x * rstd;
                }
                store<E>(dx, k, a.d, o);
            }
        }
        s = s + 1 == R::stages ? 0 : s + 1;
    }
    if (a.part) {
        float *to = a.part + (size_t)blockIdx.x * a.d;
#pragma unroll
        for (int i = 0; i < HELD; ++i)
#pragma unroll
            for (int e = 0; e < E; ++e)
                if ((t + i * P) * E + e < a.d) to[(t + i * P) * E + e] = acc[i][e];
    }
}

// The form for few rows holds four units a thread, so that P alone decides its sums.
// `f(P, HELD)`, as integral constants, for the fewest threads whose units hold a row of
// d elements of type T; false where none do.
template <class T, class F>
bool with_threads(int d, F f) {
    constexpr int E = kUnit<T>;
    using std::integral_constant;
    auto fits = [&](auto p, auto held) {
        if (d > p.value * held.value * E) return false;
        f(p, held);
        return true;
    };
    return fits(integral_constant<int, 128>(), integral_constant<int, 1>()) || fits(integral_constant<int, 128>(), integral_constant<int, 2>()) ||
           fits(integral_constant<int, 256>(), integral_constant<int, 2>()) || fits(integral_constant<int, 512>(), integral_constant<int, 2>()) ||
           fits(integral_constant<int, 512>(), integral_constant<int, 3>()) || fits(integral_constant<int, 1024>(), integral_constant<int, 2>());
}
// One launch of as many blocks as run at one time; `blocks`: how many those are.
template <class R, class K, class A>
cudaError_t launch_rows(K *kernel, std::atomic<unsigned long long> &done, int p, const A &a, int *blocks, cudaStream_t s) {
    const cudaError_t e = set_max_dynamic_smem((const void *)kernel, R::bytes, done);
    if (e != cudaSuccess) return e;
    *blocks = std::min(a.n, std::min(kMostGradBlocks, R::resident * num_sms()));
    return launch_k(kernel, dim3(*blocks), dim3(p), (size_t)R::bytes, s, false, a);
}
template <class T, int P, int HELD, bool RES>
cudaError_t launch_norm_rows(const NormArgs &a, cudaStream_t s) {
    static std::atomic<unsigned long long> done;
    int blocks;
    return launch_rows<Ring<P, HELD, 1 + RES>>(norm_rows_kernel<T, P, HELD, RES>, done, P, a, &blocks, s);
}
template <class T, int P, int HELD, bool STREAM>
cudaError_t launch_grad_rows(const GradArgs &a, int *blocks, cudaStream_t s) {
    static std::atomic<unsigned long long> done;
    return launch_rows<Ring<P, HELD, 2 + STREAM>>(norm_grad_rows_kernel<T, P, HELD, STREAM>, done, P, a, blocks, s);
}

template <class T, bool VEC, int P>
cudaError_t launch_norm_p(const NormArgs &a, cudaStream_t s) {
    const int64_t blocks = P == 32 ? ((int64_t)a.n + 7) / 8 : a.n;
    norm_kernel<T, VEC, P><<<(unsigned)blocks, P == 32 ? 256 : P, 0, s>>>(a);
    return cudaGetLastError();
}
template <class T, bool VEC>
cudaError_t launch_norm_t(const NormArgs &a, cudaStream_t s) {
    if (a.d <= Shape<T, VEC, 32>::row) return launch_norm_p<T, VEC, 32>(a, s);
    cudaError_t e = cudaSuccess;
    if (VEC) {
        // the threads by the width alone, so that a row's sum is added in one order
        if (with_threads<T>(a.d, [&](auto p, auto held) {
                constexpr int P = p.value, HELD = held.value;
                e = a.n <= num_sms() ? launch_norm_p<T, VEC, P>(a, s)
                    : a.R            ? launch_norm_rows<T, P, HELD, true>(a, s)
                                     : launch_norm_rows<T, P, HELD, false>(a, s);
            }))
            return e;
    } else {
        if (a.d <= Shape<T, VEC, 128>::row) return launch_norm_p<T, VEC, 128>(a, s);
        if (a.d <= Shape<T, VEC, 256>::row) return launch_norm_p<T, VEC, 256>(a, s);
        if (a.d <= Shape<T, VEC, 512>::row) return launch_norm_p<T, VEC, 512>(a, s);
    }
    return launch_norm_p<T, VEC, 1024>(a, s);
}

// after: gain_columns_kernel is the launch before, whose results it does not need.
template <class T, bool VEC, int P>
cudaError_t launch_grad_p(const GradArgs &a, int blocks, bool after, cudaStream_t s) {
    return a.part ? launch_k(norm_grad_kernel<T, VEC, P, true>, dim3(blocks), dim3(P), 0, s, false, a)
                  : launch_k(norm_grad_kernel<T, VEC, P, false>, dim3(blocks), dim3(P), 0, s, after, a);
}

template <class T, bool VEC>
cudaError_t launch_grad_t(GradArgs a, float *dgain, cudaStream_t s) {
    int parts = std::min(a.n, kMostGradBlocks);
    float *const part = a.part;
    cudaError_t e = cudaSuccess;
    const bool few = a.n <= kFewGradRows, apart = dgain && (few || a.d > Shape<T, VEC, 1024>::row);
    if (apart) {
        // few rows, or rows that no block holds: the columns' sums apart, and first, since
        // dX may be dY
        const int each = few ? a.n : (a.n + std::min(parts, 32) - 1) / std::min(parts, 32);
        parts = (a.n + each - 1) / each;
        GradArgs by = a;
        if (few) by.part = dgain;
        gain_columns_kernel<T><<<dim3((unsigned)(((int64_t)a.d + 31) / 32), parts), 256, 0, s>>>(by, each);
        count_launches(1);
        e = cudaGetLastError();
        a.part = nullptr;
    }
    if (e == cudaSuccess && (a.dX || a.part)) {
        int blocks = std::min(a.n, kMostGradBlocks);
        count_launches(1);
        if (VEC) {
            if (!with_threads<T>(a.d, [&](auto p, auto held) {
                    constexpr int P = p.value, HELD = held.value;
                    e = a.n <= kFewGradRows ? launch_grad_p<T, VEC, P>(a, blocks, apart, s)
                        : a.dH           ? launch_grad_rows<T, P, HELD, true>(a, &blocks, s)
                                         : launch_grad_rows<T, P, HELD, false>(a, &blocks, s);
                }))
                e = launch_grad_p<T, VEC, 1024>(a, blocks, apart, s);
        } else if (a.d <= Shape<T, VEC, 128>::row) {
            e = launch_grad_p<T, VEC, 128>(a, blocks, apart, s);
        } else if (a.d <= Shape<T, VEC, 512>::row) {
            e = launch_grad_p<T, VEC, 512>(a, blocks, apart, s);
        } else {
            e = launch_grad_p<T, VEC, 1024>(a, blocks, apart, s);
        }
        if (a.part) parts = blocks;
    }
    if (e == cudaSuccess && dgain && !few) {
        e = launch_pdl(gain_join_kernel, dim3((unsigned)(((int64_t)a.d + 31) / 32)), dim3(1024), 0, s, (const float *)part, parts,
                       a.d, dgain);
        count_launches(1);
    }
    return e;
}

bool aligned(const void *p, size_t b) { return ((uintptr_t)p & (b - 1)) == 0; }
// Whether all rows begin on 16-byte boundaries (n/a: no such array).
bool vector(const void *p, int64_t ld, int n, size_t size) {
    return !p || (aligned(p, 16) && (n == 1 || ld * (int64_t)size % 16 == 0));
}
bool usable(const void *p, size_t size) { return p && on_device(p) && aligned(p, size); }
bool usable_or_null(const void *p, size_t size) { return !p || usable(p, size); }

jarq_status finish(cudaError_t e) {
    if (e == cudaSuccess) return JARQ_OK;
    (void)cudaGetLastError();
    return JARQ_ERR_CUDA;
}

}  // namespace
}  // namespace jarq

using namespace jarq;

extern "C" {

jarq_status jarq_rms_norm(const void *X, jarq_dtype dtype, int n, int d, int64_t ldx, const void *R,
                          int64_t ldr, void *H, int64_t ldh, const void *gain, jarq_dtype gain_dtype,
                          float eps, void *Y, int64_t ldy, int8_t *Q, int64_t ldq, float *scale,
                          float *rstd, void *stream) {
    if (n < 0 || n > kMostIndex || d < 1 || d > kMostIndex || ldx < d || !is_dtype(dtype) || !(eps > 0.f) || isinf(eps))
        return JARQ_ERR_ARG;
    if (gain && gain_dtype != dtype && gain_dtype != JARQ_F32) return JARQ_ERR_ARG;
    if ((R != nullptr) != (H != nullptr) || (Q != nullptr) != (scale != nullptr)) return JARQ_ERR_ARG;
    if ((R && (ldr < d || ldh < d)) || (Y && ldy < d) || (Q && ldq < d) || (R == H && R && n > 1 && ldr != ldh))
        return JARQ_ERR_ARG;
    if (n == 0) return JARQ_OK;
    const size_t size = size_of(dtype);
    if (!usable(X, size) || !usable_or_null(R, size) || !usable_or_null(H, size) || !usable_or_null(Y, size) ||
        !usable_or_null(Q, 1) || !usable_or_null(scale, 4) || !usable_or_null(rstd, 4) ||
        !usable_or_null(gain, gain ? size_of(gain_dtype) : 1))
        return JARQ_ERR_ARG;
    if (const jarq_status late = async_failure()) return late;
    cudaStream_t st = (cudaStream_t)stream;
    const NormArgs a{X, R, gain, H, Y, Q, scale, rstd, ldx, ldr, ldh, ldy, ldq, n, d, eps, gain_dtype != dtype};
    const bool vec = vector(X, ldx, n, size) && vector(R, ldr, n, size) && vector(H, ldh, n, size) &&
                     vector(Y, ldy, n, size) && vector(gain, 0, 1, 1) &&
                     (!Q || (aligned(Q, 8) && (n == 1 || ldq % 8 == 0)));
    ProfScope ps("rms_norm", st);
    const cudaError_t e = with_type(dtype, [&](auto type) {
        using T = decltype(type);
        return vec ? launch_norm_t<T, true>(a, st) : launch_norm_t<T, false>(a, st);
    });
    ps.done();
    count_launches(1);
    return finish(e);
}

size_t jarq_rms_norm_grad_workspace(int n, int d) {
    if (n <= kFewGradRows || d < 1) return 0;
    return (size_t)std::min(n, kMostGradBlocks) * d * sizeof(float);
}

jarq_status jarq_rms_norm_grad(const void *H, jarq_dtype dtype, int n, int d, int64_t ldh,
                               const void *gain, jarq_dtype gain_dtype, const float *rstd,
                               const void *dY, int64_t ldy, const void *dH, int64_t lds, void *dX,
                               int64_t ldx, float *dgain, void *workspace, size_t workspace_bytes,
                               void *stream) {
    if (n < 0 || n > kMostIndex || d < 1 || d > kMostIndex || ldh < d || ldy < d || !is_dtype(dtype)) return JARQ_ERR_ARG;
    if ((gain && gain_dtype != dtype && gain_dtype != JARQ_F32) || (dH && lds < d) || (dX && ldx < d)) return JARQ_ERR_ARG;
    if (!dX && !dgain) return JARQ_ERR_ARG;
    if (n > 1 && dX && ((dX == dY && ldx != ldy) || (dX == dH && ldx != lds))) return JARQ_ERR_ARG;
    cudaStream_t st = (cudaStream_t)stream;
    const size_t size = size_of(dtype);
    if (n == 0) {
        // no rows: no gradient reaches the gains
        if (!dgain) return JARQ_OK;
        if (!usable(dgain, 4)) return JARQ_ERR_ARG;
        return finish(cudaMemsetAsync(dgain, 0, (size_t)d * sizeof(float), st));
    }
    if (!usable(H, size) || !usable(dY, size) || !usable(rstd, 4) || !usable_or_null(dH, size) || !usable_or_null(dX, size) ||
        !usable_or_null(dgain, 4) || !usable_or_null(gain, gain ? size_of(gain_dtype) : 1))
        return JARQ_ERR_ARG;
    const size_t need = dgain ? jarq_rms_norm_grad_workspace(n, d) : 0;
    if (need && (!usable(workspace, 16) || workspace_bytes < need)) return JARQ_ERR_ARG;
    if (const jarq_status late = async_failure()) return late;
    const GradArgs a{H, gain, dY, dH, dX, rstd, need ? static_cast<float *>(workspace) : nullptr, ldh, ldy, lds, ldx, n, d,
                     gain_dtype != dtype};
    const bool vec = vector(H, ldh, n, size) && vector(dY, ldy, n, size) && vector(dH, lds, n, size) &&
                     vector(dX, ldx, n, size) && vector(gain, 0, 1, 1);
    ProfScope ps("norm_grad", st);
    const cudaError_t e = with_type(dtype, [&](auto type) {
        using T = decltype(type);
        return vec ? launch_grad_t<T, true>(a, dgain, st) : launch_grad_t<T, false>(a, dgain, st);
    });
    ps.done();
    return finish(e);
}

}  // extern "C"
