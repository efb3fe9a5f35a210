// Which stage or accumulator a role of a kernel comes to next, and the parity of
// the barrier that it waits for.  A wait by parity says that a completion of that
// parity is the barrier's last: whoever waits must have seen, or know of, every
// completion before the one that it waits for, and the next one must not come
// before it has looked.  Plain arithmetic, also compiled for the host by its test.
#pragma once

#include <stdint.h>

namespace jarq {

// A position in a ring of N stages.
template <int N>
struct Slot {
    int s = 0;
    uint32_t phase;
    __device__ explicit Slot(uint32_t first) : phase(first) {}
    __device__ __forceinline__ void next() {
        if (++s == N) {
            s = 0;
            phase ^= 1;
        }
    }
};

// The accumulators of a unit's PARTS parts, N taking turns: which one a part has,
// and the parity to wait for of a barrier that completes once a use of it.  APART:
// readers wait for one part's sums alone.  An accumulator comes back with another
// part then, whose completions such a reader neither sees nor knows of, so the sums
// are reported on barriers of an accumulator and part, which complete only for
// that reader (each once in N units).
template <int N, int PARTS, bool APART = false>
struct Turn {
    static_assert(!APART || N % PARTS != 0, "else a part keeps its accumulators");
    static constexpr int kReports = APART ? N * PARTS : N;      // barriers that report sums
    int first = 0;
    uint32_t phase;
    Slot<N> own;
    __device__ explicit Turn(uint32_t p) : phase(p), own(p) {}
    __device__ __forceinline__ int acc(int part) const { return first + part < N ? first + part : first + part - N; }
    __device__ __forceinline__ uint32_t parity(int part) const { return first + part < N ? phase : phase ^ 1; }
    // the barrier that reports this part's sums, and its parity
    __device__ __forceinline__ int report(int part) const { return (APART ? part * N : 0) + acc(part); }
    __device__ __forceinline__ uint32_t report_parity(int part) const { return APART ? own.phase : parity(part); }
    __device__ __forceinline__ void next() {
        first += PARTS;
        if (first >= N) {
            first -= N;
            phase ^= 1;
        }
        if (APART) own.next();
    }
};

}  // namespace jarq
