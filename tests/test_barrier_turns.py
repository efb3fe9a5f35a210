"""The order in which the integer product's drain waits for sums, on the CPU: its
own arithmetic (``csrc/turns.cuh``), compiled for the host, against the count of
each barrier's completions.  A wait by parity is sound if it names the completion
that the sums' own barrier reports and the waiting warp has seen the one before."""
import os
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

HARNESS = r"""
#define __device__
#define __forceinline__ inline
#include "turns.cuh"
#include <cstdio>
#include <cstdlib>

// Units' waits that are not sound, of warps that read parts first .. last of every
// unit in `units` units: a completion not seen before, or a parity of another one.
template <int N, int PARTS, bool APART>
int unsound(int first, int last, int units) {
    using T = jarq::Turn<N, PARTS, APART>;
    T issuer(1), reader(0);
    int done[64] = {}, seen[64] = {}, bad = 0;
    for (int u = 0; u < units; ++u, issuer.next(), reader.next()) {
        int report[PARTS];
        for (int h = 0; h < PARTS; ++h) {               // the issuer's commits
            report[h] = issuer.report(h);
            if (report[h] < 0 || report[h] >= T::kReports || issuer.acc(h) < 0 || issuer.acc(h) >= N) return -1;
            ++done[report[h]];
            for (int o = 0; o < h; ++o)                 // parts of a unit do not share an accumulator
                if (issuer.acc(o) == issuer.acc(h)) return -1;
        }
        for (int h = first; h <= last; ++h) {           // a warp's waits
            const int b = reader.report(h), c = done[b] - 1;
            bad += b != report[h] || reader.acc(h) != issuer.acc(h) || seen[b] != c || reader.report_parity(h) != (uint32_t)(c & 1);
            seen[b] = c + 1;
        }
    }
    return bad;
}

int main() {
    printf("%d %d %d ", unsound<2, 1, false>(0, 0, 50), unsound<2, 2, false>(0, 1, 50), unsound<3, 2, false>(0, 1, 50));
    printf("%d %d ", unsound<3, 2, true>(0, 0, 50), unsound<3, 2, true>(1, 1, 50));
    printf("%d %d\n", unsound<3, 2, false>(0, 0, 50), unsound<3, 2, false>(1, 1, 50));
}
"""


@pytest.fixture(scope="module")
def counts(tmp_path_factory):
    d = tmp_path_factory.mktemp("turns")
    (d / "turns.cpp").write_text(HARNESS)
    subprocess.run(["g++", "-std=c++17", "-I", os.path.join(ROOT, "paper_2609_38599_gb300", "csrc"), str(d / "turns.cpp"),
                    "-o", str(d / "turns")], check=True)
    return [int(x) for x in subprocess.run([str(d / "turns")], check=True, capture_output=True, text=True).stdout.split()]


def test_every_wait_for_sums_follows_the_completion_before_it(counts):
    """Warps that read every part, and warps that read one with barriers of its own."""
    assert counts[:5] == [0] * 5


def test_shared_barriers_are_unsound_for_readers_of_one_part(counts):
    """What the check above sees: one barrier an accumulator, read by warps that
    take one part of each unit, as tiles of 256 tokens with groups of 64 have them."""
    assert all(c > 0 for c in counts[5:])
