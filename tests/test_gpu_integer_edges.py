"""Corners of the integer product on the GPU: sums that cancel inside a group, and
first calls of a process."""
import os
import subprocess
import sys

import numpy as np
import pytest

torch = pytest.importorskip("torch")

pytestmark = [pytest.mark.gpu,
              pytest.mark.skipif(not torch.cuda.is_available(), reason="needs a CUDA GPU")]

from test_gpu_integer import _check, _codes, _rows  # noqa: E402

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def jarq():
    from paper_2609_38599_gb300 import jarq as J
    return J


def t(a):
    return torch.as_tensor(a).cuda()


def _cancelling(rng, n, din, dout, g):
    """Codes whose sums over 16 of K are large and cancel in every group: tokens
    repeat after 16, and a group's pieces of 16 weights add up to zero."""
    x = _codes(rng, n, 16)
    x[:, 3] = 127                           # a row's scale is 1: it is quantized to itself
    m = g // 16
    C = rng.integers(-(126 // (m - 1)), 126 // (m - 1) + 1, (dout, din // g, m, 16)).astype(np.int8)
    C[:, :, -1] = -C[:, :, :-1].sum(2)
    C = rng.permuted(C, axis=2).reshape(dout, din)
    return np.tile(x, (1, din // 16)), C


# one and two tokens by dot products, three on the tensor cores; weights' rows on
# 16-byte boundaries or not
@pytest.mark.parametrize("pad", [0, 1])
@pytest.mark.parametrize("g", [64, 128])
@pytest.mark.parametrize("n", [1, 2, 3])
@pytest.mark.parametrize("din,dout", [(128, 5), (1152, 70), (4096, 333), (11008, 130)])
def test_sums_that_cancel_inside_a_group_are_exact(jarq, n, din, dout, g, pad):
    """A group's sum is an integer and exact: zero gives zero, whatever the parts'
    size, and one code more gives what it stands for, within the bound of the
    groups' terms."""
    rng = np.random.default_rng(n * din + g)
    X, C = _cancelling(rng, n, din, dout, g)
    ws = (rng.standard_normal((dout, din // g)) * 0.01).astype(np.float32)
    xs = np.ones(n, np.float32)
    c = _rows(C, din + pad)
    assert (jarq.integer_product(t(X), t(xs), c, t(ws), g, dtype="float32") == 0).all()
    assert (jarq.integer_linear(t(X.astype(np.float32)), c, t(ws), g, dtype="float32") == 0).all()
    C[np.arange(dout), rng.integers(0, din, dout)] += 1
    c = _rows(C, din + pad)
    _check(jarq.integer_product(t(X), t(xs), c, t(ws), g, dtype="float32"), X, xs, C, ws, g, None, "float32")
    _check(jarq.integer_linear(t(X.astype(np.float32)), c, t(ws), g, dtype="float32"), X, xs, C, ws, g, None, "float32")


FIRST_CALL = """
import sys, torch
sys.path.insert(0, {root!r})
from paper_2609_38599_gb300 import jarq
gen = torch.Generator("cuda").manual_seed(0)
X = torch.randn({n}, {din}, device="cuda", generator=gen)
C = torch.randint(-15, 16, (300, {din}), device="cuda", generator=gen).to(torch.int8)
ws = torch.rand(300, {din} // 64, device="cuda", generator=gen)
torch.cuda.synchronize()
graph = torch.cuda.CUDAGraph()
with torch.cuda.graph(graph):
    y = jarq.integer_linear(X, C, ws, 64, dtype="float32")
graph.replay()
torch.cuda.synchronize()
assert torch.equal(y, jarq.integer_linear(X, C, ws, 64, dtype="float32"))
"""


# a single token quantized by the product's own blocks, one with a launch for it, two
@pytest.mark.parametrize("n,din", [(1, 4096), (1, 6272), (2, 1024)])
def test_a_first_call_of_one_or_two_tokens_can_be_captured(n, din):
    """Such a call has no wait to report, and so nothing to allocate for it."""
    r = subprocess.run([sys.executable, "-c", FIRST_CALL.format(root=ROOT, n=n, din=din)], capture_output=True, text=True,
                       timeout=300)
    assert r.returncode == 0, r.stderr[-2000:]
