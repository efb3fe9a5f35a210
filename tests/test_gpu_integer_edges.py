"""Corners of the integer product on the GPU: sums that cancel inside a group, the
largest sums and rows without a scale in the linear layer, its order with the work
before and beside it, and first calls of a process."""
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


# every tile of the linear layer (dot products, 32 to 256 tokens), weights' rows on
# 16-byte boundaries or not
@pytest.mark.parametrize("pad", [0, 1])
@pytest.mark.parametrize("n", [1, 2, 20, 60, 100, 600])
@pytest.mark.parametrize("a,b", [(-127, -128), (127, -128), (127, 127)])
def test_largest_sums_of_the_linear_layer_are_exact(jarq, n, a, b, pad):
    """Codes of the largest magnitude over the longest rows, from activations that
    quantize to themselves: the exact integer, rounded to float32 once."""
    din, dout = 65536, 300
    X = torch.full((n, din), float(a), device="cuda")
    C = _rows(np.full((dout, din), b, np.int8), din + 16 * pad + pad)
    X[:, 5] = 1
    C[:, 7] = 3
    want = a * b * (din - 2) + b + 3 * a
    y = jarq.integer_linear(X, C, torch.ones(dout, device="cuda"), dtype="float32")
    assert (y == torch.tensor(float(np.float32(want)), device="cuda")).all()


@pytest.mark.parametrize("xdtype", ["float32", "float16", "bfloat16"])
@pytest.mark.parametrize("g", [0, 64, 128])
@pytest.mark.parametrize("n", [3, 20, 60, 100, 300, 700])
def test_batches_with_rows_that_have_no_scale(jarq, xdtype, n, g):
    """A NaN or an infinity in a token makes its outputs NaN and a token of zeros
    gives the bias; the other tokens' outputs are what they are without those."""
    din, dout = 640, 517
    rng = np.random.default_rng(n + g)
    X = t(rng.standard_normal((n, din)).astype(np.float32)).to(getattr(torch, xdtype))
    C, ws = t(_codes(rng, dout, din, 15)), t(rng.standard_normal((dout, din // g if g else 1)).astype(np.float32))
    bias = t(rng.standard_normal(dout).astype(np.float32))
    plain = jarq.integer_linear(X, C, ws, g, bias, "float32")
    X[0, 17] = float("nan")
    X[n // 2, din - 1] = float("inf") if n % 2 else -float("inf")
    X[n - 1] = 0
    y = jarq.integer_linear(X, C, ws, g, bias, "float32")
    assert torch.isnan(y[0]).all() and torch.isnan(y[n // 2]).all() and torch.equal(y[n - 1], bias)
    rest = [r for r in range(n) if r not in (0, n // 2, n - 1)]
    assert torch.equal(y[rest], plain[rest]) and torch.isfinite(plain).all()


@pytest.mark.parametrize("n,din,dout,g", [(1, 4096, 3000, 128), (1, 8192, 1500, 0), (2, 4096, 3000, 64), (40, 4096, 2000, 128),
                                          (300, 2048, 2000, 0), (600, 2048, 1500, 64)])
def test_weights_written_just_before(jarq, n, din, dout, g):
    """Codes, scales and bias are the results of the work just before on the stream:
    the product, which starts under the quantization, must not read older ones."""
    rng = np.random.default_rng(din + n)
    X = t(rng.standard_normal((n, din)).astype(np.float32)).half()
    G = din // g if g else 1
    layers = [(t(_codes(rng, dout, din, 15)), t(rng.standard_normal((dout, G)).astype(np.float32)),
               t(rng.standard_normal(dout).astype(np.float32))) for _ in range(2)]
    want = [jarq.integer_linear(X, *(l[:2]), g, l[2], "float32") for l in layers]
    C, ws, bias = (torch.zeros_like(a) for a in layers[0])
    got = []
    for i in range(20):
        for to, new in zip((bias, ws, C), reversed(layers[i % 2])):
            to.copy_(new)
        got.append(jarq.integer_linear(X, C, ws, g, bias, "float32"))
    assert all(torch.equal(y, want[i % 2]) for i, y in enumerate(got))


def test_two_streams_at_once(jarq):
    """Products of every form beside one another on two streams."""
    rng = np.random.default_rng(9)
    work = []
    for n, din, dout, g in ((1, 4096, 3000, 128), (2, 1024, 900, 0), (24, 4096, 2000, 128), (60, 1001, 700, 0), (300, 2048, 2000, 64),
                            (900, 1024, 3000, 0)):
        X = t(rng.standard_normal((n, din)).astype(np.float32)).half()
        C, ws = t(_codes(rng, dout, din, 15)), t(rng.standard_normal((dout, din // g if g else 1)).astype(np.float32))
        work.append((X, C, ws, g))
    want = [jarq.integer_linear(*w, dtype="float32") for w in work]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    got = [[], []]
    for _ in range(10):
        for s, stream in enumerate(streams):
            with torch.cuda.stream(stream):
                for i in (range(len(work)) if s else reversed(range(len(work)))):
                    got[s].append((i, jarq.integer_linear(*work[i], dtype="float32")))
    torch.cuda.synchronize()
    assert all(torch.equal(y, want[i]) for half in got for i, y in half)
    assert jarq.async_status() == jarq.JARQ_OK
