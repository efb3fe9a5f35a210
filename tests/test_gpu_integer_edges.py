"""Corners of the integer product on the GPU: sums that cancel inside a group."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")

pytestmark = [pytest.mark.gpu,
              pytest.mark.skipif(not torch.cuda.is_available(), reason="needs a CUDA GPU")]

from test_gpu_integer import _check, _codes, _rows  # noqa: E402


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
