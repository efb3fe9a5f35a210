"""Corners of the token scores and their gradient on the GPU: logits that differ by
more than float32 holds."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")

pytestmark = [pytest.mark.gpu,
              pytest.mark.skipif(not torch.cuda.is_available(), reason="needs a CUDA GPU")]

from test_gpu_logprob import DT, _logits, check_grad  # noqa: E402


@pytest.fixture(scope="module")
def jarq():
    from paper_2609_38599_gb300 import jarq as J
    return J


@pytest.mark.parametrize("entropy", [False, True])
@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("v", [7, 3001])
def test_gradient_where_differences_overflow(jarq, dtype, v, entropy):
    """The type's lowest value beside a large logit: their difference is below
    float32's range, the token's probability is 0 and so is its gradient."""
    low, most = float(torch.finfo(DT[dtype]).min), float(torch.finfo(DT[dtype]).max)
    x = _logits(np.random.default_rng(v), 5, v, dtype)
    x[0, 2:] = low
    x[0, :2] = 1e37
    x[1, v // 2:] = low
    x[1, 1] = 1e37
    x[2, 3] = most
    x[2, 4] = low
    x[3] = low                     # and one with nothing else, and beside -inf
    x[4, : v // 2] = low
    x[4, v // 2] = 1e37
    x[4, v // 2 + 1:] = -np.inf
    tok = np.array([[0, 1], [1, v - 1], [4, 3], [0, v - 1], [0, v // 2]])
    dx = check_grad(jarq, x, tok, 5, entropy, dtype)
    assert torch.isfinite(dx).all()
