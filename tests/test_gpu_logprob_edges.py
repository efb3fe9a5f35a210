"""Corners of the token scores and their gradient on the GPU: logits that differ by
more than float32 holds, and rows with all mass on one token."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")

pytestmark = [pytest.mark.gpu,
              pytest.mark.skipif(not torch.cuda.is_available(), reason="needs a CUDA GPU")]

from test_gpu_logprob import DT, _logits, check, check_grad  # noqa: E402


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


@pytest.mark.parametrize("dtype", list(DT))
@pytest.mark.parametrize("v", [1, 33, 5000, 70001])
def test_probabilities_are_at_most_one(jarq, dtype, v):
    """One token with all the mass, by a mask or far above the rest, at maxima of
    many sizes and last places; then rows as they come: no log probability is
    above 0, no entropy below, and lse not below the largest logit."""
    rng = np.random.default_rng(v)
    n = 96
    top = torch.as_tensor((rng.standard_normal(n) * np.exp(rng.uniform(-5, 5, n))).astype(np.float32)).to(DT[dtype])
    at = rng.integers(0, v, n)
    x = torch.full((n, v), -np.inf).to(DT[dtype])
    x[n // 2:] = (top[n // 2:].float() - 400.0)[:, None].to(DT[dtype])
    x[torch.arange(n), torch.as_tensor(at)] = top
    x = torch.cat([x, _logits(rng, 8, v, dtype, 0.1), _logits(rng, 8, v, dtype, 30.0)])
    tok = np.concatenate([at, x[n:].float().argmax(1).numpy()])
    r, ref = check(jarq, x, tok, min(v, 3))
    assert (r.logprob <= 0).all() and (r.entropy >= 0).all() and (r.top_logprob <= 0).all()
    assert (r.lse >= x.float().max(1).values.cuda()).all()
