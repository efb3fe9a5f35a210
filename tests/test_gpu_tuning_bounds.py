"""What the norm, the head's loss and the adapters promise at the ends of their ranges on
the GPU: rows whose squares leave float32's range, losses of certain tokens, long sums,
small weights, adapters' terms that cancel or leave the range."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")

pytestmark = [pytest.mark.gpu,
              pytest.mark.skipif(not torch.cuda.is_available(), reason="needs a CUDA GPU")]

import test_gpu_norm as TN  # noqa: E402
from test_gpu_norm import randn  # noqa: E402


@pytest.fixture(scope="module")
def jarq():
    from paper_2609_38599_gb300 import jarq as J
    return J


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("size", [1e-20, 1e20, 1e24, 1e36])
@pytest.mark.parametrize("n,d", [(3, 1000), (200, 1000), (5, 999), (160, 999), (2, 17000), (160, 17000)])
def test_gradient_of_rows_whose_squares_leave_the_range(jarq, dtype, size, n, d):
    """Rows that the norm itself takes: neither the square of 1 / rms nor the products of
    rows and gradients, before the row's own factor, fit float32."""
    rng = np.random.default_rng(n + d)
    h = randn(rng, n, d, dtype, size)
    gain, dy, dh = randn(rng, 1, d, dtype)[0], randn(rng, n, d, dtype, 100.0), randn(rng, n, d, dtype, 1 / size)
    rstd = jarq.rms_norm(h.cuda(), eps=1e-45).rstd.cpu()
    TN.check_grad(jarq, h, gain, rstd, dy, dh)
    TN.check_grad(jarq, h, gain.float(), rstd, dy, None)
    # one row in plain numbers: entries of 1 and -1/2 times a size, a gradient of ones
    row = torch.full((n, d), -0.5)
    row[:, ::2] = 1.0
    h = (row * size).to(h.dtype)
    TN.check_grad(jarq, h, None, jarq.rms_norm(h.cuda(), eps=1e-45).rstd.cpu(), torch.ones_like(h), None)
