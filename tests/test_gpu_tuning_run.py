"""The end of a model as it is tuned: the final norm with the residual, the head's loss
and the way back through both, against automatic differentiation in float64."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")

pytestmark = [pytest.mark.gpu,
              pytest.mark.skipif(not torch.cuda.is_available(), reason="needs a CUDA GPU")]

from test_gpu_cross_entropy import sum_error  # noqa: E402
from test_gpu_norm import HALF, U, f64, near, randn  # noqa: E402


@pytest.fixture(scope="module")
def jarq():
    from paper_2609_38599_gb300 import jarq as J
    return J


def step(jarq, x, res, gain, W, tok, g):
    r = jarq.rms_norm(x, gain, eps=1e-5, residual=res)
    loss, lse = jarq.cross_entropy(r.y, W, tok)
    dy, dW = jarq.cross_entropy_grad(r.y, W, tok, lse, g)
    dx, dgain = jarq.rms_norm_grad(r.h, gain, r.rstd, dy)
    return r, loss, dy, dW, dx, dgain


@pytest.mark.parametrize("dtype", ["float16", "bfloat16"])
@pytest.mark.parametrize("n,d,vocab", [(1, 64, 300), (37, 256, 1000), (300, 1000, 2001)])
def test_norm_loss_and_back(jarq, dtype, n, d, vocab):
    rng = np.random.default_rng(n)
    x, res, gain = randn(rng, n, d, dtype), randn(rng, n, d, dtype), (1 + 0.2 * randn(rng, 1, d, "float32")[0]).to(randn(rng, 1, 1, dtype).dtype)
    W = randn(rng, vocab, d, dtype, 2.0 / d ** 0.5)
    tok = torch.as_tensor(rng.integers(0, vocab, n))
    if n > 1:
        tok[1] = -1
    g = torch.full((n,), 1.0 / n)
    r, loss, dy, dW, dx, dgain = step(jarq, *(t.cuda() for t in (x, res, gain, W, tok, g)))

    h = (x.float() + res.float()).to(x.dtype).double().requires_grad_()
    wg, ww = gain.double().requires_grad_(), W.double().requires_grad_()
    y = h * torch.rsqrt((h * h).mean(1, keepdim=True) + 1e-5) * wg
    y.retain_grad()
    counts = tok >= 0
    total = (torch.nn.functional.cross_entropy((y @ ww.T)[counts], tok[counts], reduction="none") * g.double()[counts]).sum()
    total.backward()
    # y is rounded before the product: the logits are off by half a step of each y, and
    # the probabilities relatively by as much
    u = HALF[dtype]
    dl = 1.01 * u * (np.abs(f64(y)) @ np.abs(f64(W)).T).max(1) + sum_error(d) * (np.abs(f64(y)) @ np.abs(f64(W)).T).max(1) + 100 * U
    want = torch.where(counts, torch.logsumexp(y @ ww.T, 1) - (y @ ww.T).gather(1, tok.clamp(min=0)[:, None])[:, 0], 0.0)
    near(loss, f64(want), 2 * dl * 1.01 + 4 * U * np.abs(f64(want)) + 1e-6)
    p = f64(torch.softmax(y @ ww.T, 1)) * (f64(g) * f64(counts.double()))[:, None]
    D = p.copy()
    D[np.flatnonzero(f64(counts.double())), f64(tok[counts]).astype(int)] -= f64(g)[f64(counts.double()) > 0]
    errD = p * (2.02 * dl)[:, None] + np.abs(D) * 1.01 * u + (2.0 ** -38 / n if dtype == "float16" else 0)
    tiny = float(torch.finfo(x.dtype).tiny) * u
    err_y = errD @ np.abs(f64(W)) + sum_error(vocab) * 2 * (np.abs(D) @ np.abs(f64(W)))
    near(dy, f64(y.grad), 1.01 * (err_y + u * np.abs(f64(y.grad))) + tiny)
    err_w = errD.T @ np.abs(f64(y)) + np.abs(D).T @ (np.abs(f64(y)) * u) * 1.01 + sum_error(n) * 2 * (np.abs(D).T @ np.abs(f64(y)))
    near(dW, f64(ww.grad), 1.01 * (err_w + u * np.abs(f64(ww.grad))) + tiny)
    # the norm's way back is linear in dy: its error passes through the same formula, in
    # magnitudes; what the norm's own float32 adds is far below dy's rounding
    e = 1.01 * (err_y + u * np.abs(f64(y.grad))) + tiny
    hh, rs, gg = np.abs(f64(h)), f64(r.rstd)[:, None], np.abs(f64(gain))
    back = rs * (e * gg + hh * rs ** 2 * (e * gg * hh).mean(1, keepdims=True))
    size = rs * (np.abs(f64(y.grad)) * gg + hh * rs ** 2 * (np.abs(f64(y.grad)) * gg * hh).mean(1, keepdims=True))
    near(dx, f64(h.grad), 1.02 * back + 200 * U * size + 1.01 * u * np.abs(f64(h.grad)) + tiny)
    near(dgain, f64(wg.grad), 1.02 * (e * hh * rs).sum(0) + 200 * U * (np.abs(f64(y.grad)) * hh * rs).sum(0) + 1e-30)
    assert jarq.async_status() == jarq.JARQ_OK


def test_step_in_a_graph_between_eager_steps(jarq):
    """A captured step, replayed with other inputs, beside eager ones on another stream."""
    rng = np.random.default_rng(3)
    n, d, vocab = 120, 512, 3000
    make = lambda s: [t.cuda() for t in (randn(np.random.default_rng(s), n, d, "bfloat16"), randn(np.random.default_rng(s + 50), n, d, "bfloat16"))]
    x, res = make(1)
    gain, W = randn(rng, 1, d, "bfloat16")[0].cuda(), randn(rng, vocab, d, "bfloat16", 0.08).cuda()
    tok = torch.as_tensor(rng.integers(0, vocab, n)).cuda()
    g = torch.full((n,), 1.0 / n, device="cuda")
    step(jarq, x, res, gain, W, tok, g)
    stream, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.graph(graph, stream=stream):
        got = step(jarq, x, res, gain, W, tok, g)
    for s in (2, 3):
        a, b = make(s)
        x.copy_(a)
        res.copy_(b)
        want = step(jarq, a, b, gain, W, tok, g)
        graph.replay()
        again = step(jarq, a, b, gain, W, tok, g)
        torch.cuda.synchronize()
        for w, v, u in zip(want[1:], got[1:], again[1:]):
            assert torch.equal(w, v) and torch.equal(w, u)
