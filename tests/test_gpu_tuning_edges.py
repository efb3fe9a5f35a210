"""Corners of the norm, the head's loss and the adapters on the GPU: more than 2^31
elements, two calls at once, tensors of another stream, the smallest calls of each form
beside the largest, and sizes on both sides of where a form is chosen."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")

pytestmark = [pytest.mark.gpu,
              pytest.mark.skipif(not torch.cuda.is_available(), reason="needs a CUDA GPU")]

import test_gpu_adapters as TA  # noqa: E402
import test_gpu_cross_entropy as TC  # noqa: E402
import test_gpu_norm as TN  # noqa: E402
from test_gpu_norm import HALF, f64, near, randn  # noqa: E402


@pytest.fixture(scope="module")
def jarq():
    from paper_2609_38599_gb300 import jarq as J
    return J


def _random(n, d, seed, dtype=torch.bfloat16, scale=1.0):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    out = torch.empty(n, d, dtype=dtype, device="cuda")
    for part in out.split(1 << 15):
        part.copy_(torch.randn(part.shape, generator=gen, device="cuda") * scale)
    return out


def test_norm_of_more_than_2_31_elements(jarq):
    n, d = 530000, 4096
    x, r = _random(n, d, 1), _random(n, d, 2)
    gain = _random(1, d, 3)[0]
    a = jarq.rms_norm(x, gain, residual=r, codes=True)
    for at in (slice(0, 200), slice(n // 2 - 100, n // 2 + 100), slice(n - 200, n)):
        b = jarq.rms_norm(x[at], gain, residual=r[at], codes=True)
        for name in ("h", "y", "codes", "scale", "rstd"):
            assert torch.equal(getattr(a, name)[at], getattr(b, name)), name
    dx, dgain = jarq.rms_norm_grad(a.h, gain, a.rstd, a.y, dh=r)
    for at in (slice(0, 200), slice(n - 200, n)):
        assert torch.equal(jarq.rms_norm_grad(a.h[at], gain, a.rstd[at], a.y[at], dh=r[at], gains=False)[0], dx[at])
    want = sum((p.double() * h.double() * s.double()[:, None]).sum(0)
               for p, h, s in zip(a.y.split(1 << 14), a.h.split(1 << 14), a.rstd.split(1 << 14)))
    size = sum((p.double() * h.double() * s.double()[:, None]).abs().sum(0)
               for p, h, s in zip(a.y.split(1 << 14), a.h.split(1 << 14), a.rstd.split(1 << 14)))
    # a block adds up n / 456 rows or fewer; two products a term and the join
    assert ((dgain.double() - want).abs() <= (n / 456 + 60) * TN.U * size).all()


def test_head_of_more_than_2_31_elements(jarq):
    n, d, vocab = 5, 4096, 530000
    W = _random(vocab, d, 4, scale=1 / 64)
    X = _random(n, d, 5)
    tok = torch.tensor([0, vocab - 1, vocab // 2, 524289, -1], device="cuda")
    loss, lse = jarq.cross_entropy(X, W, tok)
    logits = torch.cat([X.double() @ p.double().T for p in W.split(1 << 14)], 1)
    want = torch.logsumexp(logits, 1)
    bound = 1e-5 * (want.abs() + logits.abs().amax(1))            # 2^31 elements or not: as in check_loss, roughly
    assert ((lse - want).abs() <= bound).all()
    mine = logits.gather(1, tok.clamp(min=0)[:, None])[:, 0]
    assert ((loss - torch.where(tok < 0, 0.0, want - mine)).abs() <= 2 * bound).all() and loss[4] == 0
    g = torch.full((n,), 0.25, device="cuda")
    dX, dW = jarq.cross_entropy_grad(X, W, tok, lse, g)
    D = torch.exp(logits - lse.double()[:, None]) * 0.25
    D[4] = 0
    D[torch.arange(4), tok[:4]] -= 0.25
    h = HALF["bfloat16"]
    rows = torch.tensor([0, 1, 524287, 524288, 524289, vocab // 2, vocab - 2, vocab - 1], device="cuda")
    want = D[:, rows].T @ X.double()
    size = D[:, rows].T.abs() @ X.double().abs()
    assert ((dW[rows].double() - want).abs() <= 1.01 * h * (size + want.abs()) + 1e-4 * size + 1e-30).all()
    want = sum(D[:, i * 16384:(i + 1) * 16384] @ p.double() for i, p in enumerate(W.split(16384)))
    size = sum(D[:, i * 16384:(i + 1) * 16384].abs() @ p.double().abs() for i, p in enumerate(W.split(16384)))
    assert ((dX.double() - want).abs() <= 1.01 * h * (size + want.abs()) + 1e-4 * size).all()


def test_adapters_of_more_than_2_31_outputs(jarq):
    n, din, dout, r, m = 70000, 64, 32768, 16, 4
    X, base = _random(n, din, 6), _random(n, dout, 7)
    A, B = _random(m * r, din, 8, scale=0.1).view(m, r, din), _random(m * dout, r, 9, scale=0.1).view(m, dout, r)
    ids = torch.randint(-1, m, (n,), generator=torch.Generator(device="cuda").manual_seed(1), device="cuda", dtype=torch.int32)
    keep = [slice(0, 130), slice(n - 130, n)]
    before = [base[k].clone() for k in keep]
    out = jarq.apply_adapters(X, A, B, ids, base=base, out=base)
    assert out.data_ptr() == base.data_ptr()
    for k, b in zip(keep, before):
        # 16-bit sums of the same size class: the same tiles, so the same bits
        assert torch.equal(jarq.apply_adapters(X[k], A, B, ids[k].contiguous(), base=b), out[k])


@pytest.mark.parametrize("n", [64, 65])
def test_adapters_on_both_sides_of_the_choice_of_form(jarq, n):
    rng = np.random.default_rng(n)
    for rank in (8, 40, 128):
        TA.check(jarq, *TA.inputs(rng, n, 320, 300, rank, 5, "float16"))


@pytest.mark.parametrize("n", [152, 153, 304, 305])
@pytest.mark.parametrize("d", [1024, 1032, 4096, 6144, 12288, 16384, 16392])
def test_norm_on_both_sides_of_the_choice_of_form(jarq, n, d):
    rng = np.random.default_rng(n + d)
    for dtype in ("float16", "float32"):
        TN.check(jarq, randn(rng, n, d, dtype), None, residual=randn(rng, n, d, dtype))
        h, gain, rstd, dy, dh = TN._grad_inputs(rng, n, d, dtype)
        TN.check_grad(jarq, h, gain, rstd, dy, dh)
        TN.check_grad(jarq, h, gain, rstd, dy, None)


@pytest.mark.parametrize("n", [127, 128, 129, 255, 256, 257])
def test_loss_on_both_sides_of_a_tile(jarq, n):
    rng = np.random.default_rng(n)
    for d, vocab in ((64, 255), (72, 257), (128, 1100)):
        X, W, tok, g = TC.inputs(rng, n, d, vocab, "bfloat16")
        loss, lse = TC.check_loss(jarq, X, W, tok)
        TC.check_grad(jarq, X, W, tok, lse, g)


def test_a_long_sum_of_equal_signs(jarq):
    """Logits that grow over all of K, where sums that round toward zero drift most."""
    rng = np.random.default_rng(1)
    for d in (1024, 1088, 8192):
        X = torch.as_tensor(rng.uniform(0.5, 1.0, (20, d)).astype(np.float32)).bfloat16()
        W = torch.as_tensor((rng.uniform(0.5, 1.0, (300, d)) * 20 / d).astype(np.float32)).bfloat16()
        tok = torch.as_tensor(rng.integers(0, 300, 20))
        loss, lse = TC.check_loss(jarq, X, W, tok)
        logits = f64(X) @ f64(W).T
        # each of the d / 1024 sums is 64 additions that round toward zero: at most 64
        # units of its size, and on average half of half of that as it grows
        want = torch.logsumexp(torch.as_tensor(logits), 1).numpy()
        assert (np.abs(f64(lse) - want) <= 64 * 2.0 ** -23 * logits.max(1) + 1e-5).all()


def test_norms_at_once_on_two_streams(jarq):
    rng = np.random.default_rng(2)
    sets = [[randn(rng, n, 2048, "bfloat16").cuda() for _ in range(2)] for n in (900, 500)]
    want = [jarq.rms_norm(x, None, residual=r, codes=True) for x, r in sets]
    wg = [jarq.rms_norm_grad(w.h, None, w.rstd, s[0]) for w, s in zip(want, sets)]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in sets]
    for _ in range(5):
        got = []
        for s, (x, r), w in zip(streams, sets, want):
            with torch.cuda.stream(s):
                a = jarq.rms_norm(x, None, residual=r, codes=True)
                got.append((a, jarq.rms_norm_grad(a.h, None, a.rstd, x)))
        torch.cuda.synchronize()
        for (a, (dx, dgain)), w, (wx, wgain) in zip(got, want, wg):
            assert torch.equal(a.y, w.y) and torch.equal(a.codes, w.codes) and torch.equal(dx, wx) and torch.equal(dgain, wgain)


def test_adapters_at_once_and_in_graphs_that_share_memory(jarq):
    rng = np.random.default_rng(4)
    sets = [[t.cuda() for t in TA.inputs(rng, n, 512, 768, 16, 4, "bfloat16")] for n in (200, 33)]
    call = lambda s: jarq.apply_adapters(*s[:4], scale=s[4], base=s[5])
    want = [call(s) for s in sets]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in sets]
    for _ in range(5):
        got = []
        for st, s in zip(streams, sets):
            with torch.cuda.stream(st):
                got.append(call(s))
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, want))
    graphs, outs, pool = [], [], torch.cuda.graph_pool_handle()
    for s in sets:
        graph = torch.cuda.CUDAGraph()
        streams[0].wait_stream(torch.cuda.current_stream())
        with torch.cuda.graph(graph, pool=pool, stream=streams[0]):
            outs.append(call(s))
        graphs.append(graph)
    for _ in range(2):
        for graph, out, w, s in zip(graphs, outs, want, sets):
            graph.replay()
            assert torch.equal(call(s), w) and torch.equal(out, w)


def test_weights_written_just_before_on_the_same_stream(jarq):
    """Inputs that the kernel before in the stream writes are read after it has."""
    rng = np.random.default_rng(5)
    X, W, tok, g = (t.cuda() for t in TC.inputs(rng, 200, 512, 3000, "bfloat16"))
    want = jarq.cross_entropy(X, W, tok)
    x2, w2 = torch.zeros_like(X), torch.zeros_like(W)
    for _ in range(5):
        x2.zero_(), w2.zero_()
        torch.cuda.synchronize()
        w2.copy_(W)
        x2.copy_(X)
        assert torch.equal(jarq.cross_entropy(x2, w2, tok)[0], want[0])
    Xa, A, B, ids, scale, base = (t.cuda() for t in TA.inputs(rng, 20, 512, 700, 16, 3, "float16"))
    want = jarq.apply_adapters(Xa, A, B, ids, scale=scale, base=base)
    b2, y2 = torch.zeros_like(B), torch.zeros_like(base)
    for _ in range(5):
        b2.zero_(), y2.zero_()
        torch.cuda.synchronize()
        b2.copy_(B)
        y2.copy_(base)
        assert torch.equal(jarq.apply_adapters(Xa, A, b2, ids, scale=scale, base=y2), want)
