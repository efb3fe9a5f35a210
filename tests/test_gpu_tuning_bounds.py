"""What the norm, the head's loss and the adapters promise at the ends of their ranges on
the GPU: rows whose squares leave float32's range, losses of certain tokens, long sums,
small weights, adapters' terms that cancel or leave the range."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")

pytestmark = [pytest.mark.gpu,
              pytest.mark.skipif(not torch.cuda.is_available(), reason="needs a CUDA GPU")]

import test_gpu_adapters as TA  # noqa: E402
import test_gpu_cross_entropy as TC  # noqa: E402
import test_gpu_norm as TN  # noqa: E402
from oracle import jarq_tuning as O  # noqa: E402
from test_gpu_norm import HALF, U, f64, near, randn  # noqa: E402


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


@pytest.mark.parametrize("n,d", [(3, 1000), (200, 4096), (5, 999), (2, 40000)])
@pytest.mark.parametrize("size,eps", [(3e18, 1e37), (3e18, 3e38), (1e19, 1e38), (1e-3, 3.4e38), (3e-21, 1e-41), (1e-22, 1e-44),
                                      (1e-20, 1e-45), (0.0, 1e-45)])
def test_eps_of_any_size_counts(jarq, n, d, size, eps):
    """Sums of squares above and below float32's numbers, beside an eps of their own size."""
    eps = float(np.float32(eps))
    rng = np.random.default_rng(d)
    for dtype in ("float32", "bfloat16"):
        r, ref = TN.check(jarq, randn(rng, n, d, dtype, size), None, eps=eps)
        assert r.rstd.isfinite().all() and (r.rstd > 0).all()


def _sure_rows(dtype):
    """Rows whose largest logit, of many sizes, is all of their mass, and its token."""
    top = torch.arange(1, 2048) / 32.0
    whole = top.floor()
    X = torch.zeros(len(top), 64)
    X[:, 0], X[:, 1], X[:, 2] = whole, top - whole, 1.0
    W = torch.zeros(40, 64)
    W[:, 2] = -200.0
    W[7, :3] = torch.tensor([1.0, 1.0, 0.0])
    t = TN.DT[dtype]
    return X.to(t), W.to(t), torch.full((len(top),), 7), top


@pytest.mark.parametrize("dtype", TC.TYPES)
def test_a_sure_row_has_no_loss_below_0(jarq, dtype):
    X, W, tok, top = _sure_rows(dtype)
    for w, t in ((W, tok), (W[7:8], tok - 7)):
        loss, lse = jarq.cross_entropy(X.cuda(), w.cuda(), t.cuda())
        # the sum is 1 but for two exponentials of 2^-22 each and the roundings of two
        # products, an addition and the logarithm
        top64 = top.double().cuda()
        assert (loss >= 0).all() and (loss <= 12 * U).all()
        assert (lse >= top.cuda()).all() and (lse.double() - top64 <= 12 * U + U * top64).all()


@pytest.mark.parametrize("dtype", TC.TYPES)
@pytest.mark.parametrize("rival", [0.82, 0.7])
@pytest.mark.parametrize("n,d,vocab", [(40, 1024, 300), (60, 4096, 300), (300, 8192, 700), (3, 8200, 300)])
def test_gradient_of_a_sure_token_is_that_of_its_loss(jarq, dtype, n, d, vocab, rival):
    """Logits of one sign over a long K, and a token that has all but 1e-4 to 1e-2 of the
    mass: its entry of D is -(1 - exp(-loss)), so the gradient's logits have to be as good
    as the loss's own."""
    rng = np.random.default_rng(d)
    X = torch.as_tensor(rng.uniform(0.5, 1.0, (n, d)).astype(np.float32)).to(TN.DT[dtype])
    W = torch.zeros(vocab, d, dtype=X.dtype)
    W[0] = torch.as_tensor((rng.uniform(0.5, 1.0, d) * 50 / d).astype(np.float32)).to(X.dtype)
    W[1] = (W[0].float() * rival).to(X.dtype)
    g = torch.full((n,), 64.0)
    for r in {0, n // 2, n - 1}:
        # the only row that counts: the token's row of dW is its entry of D times this row of X
        tok = torch.full((n,), -1)
        tok[r] = 0
        x, w, t = X.cuda(), W.cuda(), tok.cuda()
        loss, lse = jarq.cross_entropy(x, w, t)
        dW = jarq.cross_entropy_grad(x, w, t, lse, g.cuda(), hidden=False)[1]
        entry = -np.expm1(-f64(loss)[r])
        assert 3e-5 < entry < 2e-2
        # lse rounded once; the loss's sum and D's exponential, 2^-22 each with their factors
        # and products
        err = U * abs(f64(lse)[r]) + 16 * U
        got = -f64(dW[0]) / (64.0 * f64(X[r]))
        assert (np.abs(got - entry) <= 1.01 * (err + HALF[dtype] * entry)).all(), (np.abs(got - entry).max(), entry)


# The tensor cores' additions round toward zero, so a sum of one sign that grows in an
# accumulator loses a part of itself that grows with the number of its terms.  Over 4096 of K,
# what one accumulator may hold, that part is measured; longer sums are made up of such ones
# by float32 additions to nearest, and lose no larger a part of themselves.  What is added
# for: a dozen roundings of an exponential, its factors and the row's lse, as if all had the
# same sign, and six deviations of a mean of so many uniform errors of half a step of float16.
def _noise(count):
    return 6 * HALF["float16"] / (3 * count) ** 0.5 + 12 * U


def _drift_of_rows(jarq, n):
    """Mean part that entries of dW of n rows, all of one sign, are off by, and its noise."""
    d, vocab = 1280, 4096
    gen = torch.Generator(device="cuda").manual_seed(1)
    X = (0.5 + 0.5 * torch.rand(1 << 17, d, generator=gen, device="cuda")).half()[:n]
    W = (torch.randn(vocab, d, generator=gen, device="cuda") * 0.01).half()
    tok = torch.randint(0, 64, (1 << 17,), generator=gen, device="cuda")[:n]
    loss, lse = jarq.cross_entropy(X, W, tok)
    dW = jarq.cross_entropy_grad(X, W, tok, lse, torch.ones(n, device="cuda"), hidden=False)[1]
    want = torch.zeros(vocab, d, dtype=torch.float64, device="cuda")
    for a, s in zip(X.split(1 << 14), lse.split(1 << 14)):
        want += torch.exp(a.double() @ W.double().T - s.double()[:, None]).T @ a.double()
    # rows that are no row's token
    return abs(((dW[64:].double() - want[64:]) / want[64:]).mean().item()), _noise(dW[64:].numel())


def test_sums_over_many_rows_do_not_drift(jarq):
    """dW over 2^17 rows."""
    part, noise = _drift_of_rows(jarq, 4096)
    drift, more = _drift_of_rows(jarq, 1 << 17)
    assert drift <= part + noise + more


def test_sums_over_a_large_vocabulary_do_not_drift(jarq):
    """dX over 2^17 tokens of a head of one sign."""
    n, d, vocab = 2048, 1280, 1 << 17
    gen = torch.Generator(device="cuda").manual_seed(2)
    X = (torch.randn(n, d, generator=gen, device="cuda") * 0.2 / d ** 0.5).half()
    W = (0.5 + 0.5 * torch.rand(vocab, d, generator=gen, device="cuda")).half()
    tok = torch.randint(0, vocab, (n,), generator=gen, device="cuda")
    loss, lse = jarq.cross_entropy(X, W, tok)
    dX = jarq.cross_entropy_grad(X, W, tok, lse, torch.ones(n, device="cuda"), head=False)[0]
    size = torch.zeros(n, d, dtype=torch.float64, device="cuda")
    for w in W.split(1 << 14):
        size += torch.exp(X.double() @ w.double().T - lse.double()[:, None]) @ w.double()
    drift = abs(((dX.double() - (size - W[tok].double())) / size).mean().item())
    # The part is measured on sums of one sign (a row of D is of both: of 4096 tokens its own
    # entry would turn the sum's sign).  An addition loses units of the sum so far: 2^-23 to 2^-24
    # of it, by where in a power of two it lies, and so up to twice what other sums lose.
    part, noise = _drift_of_rows(jarq, 4096)
    assert drift <= 2 * part + 2 * noise + _noise(dX.numel())


@pytest.mark.parametrize("dtype", TA.TYPES)
@pytest.mark.parametrize("n", [40, 65, 300])
@pytest.mark.parametrize("din,dout,rank", [(8, 64, 8), (12, 33, 16), (40, 300, 64)])
def test_adapters_terms_that_cancel(jarq, dtype, n, din, dout, rank):
    """Terms of B (A x) that cancel all but 2^-14 of themselves: the sums A x are kept to
    2^-22 of a token's largest, for outputs of the inputs' own type too, whatever the form."""
    rng = np.random.default_rng(n + din)
    t = TN.DT[dtype]
    X = torch.as_tensor(rng.integers(4, 8, (n, din)) / 8.0).to(t)
    # multiples of 2^-21 below 8: sums A x that any order of float32 additions has exactly
    A = torch.zeros(3, rank, din, dtype=torch.float64)
    A[:, ::2, :8] = torch.as_tensor(rng.integers(4, 8, (3, rank // 2, 8)) / 8.0)
    A[:, 1::2] = A[:, ::2]
    A[:, :, 3] = torch.as_tensor(rng.integers(64, 128, (3, rank)) * 2.0 ** -18)
    A = A.to(t)
    # pairs of rows that differ in that column alone, with opposite powers of two
    B = torch.as_tensor(2.0 ** rng.integers(-1, 1, (3, dout, rank))).to(t)
    B[:, :, 1::2] = -B[:, :, ::2]
    ids = torch.as_tensor(rng.integers(0, 3, n).astype(np.int32))
    got = jarq.apply_adapters(*(v.cuda() for v in (X, A, B, ids)))
    x, a, b, i = f64(X), f64(A), f64(B), ids.numpy()
    want = O.apply_adapters(x, a, b, i)
    # what is kept of the sums, and an addition a term
    err = [np.abs(a[k] @ row).max() * (np.abs(b[k]).sum(1) * 2.0 ** -22 + rank * U) for k, row in zip(i, x)]
    near(got, want, 1.01 * (np.array(err) + HALF[dtype] * np.abs(want)) + float(torch.finfo(t).tiny) * HALF[dtype])


@pytest.mark.parametrize("dtype", TA.TYPES)
@pytest.mark.parametrize("n", [5, 65, 200])
@pytest.mark.parametrize("scale", [1e-36, 1e-30, 1e28, 1e32, 1e35])
def test_adapters_scales_of_any_size(jarq, dtype, n, scale):
    """float32 outputs of scaled sums beyond 2^100 and below 2^-100."""
    rng = np.random.default_rng(n)
    X, A, B, ids, s, base = TA.inputs(rng, n, 200, 96, 24, 3, dtype, "float32")
    TA.check(jarq, X, A, B, ids, s * scale, base * scale)


@pytest.mark.parametrize("dtype", TA.TYPES)
def test_adapters_infinite_sums_are_the_same_in_both_forms(jarq, dtype):
    """An infinity in a token: its outputs are infinite, or NaN where terms of both signs
    meet, whatever the number of tokens."""
    rng = np.random.default_rng(1)
    X, A, B, ids, s, base = TA.inputs(rng, 80, 64, 40, 16, 3, dtype)
    X[5, 3], X[60, 9] = float("inf"), -float("inf")
    ids[5], ids[60] = 1, 2
    A[1, :, 3], A[2, :, 9] = A[1, :, 3].abs() + 0.01, A[2, :, 9].abs() + 0.01
    B[1, :20], B[2, 10:] = B[1, :20].abs() + 0.01, -B[2, 10:].abs() - 0.01
    many = jarq.apply_adapters(*(t.cuda() for t in (X, A, B, ids)), scale=s.cuda(), base=base.cuda())
    few = torch.cat([jarq.apply_adapters(X[k].cuda(), A.cuda(), B.cuda(), ids[k].contiguous().cuda(), scale=s.cuda(), base=base[k].cuda())
                     for k in (slice(0, 40), slice(40, 80))])
    assert (few[5, :20] == float("inf")).all() and (few[60, 10:] == float("inf")).all()
    for f in (torch.isnan, torch.isposinf, torch.isneginf):
        assert torch.equal(f(many), f(few))


@pytest.mark.parametrize("n,d,vocab,pitch", [(100, 128, 300, 128), (1000, 72, 500, 72), (100, 77, 300, 80)])
@pytest.mark.parametrize("size,spread", [(1.0, 14), (0.05, 12), (2.0 ** -9, 10), (30.0, 14), (0.05, 0)])
def test_float16_head_gradient_of_small_states_and_weights(jarq, n, d, vocab, pitch, size, spread):
    """Rows of small weight that alone have their token, of hidden states of any size: their
    share of dW keeps all its bits beside rows of large weight."""
    rng = np.random.default_rng(n)
    X, W = randn(rng, n, d, "float16", size), randn(rng, vocab, d, "float16", 1 / (size * d ** 0.5))
    X[:, ::7] = (X[:, ::7].float() * 2.0 ** -3).half()
    tok = torch.as_tensor(rng.permutation(vocab)[np.arange(n) % vocab])
    tok[3] = -1
    g = 2.0 ** -rng.uniform(0, spread, n)
    g[::9] = 2.0 ** -spread
    # up to where float16 holds the largest of the results, and the smallest are normal numbers
    g = torch.as_tensor((g * 2.0 ** (12 - np.ceil(np.log2(size)))).astype(np.float32))
    x, w, t = TN.device(X, pitch), W.cuda(), tok.cuda()
    loss, lse = jarq.cross_entropy(x, w, t)
    # (dX of the same weights would leave float16's range)
    dW = TC.check_grad(jarq, X, W, tok, lse, g, (x, w, t, lse, g.cuda()), hidden=False)[1]
    again = jarq.cross_entropy_grad(x, w, t, lse, g.cuda(), hidden=False)[1]
    assert torch.equal(again, dW)


def test_float16_head_gradient_of_states_that_are_zero_or_not_finite(jarq):
    rng = np.random.default_rng(1)
    X, W, tok, g = TC.inputs(rng, 70, 64, 300, "float16", ignored=False)
    for rows in (slice(0, 70), slice(0, 0)):
        Y = X.clone()
        Y[rows] = 0
        Y[5] = 65504.0 if rows.stop == 0 else 0
        loss, lse = jarq.cross_entropy(Y.cuda(), W.cuda(), tok.cuda())
        TC.check_grad(jarq, Y, W, tok, lse, g)
    X[9], tok[9] = float("inf"), -1
    X[11], g[11] = float("nan"), 0.0
    tok[11] = -1
    loss, lse = jarq.cross_entropy(X.cuda(), W.cuda(), tok.cuda())
    lse[[9, 11]] = 0
    Y = X.clone()
    Y[[9, 11]] = 0
    TC.check_grad(jarq, Y, W, tok, lse, g, (X.cuda(), W.cuda(), tok.cuda(), lse, g.cuda()))


@pytest.mark.parametrize("dtype", TC.TYPES)
@pytest.mark.parametrize("n,d,vocab", [(8200, 1280, 4096), (2048, 1278, 16390), (4100, 2056, 4100), (200, 1100, 60001)])
def test_sums_of_several_accumulators(jarq, dtype, n, d, vocab):
    """Every entry of both gradients where sums take more than one accumulator: with and
    without splits, tiles of any width, edges of rows and columns."""
    gen = torch.Generator(device="cuda").manual_seed(n)
    t = TN.DT[dtype]
    X = torch.randn(n, d, generator=gen, device="cuda").to(t)
    W = (torch.randn(vocab, d, generator=gen, device="cuda") * 2 / d ** 0.5).to(t)
    tok = torch.randint(-1, vocab, (n,), generator=gen, device="cuda")
    g = 0.5 + torch.rand(n, generator=gen, device="cuda")
    loss, lse = jarq.cross_entropy(X, W, tok)
    dX, dW = jarq.cross_entropy_grad(X, W, tok, lse, g)
    x, w = X.double(), W.double()
    D = torch.exp(x @ w.T - lse.double()[:, None])
    live = (tok >= 0).nonzero()[:, 0]
    D[live, tok[live]] -= 1.0
    D *= torch.where(tok >= 0, g, 0.0).double()[:, None]
    h = HALF[dtype]
    for got, want, size in ((dX, D @ w, D.abs() @ w.abs()), (dW, D.T @ x, D.abs().T @ x.abs())):
        # one rounding of D and one of the result; sums and statistics in float32
        assert ((got.double() - want).abs() <= 1.01 * h * (size + want.abs()) + 1e-4 * size + 2.0 ** -24).all()
    again = jarq.cross_entropy_grad(X, W, tok, lse, g)
    assert torch.equal(again[0], dX) and torch.equal(again[1], dW)


@pytest.mark.parametrize("dtype", TC.TYPES)
@pytest.mark.parametrize("n,d,vocab", [(1, 1, 1), (3, 1, 5), (5, 3, 300), (1, 7, 40), (300, 2, 1)])
def test_narrowest_heads(jarq, dtype, n, d, vocab):
    rng = np.random.default_rng(n + d)
    X, W, tok, g = TC.inputs(rng, n, d, vocab, dtype)
    loss, lse = TC.check_loss(jarq, X, W, tok)
    TC.check_grad(jarq, X, W, tok, lse, g)


@pytest.mark.parametrize("dtype", TC.TYPES)
@pytest.mark.parametrize("size", [40.0, 300.0])
@pytest.mark.parametrize("d", [64, 1100])
def test_logits_of_any_size(jarq, monkeypatch, dtype, size, d):
    """Logits on both sides of 2^16, where the exponentials are formed another way, in the
    same rows' neighbours too."""
    # an exponential below 2^-126, float32's smallest normal number, is 0: so much of |g| may be
    # missing from an entry of D, which bfloat16 would hold (and round by less than 2^-133)
    monkeypatch.setitem(TC.FLOOR, "bfloat16", 2.0 ** -126 + 2.0 ** -133)
    rng = np.random.default_rng(d)
    X, W, tok, g = TC.inputs(rng, 50, d, 700, dtype, scale=2.0, ignored=False)
    X[::3] = (X[::3].float() * size).to(X.dtype)
    W = (W.float() * size).to(W.dtype)
    g[::2] = -g[::2]
    loss, lse = TC.check_loss(jarq, X, W, tok)
    TC.check_grad(jarq, X, W, tok, lse, g)


@pytest.mark.parametrize("dtype", TA.TYPES)
@pytest.mark.parametrize("n", [1, 3, 70])
@pytest.mark.parametrize("din,dout", [(1, 1), (3, 1), (1, 70), (7, 5)])
def test_narrowest_adapters(jarq, dtype, n, din, dout):
    TA.check(jarq, *TA.inputs(np.random.default_rng(n), n, din, dout, 8, 3, dtype))
