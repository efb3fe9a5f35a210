"""The loss of an output head and its gradient on the GPU against the float64
reference, within bounds counted from the products' float32 sums, the softmax's
float32 statistics and the one rounding of the logits' gradient to 16 bits."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")

pytestmark = [pytest.mark.gpu,
              pytest.mark.skipif(not torch.cuda.is_available(), reason="needs a CUDA GPU")]

from oracle import jarq_tuning as O  # noqa: E402
from test_gpu_norm import HALF, U, device, f64, near, randn  # noqa: E402

TYPES = ["float16", "bfloat16"]
# what a float16 gradient keeps of a row: 2^-24 of 2^14 for |g| up to 1 (its smallest number)
FLOOR = {"float16": 2.0 ** -25 / 2.0 ** 13, "bfloat16": 0.0}


@pytest.fixture(scope="module")
def jarq():
    from paper_2609_38599_gb300 import jarq as J
    return J


def inputs(rng, n, d, vocab, dtype, scale=2.0, ignored=True):
    X, W = randn(rng, n, d, dtype), randn(rng, vocab, d, dtype, scale / np.sqrt(d))
    tok = torch.as_tensor(rng.integers(0, vocab, n))
    # half of the rows know their token
    X[::2] = (X[::2].double() + 3.0 * W[tok[::2]].double()).to(X.dtype)
    if ignored and n > 3:
        tok[1::5] = -1
    return X, W, tok, torch.as_tensor(rng.uniform(0.2, 1.0, n).astype(np.float32) / n)


def sum_error(k):
    """Bound of a float32 sum of k exact products on the tensor cores, relative to the
    sum of their magnitudes: sixteen at a time, each addition counted as two roundings."""
    return (2 * -(-k // 16) + 2) * 2.0 ** -23


def logit_error(X, W):
    """Largest error of a row's logits."""
    return sum_error(X.shape[1]) * (np.abs(X) @ np.abs(W).T).max(1)


def check_loss(jarq, X, W, tok, args=None):
    loss, lse = jarq.cross_entropy(*(args or (X.cuda(), W.cuda(), tok.cuda())))
    x, w, t = f64(X), f64(W), tok.numpy()
    wl, ws = O.cross_entropy(x, w, t)
    logits = x @ w.T
    # exponentials: two units of their own and 1.5 |distance| of their argument; a
    # thread adds up to 32 terms of 128, and a row's parts are joined
    far = (np.exp(logits - ws[:, None]) * (logits.max(1)[:, None] - logits)).sum(1)
    rel = U * (40 + 4 + w.shape[0] / 128 / 4 + 20 + 4 * (far + 1))
    err = logit_error(x, w) + rel
    near(lse, ws, 1.01 * (err + 2 * U * (np.abs(ws) + np.abs(logits.max(1)))))
    near(loss, wl, 1.01 * (2 * err + 4 * U * (np.abs(ws) + np.abs(np.nan_to_num(wl)))))
    assert not (loss < 0).any()
    return loss, lse


def check_grad(jarq, X, W, tok, lse, g, args=None, **kw):
    dtype = str(X.dtype)[6:]
    dX, dW = jarq.cross_entropy_grad(*(args or (X.cuda(), W.cuda(), tok.cuda(), lse, g.cuda())), **kw)
    x, w, t, s = f64(X), f64(W), tok.numpy(), f64(lse)
    gn = f64(g)
    D = O.logit_gradient(x, w, t, s, gn)
    logits = x @ w.T
    p = np.where((t >= 0)[:, None], np.exp(logits - s[:, None]), 0.0)
    # p's relative error: the logit's, its distance from lse rounded, the exponential's;
    # then p - 1 and the product with g in float32, and one rounding to 16 bits
    rel = logit_error(x, w)[:, None] + 4 * U * (np.abs(logits) + np.abs(s)[:, None] + 2)
    a = np.abs(gn)[:, None]
    errD = a * p * rel + np.abs(D) * (HALF[dtype] + 4 * U) + a * FLOOR[dtype]
    tiny = float(torch.finfo(X.dtype).tiny) * HALF[dtype]
    for got, want, err in ((dX, D @ w, errD @ np.abs(w) + sum_error(len(w)) * 2 * (np.abs(D) @ np.abs(w))),
                           (dW, D.T @ x, errD.T @ np.abs(x) + sum_error(len(x)) * 2 * (np.abs(D).T @ np.abs(x)))):
        if got is not None:
            near(got, want, 1.01 * err + HALF[dtype] * 1.01 * np.abs(want) + tiny)
    return dX, dW


SIZES = [(1, 8, 1), (1, 64, 2), (3, 64, 257), (2, 16, 129), (5, 4096, 2001), (130, 72, 1000), (257, 200, 1023),
         (300, 512, 5000), (513, 64, 300), (64, 1344, 3000), (1, 1000, 4099)]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("n,d,vocab", SIZES)
def test_loss_and_gradient(jarq, dtype, n, d, vocab):
    rng = np.random.default_rng(n + d + vocab)
    X, W, tok, g = inputs(rng, n, d, vocab, dtype)
    loss, lse = check_loss(jarq, X, W, tok)
    assert (loss[tok.cuda() < 0] == 0).all()
    both = check_grad(jarq, X, W, tok, lse, g)
    # each gradient alone is the same
    assert torch.equal(check_grad(jarq, X, W, tok, lse, g, head=False)[0], both[0])
    assert torch.equal(check_grad(jarq, X, W, tok, lse, g, hidden=False)[1], both[1])
    assert jarq.async_status() == jarq.JARQ_OK


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("n,d,vocab,px,pw,ox,ow", [(33, 77, 515, 77, 77, 0, 0), (40, 64, 300, 72, 64, 8, 0),
                                                   (40, 64, 300, 64, 72, 0, 8), (7, 100, 260, 101, 104, 3, 0),
                                                   (300, 129, 1025, 136, 131, 0, 5), (1, 65, 200, 65, 72, 1, 0)])
def test_strides_and_alignment(jarq, dtype, n, d, vocab, px, pw, ox, ow):
    rng = np.random.default_rng(px + pw)
    X, W, tok, g = inputs(rng, n, d, vocab, dtype)
    x, w = device(X, px, ox), device(W, pw, ow)
    loss, lse = check_loss(jarq, X, W, tok, (x, w, tok.cuda()))
    check_grad(jarq, X, W, tok, lse, g, (x, w, tok.cuda(), lse, g.cuda()))


@pytest.mark.parametrize("dtype", TYPES)
def test_ignored_rows_may_hold_anything(jarq, dtype):
    """NaN and infinities in rows that do not count: their gradient is 0, and the head's
    is that of the other rows."""
    rng = np.random.default_rng(3)
    X, W, tok, g = inputs(rng, 70, 128, 700, dtype, ignored=False)
    dead = torch.zeros(70, dtype=torch.bool)
    dead[[0, 7, 33, 69]] = True
    dead[40:60] = True
    tok[dead] = -5
    g[7] = float("nan")
    X[dead] = float("nan")
    X[33] = float("inf")
    x, w, t, gg = X.cuda(), W.cuda(), tok.cuda(), g.cuda()
    loss, lse = jarq.cross_entropy(x, w, t)
    assert (loss[dead.cuda()] == 0).all()
    l2, s2 = check_loss(jarq, X[~dead], W, tok[~dead])
    assert torch.equal(loss[~dead.cuda()], l2)
    # against the reference of the same rows with zeros in their place
    lse[dead.cuda()] = 0
    args = (x, w, t, lse, gg)
    X, g = X.clone(), g.clone()
    X[dead], g[dead] = 0, 0
    dX, dW = check_grad(jarq, X, W, tok, lse, g, args)
    assert (dX[dead.cuda()] == 0).all()


@pytest.mark.parametrize("dtype", TYPES)
def test_all_rows_ignored(jarq, dtype):
    X, W, tok, g = inputs(np.random.default_rng(4), 20, 64, 300, dtype)
    tok[:] = -1
    loss, lse = check_loss(jarq, X, W, tok)
    dX, dW = jarq.cross_entropy_grad(X.cuda(), W.cuda(), tok.cuda(), lse, g.cuda())
    assert (loss == 0).all() and (dX == 0).all() and (dW == 0).all()


@pytest.mark.parametrize("dtype", TYPES)
def test_tokens_past_the_vocabulary_and_rows_that_are_not_finite(jarq, dtype):
    X, W, tok, g = inputs(np.random.default_rng(5), 9, 64, 300, dtype, ignored=False)
    tok[4] = 300
    X[6, 3] = float("nan")
    loss, lse = jarq.cross_entropy(X.cuda(), W.cuda(), tok.cuda())
    assert loss.isnan().nonzero().flatten().tolist() == [4, 6] and lse.isnan().nonzero().flatten().tolist() == [6]
    dX, _ = jarq.cross_entropy_grad(X.cuda(), W.cuda(), tok.cuda(), lse, g.cuda(), head=False)
    assert dX.isnan().any(1).nonzero().flatten().tolist() == [4, 6]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("vocab", [3, 500])
def test_confident_rows(jarq, dtype, vocab):
    """All mass on one token: a loss of 0, not below, and nothing but that token's
    rounding in the gradient; and a token with no mass at all."""
    n, d = 40, 64
    rng = np.random.default_rng(6)
    W = randn(rng, vocab, d, dtype, 0.1)
    W[1] = 8.0
    X = torch.ones(n, d, dtype=W.dtype)
    tok = torch.ones(n, dtype=torch.int64)
    tok[n // 2:] = 2
    loss, lse = jarq.cross_entropy(X.cuda(), W.cuda(), tok.cuda())
    assert (loss[: n // 2] == 0).all() and (loss[n // 2:] > 400).all() and (lse == 512).all()
    g = torch.full((n,), 1.0)
    dX, _ = jarq.cross_entropy_grad(X.cuda(), W.cuda(), tok.cuda(), lse, g.cuda())
    assert (dX[: n // 2] == 0).all()
    near(dX[n // 2:], np.broadcast_to(f64(W[1] - W[2].float()), (n // 2, d)), HALF[dtype] * 1.01 * 9.0)


@pytest.mark.parametrize("dtype", TYPES)
def test_masked_logits(jarq, dtype):
    """Logits of minus infinity: no probability and no gradient; rows with nothing else."""
    n, d, vocab = 6, 64, 400
    X, W, tok, g = inputs(np.random.default_rng(7), n, d, vocab, dtype, ignored=False)
    X[:, 0] = 1.0
    W[300:, 0] = -float("inf")
    tok[:] = 5
    tok[3] = 350
    loss, lse = jarq.cross_entropy(X.cuda(), W.cuda(), tok.cuda())
    wl, ws = jarq.cross_entropy(X.cuda(), W[:300].cuda(), tok.cuda() % 300)
    assert torch.equal(lse, ws) and torch.equal(loss[:3], wl[:3]) and loss[3] == float("inf")
    W[:, 0] = -float("inf")
    loss, lse = jarq.cross_entropy(X.cuda(), W.cuda(), tok.cuda())
    assert (lse == -float("inf")).all() and (loss == float("inf")).all()


@pytest.mark.parametrize("spread", [0, 6, 12])
def test_float16_gradient_keeps_small_weights(jarq, spread):
    """Weights of the loss far below float16's range, and of different sizes."""
    rng = np.random.default_rng(8)
    X, W, tok, g = inputs(rng, 100, 128, 900, "float16", ignored=False)
    g = torch.as_tensor((2.0 ** -40 * 2.0 ** rng.uniform(-spread, 0, 100)).astype(np.float32))
    loss, lse = jarq.cross_entropy(X.cuda(), W.cuda(), tok.cuda())
    # scaled back into range by an exact power of two after the fact: the same products
    dX, dW = jarq.cross_entropy_grad(X.cuda(), W.cuda(), tok.cuda(), lse, (g * 2.0 ** 40).cuda())
    check_grad(jarq, X, W, tok, lse, g * 2.0 ** 40)
    small = jarq.cross_entropy_grad(X.cuda(), W.cuda(), tok.cuda(), lse, (g * 2.0 ** 30).cuda())
    # powers of two are exact but where the result is below float16's normal numbers
    for a, b in ((dX, small[0]), (dW, small[1])):
        assert ((a.double() * 2.0 ** -10 - b.double()).abs() <= 2.0 ** -24).all()


def test_gradient_against_differences(jarq):
    rng = np.random.default_rng(10)
    X, W, tok, g = inputs(rng, 6, 64, 200, "bfloat16", ignored=False)
    g = g * 6
    loss, lse = jarq.cross_entropy(X.cuda(), W.cuda(), tok.cuda())
    dX, dW = jarq.cross_entropy_grad(X.cuda(), W.cuda(), tok.cuda(), lse, g.cuda())
    total = lambda x, w: (f64(jarq.cross_entropy(x.cuda(), w.cuda(), tok.cuda())[0]) * f64(g)).sum()
    for which, grad, at in ((0, dX, [(0, 0), (3, 17), (5, 63)]), (1, dW, [(0, 5), (int(tok[2]), 9), (199, 63)])):
        for i in at:
            hi, lo = [X.clone(), W.clone()], [X.clone(), W.clone()]
            step = 2.0 ** -4
            hi[which][i] += step
            lo[which][i] -= step
            diff = (total(*hi) - total(*lo)) / float(hi[which][i].double() - lo[which][i].double())
            # the gradient's two roundings; third derivatives (at most |w|^3 or |x|^3 below
            # 60 here, 1/6 and g at most 1) times step^2 / 6; the losses' rounding over the step
            assert abs(diff - grad[i].item()) < 2 * HALF["bfloat16"] * (abs(diff) + 1) + 60 * step ** 2 / 6 * 0.5 + 1e-4


def test_several_pieces_and_splits(jarq):
    """A gradient in two pieces of the vocabulary, and sums in several splits, against
    plain products in float64."""
    for n, d, vocab in ((8192, 64, 40000), (64, 320, 9000), (2000, 64, 1100)):
        gen = torch.Generator(device="cuda").manual_seed(n)
        X = torch.randn(n, d, generator=gen, device="cuda").bfloat16()
        W = (torch.randn(vocab, d, generator=gen, device="cuda") * 0.3).bfloat16()
        tok = torch.randint(0, vocab, (n,), generator=gen, device="cuda")
        g = torch.rand(n, generator=gen, device="cuda") / n
        loss, lse = jarq.cross_entropy(X, W, tok)
        dX, dW = jarq.cross_entropy_grad(X, W, tok, lse, g)
        logits = X.double() @ W.double().T
        # as in check_loss, every exponential at the row's range from the maximum
        err = sum_error(d) * (X.double().abs() @ W.double().abs().T).amax(1)
        err += U * (68 + vocab / 512 + 4 * (logits.amax(1) - logits.amin(1) + 1))
        want = torch.logsumexp(logits, 1)
        assert ((want - lse).abs() <= 1.01 * (err + 4 * U * want.abs())).all()
        wl = want - logits.gather(1, tok[:, None])[:, 0]
        assert ((wl - loss).abs() <= 1.01 * (2 * err + 4 * U * (want.abs() + wl.abs()))).all()
        D = torch.exp(logits - lse.double()[:, None])
        D[torch.arange(n), tok] -= 1.0
        D *= g.double()[:, None]
        h = HALF["bfloat16"]
        for got, want, size in ((dX, D @ W.double(), D.abs() @ W.double().abs()), (dW, D.T @ X.double(), D.T.abs() @ X.double().abs())):
            # one rounding of D and one of the result; sums and statistics in float32
            assert ((got.double() - want).abs() <= 1.01 * h * (size + want.abs()) + 1e-4 * size + 1e-30).all()
        del logits, D


def test_no_rows(jarq):
    X, W = torch.zeros(0, 64, device="cuda").half(), torch.zeros(100, 64, device="cuda").half()
    tok = torch.zeros(0, dtype=torch.int64, device="cuda")
    loss, lse = jarq.cross_entropy(X, W, tok)
    dX, dW = jarq.cross_entropy_grad(X, W, tok, lse, loss)
    assert loss.shape == lse.shape == (0,) and dX.shape == (0, 64) and dW.shape == (100, 64) and (dW == 0).all()


def test_same_bits_again_and_in_graphs_that_share_memory(jarq):
    """Two captured graphs with workspaces of one pool, replayed in turn, an eager call
    between them, give what eager calls give."""
    rng = np.random.default_rng(12)
    sets = [[t.cuda() for t in inputs(rng, n, 192, 3001, "bfloat16")] for n in (200, 90)]
    want = []
    for X, W, tok, g in sets:
        loss, lse = jarq.cross_entropy(X, W, tok)
        want.append((loss, lse, *jarq.cross_entropy_grad(X, W, tok, lse, g)))
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    graphs, got, pool = [], [], torch.cuda.graph_pool_handle()
    for X, W, tok, g in sets:
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, pool=pool, stream=stream):
            loss, lse = jarq.cross_entropy(X, W, tok)
            got.append((loss, lse, *jarq.cross_entropy_grad(X, W, tok, lse, g)))
        graphs.append(graph)
    for _ in range(2):
        for i, graph in enumerate(graphs):
            graph.replay()
            X, W, tok, g = sets[i]
            assert torch.equal(jarq.cross_entropy(X, W, tok)[0], want[i][0])
            assert all(torch.equal(a, b) for a, b in zip(got[i], want[i]))
    assert jarq.async_status() == jarq.JARQ_OK


def test_two_streams_at_once(jarq):
    rng = np.random.default_rng(13)
    sets = [[t.cuda() for t in inputs(rng, n, 256, 4000, "float16")] for n in (300, 280)]
    want = [jarq.cross_entropy(X, W, tok)[0] for X, W, tok, _ in sets]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in sets]
    for _ in range(5):
        got = []
        for s, (X, W, tok, g) in zip(streams, sets):
            with torch.cuda.stream(s):
                loss, lse = jarq.cross_entropy(X, W, tok)
                got.append((loss, jarq.cross_entropy_grad(X, W, tok, lse, g)))
        torch.cuda.synchronize()
        assert all(torch.equal(a[0], b) for a, b in zip(got, want))


def test_a_wait_that_gives_up_is_reported(jarq):
    assert jarq.selftest_stalled_kernel("cross_entropy") == jarq.JARQ_ERR_TIMEOUT
    assert jarq.async_status() == jarq.JARQ_OK


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("n,d,vocab,px", [(1, 64, 2000, 64), (60, 72, 4000, 72), (60, 77, 4000, 80), (700, 264, 9000, 264),
                                          (8300, 40, 40000, 40)])
def test_a_tokens_own_entry_is_not_rounded(jarq, dtype, n, d, vocab, px):
    """Equal weights whose mantissa lies between two of the type's: rounding the entry of
    a row's own token, about -g, would move the whole row the same way."""
    rng = np.random.default_rng(n + d)
    ulp = 2.0 * HALF[dtype]
    X = randn(rng, n, d, dtype)
    W = torch.zeros(vocab, d).to(X.dtype)              # only tokens that occur hold anything
    known = torch.as_tensor(rng.choice(vocab, 16, replace=False))
    W[known] = randn(rng, 16, d, dtype, 1 / np.sqrt(d))
    tok = known[torch.as_tensor(rng.integers(0, 16, n))]
    if n > 3:
        tok[1::5] = -1
    g = torch.full((n,), 2.0 ** -6 * (1 + 0.45 * ulp))
    x, w = device(X, px, 0), device(W, px, 0)
    t = tok.cuda()
    loss, lse = jarq.cross_entropy(x, w, t)
    dX, dW = jarq.cross_entropy_grad(x, w, t, lse, g.cuda())
    xn, wn, gn, tn = f64(X), f64(W), f64(g), tok.numpy()
    logits = xn @ wn.T
    D = O.logit_gradient(xn, wn, tn, f64(lse), gn)
    p = np.where((tn >= 0)[:, None], np.exp(logits - f64(lse)[:, None]), 0.0)
    rel = logit_error(xn, wn)[:, None] + 4 * U * (np.abs(logits) + np.abs(f64(lse))[:, None] + 2)
    rounded = np.abs(D)
    rows = np.flatnonzero(tn >= 0)
    rounded[rows, tn[rows]] = 0                         # these are put right
    errD = gn[:, None] * (p * rel + FLOOR[dtype]) + rounded * HALF[dtype] + np.abs(D) * 4 * U
    tiny = float(torch.finfo(X.dtype).tiny) * HALF[dtype]
    # what is put back: at most HALF |D|, its products and sums in float32
    back = HALF[dtype] * (n + 2) * U
    for got, want, err, size in ((dX, D @ wn, errD @ np.abs(wn), np.abs(D) @ np.abs(wn)), (dW, D.T @ xn, errD.T @ np.abs(xn), np.abs(D).T @ np.abs(xn))):
        k = vocab if got is dX else n
        near(got, want, 1.01 * (err + (2 * sum_error(k) + back) * size + HALF[dtype] * np.abs(want)) + tiny)
    again = jarq.cross_entropy_grad(x, w, t, lse, g.cuda())
    assert torch.equal(again[0], dX) and torch.equal(again[1], dW)
    assert torch.equal(jarq.cross_entropy_grad(x, w, t, lse, g.cuda(), hidden=False)[1], dW)
    assert jarq.async_status() == jarq.JARQ_OK


@pytest.mark.parametrize("dtype", TYPES)
def test_rows_of_the_same_token(jarq, dtype):
    """Tokens that first occur, and come again, on both sides of 16, 2048 and 4096 rows, tokens
    whose low bytes agree, and one token in every row."""
    rng = np.random.default_rng(3)
    n, d, vocab = 9001, 24, 600
    X = randn(rng, n, d, dtype)
    W = randn(rng, vocab, d, dtype, 0.1)
    g = torch.full((n,), 2.0 ** -6 * (1 + 0.9 * HALF[dtype]))
    for case in ("borders", "all", "any"):
        tok = torch.as_tensor(rng.integers(0, vocab, n)) if case == "any" else torch.full((n,), 256 if case == "all" else -1)
        if case == "borders":
            tok[[0, 15, 16, 2047, 2048, 4095, 4096, 8191, 8192, 9000]] = torch.as_tensor([0, 256, 0, 512, 256, 0, 512, 1, 0, 257])
        loss, lse = jarq.cross_entropy(X.cuda(), W.cuda(), tok.cuda())
        args = (X.cuda(), W.cuda(), tok.cuda(), lse, g.cuda())
        dX, dW = jarq.cross_entropy_grad(*args)
        assert torch.equal(jarq.cross_entropy_grad(*args)[1], dW)
        x, w, t = f64(X), f64(W), tok.numpy()
        logits = x @ w.T
        live = np.flatnonzero(t >= 0)
        D = O.logit_gradient(x, w, t, f64(lse), f64(g))
        p = np.where((t >= 0)[:, None], np.exp(logits - f64(lse)[:, None]), 0.0)
        rel = logit_error(x, w)[:, None] + 4 * U * (np.abs(logits) + np.abs(f64(lse))[:, None] + 2)
        rounded = np.abs(D)
        rounded[live, t[live]] = 0
        errD = f64(g)[:, None] * (p * rel + FLOOR[dtype]) + rounded * HALF[dtype] + np.abs(D) * 4 * U
        tiny = float(torch.finfo(X.dtype).tiny) * HALF[dtype]
        size = np.abs(D).T @ np.abs(x)
        err = errD.T @ np.abs(x) + (2 * sum_error(n) + HALF[dtype] * (n + 2) * U) * size
        want = D.T @ x
        near(dW, want, 1.01 * (err + HALF[dtype] * np.abs(want)) + tiny)

