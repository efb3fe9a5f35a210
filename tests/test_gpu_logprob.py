"""Log probabilities of tokens, entropies, alternatives and their gradient on
the GPU against the float64 reference, within bounds derived from the float32
sums, and exactly where values are whole numbers or have no rounding."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")

pytestmark = [pytest.mark.gpu,
              pytest.mark.skipif(not torch.cuda.is_available(), reason="needs a CUDA GPU")]

from oracle import jarq_inference as O  # noqa: E402

DT = {"float32": torch.float32, "float16": torch.float16, "bfloat16": torch.bfloat16}
U = 2.0 ** -24


@pytest.fixture(scope="module")
def jarq():
    from paper_2609_38599_gb300 import jarq as J
    return J


def _device(x, pitch=None, offset=0):
    n, v = x.shape
    pitch = pitch or v
    flat = torch.full((offset + max(0, n - 1) * pitch + v,), float("nan"), dtype=x.dtype, device="cuda")
    d = torch.as_strided(flat, (n, v), (pitch, 1), offset)
    d.copy_(x)
    return d


def _same(got, want):
    """Equal where the value is NaN or infinite."""
    got, want = got.double().cpu().numpy(), np.asarray(want, dtype=np.float64)
    fine = np.isfinite(want)
    assert np.array_equal(np.isnan(got), np.isnan(want))
    assert np.array_equal(got[~fine & ~np.isnan(want)], want[~fine & ~np.isnan(want)])
    return np.where(fine, got, 0.0), np.where(fine, want, 0.0), fine


def _bounds(x, ref):
    """Per row: bound of the relative error of the sum of exponentials, the mean
    distance from the maximum, and the sizes of m and ln s.  A thread adds at
    most V / 256 + 8 terms one after the other and 16 more levels join them, an
    exponential has 2 units of its own and those of its rounded argument, |d|
    units of 1.5 2^-24 each."""
    out = []
    for r in range(x.shape[0]):
        row = x[r][np.isfinite(x[r])]
        if row.size == 0 or not np.isfinite(ref["lse"][r]):
            out.append((0.0, 0.0, 0.0, 0.0))
            continue
        m = row.max()
        d = row - m
        w = np.exp(d)
        mean = float((w * -d).sum() / w.sum())
        out.append((U * (x.shape[1] / 256 + 32 + 4 + 3 * mean), mean, abs(m), abs(float(np.log(w.sum())))))
    return np.array(out).T


def check(jarq, x, tok, top, logits=None):
    """`x`: torch matrix (host); the library's results against the reference's."""
    x64 = x.double().numpy()
    d = logits if logits is not None else _device(x)
    r = jarq.token_logprobs(d, None if tok is None else torch.as_tensor(tok).cuda(), top)
    t2 = np.zeros((x.shape[0], 0), np.int64) if tok is None else np.asarray(tok).reshape(x.shape[0], -1)
    ref = O.token_logprobs(x64, t2, top)
    rel, mean, m, logz = _bounds(x64, ref)
    # lse = m + ln s: the sum's relative error, ln's last place and one rounding
    got, want, _ = _same(r.lse, ref["lse"])
    assert (np.abs(got - want) <= 1.01 * (rel + 2 * U * logz + U * (m + logz)) + 1e-37).all()
    # entropy = ln s - u / s; u's terms carry the exponentials' errors and one of their own
    got, want, _ = _same(r.entropy, ref["entropy"])
    assert (np.abs(got - want) <= 1.01 * (rel + 2 * U * logz + (2 * rel + 4 * U) * (mean + 1) + U * (logz + mean)) + 1e-37).all()
    def close(got, want):
        got, want, _ = _same(got, want)
        bound = rel + 2 * U * logz
        assert (np.abs(got - want) <= 1.01 * (bound[:, None] + U * (2 * np.abs(want) + logz[:, None])) + 1e-37).all()
    if tok is None:
        assert r.logprob is None
    else:
        assert tuple(r.logprob.shape) == tuple(np.shape(tok))
        close(r.logprob.reshape(x.shape[0], -1), ref["logprob"])
    if top:
        assert np.array_equal(r.top_token.cpu().numpy(), ref["top_token"])
        close(r.top_logprob, ref["top_logprob"])
    return r, ref


def _logits(rng, n, v, dtype, scale=3.0):
    return torch.as_tensor((rng.standard_normal((n, v)) * scale).astype(np.float32)).to(DT[dtype])


@pytest.mark.parametrize("dtype", list(DT))
@pytest.mark.parametrize("n,v,t,top", [(1, 1, 1, 1), (2, 2, 1, 2), (3, 31, 2, 31), (5, 33, 1, 32), (4, 1000, 3, 5),
                                       (1, 32000, 1, 8), (2, 50001, 4, 20), (7, 4099, 1, 0), (1, 131072, 1, 32),
                                       (200, 2500, 1, 3), (700, 301, 2, 4), (3, 131075, 256, 1)])
def test_scores(jarq, dtype, n, v, t, top):
    rng = np.random.default_rng(n + v)
    tok = rng.integers(0, v, (n, t))
    tok[::3, 0] = -1
    check(jarq, _logits(rng, n, v, dtype), tok, top)


@pytest.mark.parametrize("dtype", list(DT))
@pytest.mark.parametrize("pitch,offset", [(None, 1), (1003, 0), (1010, 3), (1024, 8)])
def test_strides_and_alignment(jarq, dtype, pitch, offset):
    """What lies between the rows (NaN here) is not read."""
    rng = np.random.default_rng(offset)
    x = _logits(rng, 9, 1001, dtype)
    check(jarq, x, rng.integers(0, 1001, 9), 7, _device(x, pitch, offset))


def test_no_tokens_and_no_alternatives(jarq):
    check(jarq, _logits(np.random.default_rng(0), 3, 100, "float32"), None, 0)


@pytest.mark.parametrize("dtype", list(DT))
@pytest.mark.parametrize("v", [40, 3001, 40000])
def test_equal_logits_go_to_the_lowest_token(jarq, dtype, v):
    rng = np.random.default_rng(v)
    x = torch.zeros(6, v)
    x[1] = -7.5
    x[2] = torch.as_tensor(rng.integers(0, 2, v).astype(np.float32))
    x[3] = torch.as_tensor(rng.integers(0, 4, v).astype(np.float32))
    x[4, ::2] = -0.0
    x[5, v // 2:] = 1.0
    check(jarq, x.to(DT[dtype]), np.full((6, 1), v - 1), 32)


@pytest.mark.parametrize("v", [2000, 70000])
def test_sorted_rows(jarq, v):
    """The order of the logits that finds the most candidates, and its mirror."""
    x = torch.stack([torch.linspace(-20, 5, v), torch.linspace(5, -20, v), torch.linspace(-1e-3, 1e-3, v)])
    check(jarq, x, np.array([[0, v - 1]] * 3), 32)


@pytest.mark.parametrize("dtype", list(DT))
@pytest.mark.parametrize("v", [70, 5000, 33333])
def test_masks(jarq, dtype, v):
    """-inf in part of a row, all but some, all but one, all; the type's lowest
    value in their place, alone and beside -inf."""
    rng = np.random.default_rng(v)
    low = float(torch.finfo(DT[dtype]).min)
    x = _logits(rng, 9, v, dtype)
    x[0, torch.as_tensor(rng.random(v) < 0.5)] = -np.inf
    x[1, 3:] = -np.inf
    x[2] = -np.inf
    x[2, v - 1] = 2.0
    x[3] = -np.inf
    x[4, 2:] = low
    x[5] = low
    x[6] = low
    x[6, : v // 2] = -np.inf
    x[7, :-1] = -np.inf
    x[7, -1] = low
    x[8, 10] = float(torch.finfo(DT[dtype]).max)
    tok = np.stack([rng.integers(0, v, 9), np.full(9, v - 1), np.full(9, -5)], 1)
    check(jarq, x, tok, 8)


@pytest.mark.parametrize("v", [50, 9000])
@pytest.mark.parametrize("at", [0, 37])
def test_nan_and_infinity_make_the_row_nan(jarq, v, at):
    rng = np.random.default_rng(at)
    x = _logits(rng, 5, v, "float32")
    x[0, at] = np.nan
    x[1, at] = np.inf
    x[2] = -np.inf
    x[2, at] = np.nan
    x[3, at] = np.inf
    x[3, at + 1] = -np.inf
    r, _ = check(jarq, x, np.array([[at, v - 1, -1]] * 5), 4)
    assert torch.isnan(r.lse[:4]).all() and torch.isfinite(r.lse[4])
    assert (r.logprob[:, 2] == 0).all() or torch.isnan(r.logprob[:4, 2]).all()


def test_tokens_outside_the_vocabulary(jarq):
    x = _logits(np.random.default_rng(1), 3, 100, "float16")
    r, _ = check(jarq, x, np.array([[100, 2], [1 << 40, -(1 << 40)], [99, 0]]), 2)
    assert torch.isnan(r.logprob[0, 0]) and torch.isnan(r.logprob[1, 0]) and r.logprob[1, 1] == 0


def test_large_logits(jarq):
    """Logits far from zero: the result depends on their differences alone."""
    x = torch.tensor([[10000.0, 9998.0, 9000.0], [-30000.0, -30001.0, -30000.5], [1e30, 0.0, -1e30]])
    check(jarq, x, np.array([[1], [1], [0]]), 3)


@pytest.mark.parametrize("dtype", ["float16"])
def test_logits_past_two_to_the_31(jarq, dtype):
    """Rows more than 2^31 elements into the logits, and their gradient."""
    n, v = 17000, 131072
    x = torch.empty(n, v, dtype=DT[dtype], device="cuda")
    x.normal_(generator=torch.Generator("cuda").manual_seed(0))
    tok = torch.full((n,), v - 1, device="cuda")
    r = jarq.token_logprobs(x, tok, 4)
    dx = jarq.token_logprobs_grad(x, tok, r.lse, torch.ones(n, device="cuda"))
    for i in (0, n - 1):
        ref = O.token_logprobs(x[i:i + 1].double().cpu().numpy(), np.array([[v - 1]]), 4)
        assert np.array_equal(r.top_token[i:i + 1].cpu().numpy(), ref["top_token"])
        assert abs(float(r.logprob[i]) - ref["logprob"][0, 0]) < 1e-4
        assert float(dx[i, v - 1]) == pytest.approx(1.0, abs=2e-3) and float(dx[i, :v - 1].float().max()) <= 0


# ---------------------------------------------------------------- gradient

UNIT = {"float32": (2.0 ** -24, 2.0 ** -126), "float16": (2.0 ** -11, 2.0 ** -25), "bfloat16": (2.0 ** -8, 2.0 ** -126)}


def check_grad(jarq, x, tok, seed, entropy, dtype, logits=None, out=None):
    rng = np.random.default_rng(seed)
    n, v = x.shape
    x64 = x.double().numpy()
    tok = np.asarray(tok).reshape(n, -1)
    ref = O.token_logprobs(x64, tok)
    lse, ent = ref["lse"].astype(np.float32), ref["entropy"].astype(np.float32)
    g = rng.standard_normal(tok.shape).astype(np.float32)
    gh = rng.standard_normal(n).astype(np.float32) if entropy else None
    c = lambda a: None if a is None else torch.as_tensor(a).cuda()
    d = logits if logits is not None else _device(x)
    dx = jarq.token_logprobs_grad(d, c(tok), c(lse), c(g), c(ent) if entropy else None, c(gh), out)
    want = O.token_logprobs_grad(x64, tok, lse, g, ent, gh)
    # p carries the rounding of x - lse (and of its product with log2 e) and two
    # units of the exponential; then a few roundings of the terms' magnitudes
    with np.errstate(invalid="ignore", over="ignore"):
        lp = np.where(x64 > -np.inf, x64 - lse[:, None], -1e4)
        p = np.where(x64 > -np.inf, np.exp(lp), 0.0)
        G = np.where(tok < 0, 0, np.abs(g)).sum(1)[:, None]
        size = G * p
        spread = np.zeros_like(p)
        if entropy:
            size = size + np.abs(gh)[:, None] * p * (np.abs(lp) + np.abs(ent)[:, None] + 1)
        for r in range(n):
            for j in range(tok.shape[1]):
                if 0 <= tok[r, j] < v:
                    spread[r, tok[r, j]] += abs(g[r, j])
        rel = U * (8 + 3 * np.minimum(np.abs(lp), 200.0) + tok.shape[1])
        u, tiny = UNIT[dtype]
        bound = 1.01 * (rel * size + U * (tok.shape[1] + 2) * spread + u * np.abs(want)) + tiny + 1e-37 * (G + 1)
    got, want, fine = _same(dx, want)
    assert (np.abs(got - want) <= np.where(fine, bound, 0)).all()
    return dx


@pytest.mark.parametrize("entropy", [False, True])
@pytest.mark.parametrize("dtype", list(DT))
@pytest.mark.parametrize("n,v,t", [(1, 1, 1), (3, 9, 2), (5, 1001, 1), (2, 32000, 3), (4, 8193, 256), (60, 515, 4)])
def test_gradient(jarq, dtype, n, v, t, entropy):
    rng = np.random.default_rng(n + v)
    tok = rng.integers(0, v, (n, t))
    tok[::4, 0] = -1
    if t > 2:
        tok[:, 1] = tok[:, 2]              # the same token twice
    check_grad(jarq, _logits(rng, n, v, dtype), tok, v, entropy, dtype)


@pytest.mark.parametrize("dtype", list(DT))
def test_gradient_of_masked_rows(jarq, dtype):
    rng = np.random.default_rng(2)
    v = 3000
    x = _logits(rng, 6, v, dtype)
    x[0, torch.as_tensor(rng.random(v) < 0.5)] = -np.inf
    x[1, 1:] = -np.inf
    x[2] = -np.inf
    x[3, 5:] = float(torch.finfo(DT[dtype]).min)
    tok = rng.integers(0, v, (6, 2))
    tok[0, 0] = int(torch.nonzero(torch.isinf(x[0]))[0])       # a masked target
    tok[1], tok[3, 0] = 0, 2
    dx = check_grad(jarq, x, tok, 1, True, dtype)
    assert (dx[torch.isinf(x).cuda()] == 0).all() and (dx[2] == 0).all()


def test_gradient_of_a_token_outside_the_vocabulary_is_nan(jarq):
    x = _logits(np.random.default_rng(1), 2, 64, "float32")
    dx = check_grad(jarq, x, np.array([[64], [63]]), 0, False, "float32")
    assert torch.isnan(dx[0]).all() and torch.isfinite(dx[1]).all()


@pytest.mark.parametrize("dtype", list(DT))
@pytest.mark.parametrize("pitch,offset,opitch,ooffset", [(1001, 1, 1001, 1), (1016, 0, 1024, 8), (1003, 0, 1002, 3)])
def test_gradient_strides_and_in_place(jarq, dtype, pitch, offset, opitch, ooffset):
    rng = np.random.default_rng(pitch)
    x = _logits(rng, 5, 1001, dtype)
    tok = rng.integers(0, 1001, (5, 2))
    out = _device(torch.zeros_like(x), opitch, ooffset)
    want = check_grad(jarq, x, tok, 3, True, dtype, _device(x, pitch, offset), out)
    place = _device(x, pitch, offset)
    dx = check_grad(jarq, x, tok, 3, True, dtype, place, place)
    assert dx.data_ptr() == place.data_ptr() and torch.equal(dx, want)
    flat = torch.as_strided(out, (5 * opitch - opitch + 1001,), (1,), ooffset)
    between = torch.ones(flat.numel(), dtype=torch.bool, device="cuda")
    for r in range(5):
        between[r * opitch:r * opitch + 1001] = False
    assert torch.isnan(flat[between]).all()                    # nothing written between the rows


def test_gradient_equals_differences_of_the_scores(jarq):
    """The gradient of the library's own scores, by central differences."""
    rng = np.random.default_rng(11)
    v, h = 24, 2.0 ** -4
    base = torch.as_tensor(rng.integers(-64, 65, v) / 16.0).float()     # x +- h exact
    tok = torch.tensor([[3, 7]]).cuda()
    g, gh = torch.tensor([[0.75, -1.25]]).cuda(), torch.tensor([0.5]).cuda()
    x = torch.stack([base] + [base + s * h * torch.eye(v)[i] for i in range(v) for s in (1, -1)]).cuda()
    r = jarq.token_logprobs(x, tok.expand(len(x), 2).contiguous())
    f = ((r.logprob * g).sum(1) + gh * r.entropy).double().cpu().numpy()
    dx = jarq.token_logprobs_grad(x[:1], tok, r.lse[:1].clone(), g, r.entropy[:1].clone(), gh)[0].double().cpu().numpy()
    diff = (f[1::2] - f[2::2]) / (2 * h)
    # truncation h^2 / 6 max |f'''|, f''' of logprob and entropy below 8; rounding 2^-21 / h
    assert np.abs(diff - dx).max() <= h * h / 6 * 8 + 2.0 ** -21 / h


def test_other_stream_and_graph(jarq):
    x = _device(_logits(np.random.default_rng(4), 6, 20000, "bfloat16"))
    tok = torch.arange(6, device="cuda")
    one = torch.ones(6, device="cuda")
    def both():
        r = jarq.token_logprobs(x, tok, 3)
        return r.logprob, r.top_token, jarq.token_logprobs_grad(x, tok, r.lse, one)
    want = both()
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        other = both()
    s.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(want, other))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = both()
    x.mul_(0.5)
    graph.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, both()))


def test_empty_batch_and_refusals(jarq):
    dev = dict(device="cuda")
    r = jarq.token_logprobs(torch.zeros(0, 10, **dev), torch.zeros(0, dtype=torch.int64, **dev), 2)
    assert r.logprob.shape == (0,) and r.top_token.shape == (0, 2)
    x, tok, f = torch.zeros(2, 10, **dev), torch.zeros(2, dtype=torch.int64, **dev), torch.zeros(2, **dev)
    assert jarq.token_logprobs_grad(x[:0], tok[:0], f[:0], f[:0]).shape == (0, 10)
    for bad in (lambda: jarq.token_logprobs(x.cpu(), tok), lambda: jarq.token_logprobs(x, tok.int()),
                lambda: jarq.token_logprobs(x, tok[:1]), lambda: jarq.token_logprobs(x.double(), tok),
                lambda: jarq.token_logprobs(x[0], tok), lambda: jarq.token_logprobs_grad(x, tok, f, f[:1]),
                lambda: jarq.token_logprobs_grad(x, tok, f, f, out=x.half())):
        with pytest.raises(TypeError):
            bad()
    for bad in (lambda: jarq.token_logprobs(x, tok, 11), lambda: jarq.token_logprobs(torch.zeros(2, 99, **dev), tok, 33),
                lambda: jarq.token_logprobs(x, tok, -1), lambda: jarq.token_logprobs(x, torch.zeros(2, 257, dtype=torch.int64, **dev)),
                lambda: jarq.token_logprobs(x[:1].expand(2, 10), tok),
                lambda: jarq.token_logprobs_grad(x, tok, f, f, None, f)):
        with pytest.raises(jarq.JarqError) as e:
            bad()
        assert e.value.status == jarq.JARQ_ERR_ARG
    lib = jarq.library()
    host = torch.zeros(2, 10)
    assert lib.jarq_token_logprobs(host.data_ptr(), 0, 2, 10, 10, None, 0, 0, None, None, None, None, None, None) == jarq.JARQ_ERR_ARG
    assert lib.jarq_token_logprobs(x.data_ptr() + 2, 0, 1, 8, 8, None, 0, 0, None, None, None, None, None, None) == jarq.JARQ_ERR_ARG
    torch.cuda.synchronize()
