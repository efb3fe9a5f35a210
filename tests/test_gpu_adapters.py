"""Adapters of many requests on the GPU against the float64 reference, within bounds
counted from the float32 sums and the 16-bit parts that the expansion multiplies."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")

pytestmark = [pytest.mark.gpu,
              pytest.mark.skipif(not torch.cuda.is_available(), reason="needs a CUDA GPU")]

from oracle import jarq_tuning as O  # noqa: E402
from test_gpu_norm import DT, HALF, U, device, f64, near, randn  # noqa: E402

TYPES = ["float16", "bfloat16"]


@pytest.fixture(scope="module")
def jarq():
    from paper_2609_38599_gb300 import jarq as J
    return J


def inputs(rng, n, din, dout, rank, m, dtype, ydtype=None, order="any"):
    X = randn(rng, n, din, dtype)
    A = randn(rng, m * rank, din, dtype, din ** -0.5).reshape(m, rank, din)
    B = randn(rng, m * dout, rank, dtype, 0.2).reshape(m, dout, rank)
    ids = rng.integers(0, m, n).astype(np.int32)
    if order == "runs":
        ids = np.sort(ids)
    if n > 2:
        ids[n // 2] = -1
    scale = rng.uniform(0.5, 2.0, m).astype(np.float32)
    return X, A, B, torch.as_tensor(ids), torch.as_tensor(scale), randn(rng, n, dout, ydtype or dtype)


def check(jarq, X, A, B, ids, scale, base, args=None, **kw):
    got = jarq.apply_adapters(*(args or [None if t is None else t.cuda() for t in (X, A, B, ids, scale, base)]), **kw)
    x, a, b, i = f64(X), f64(A), f64(B), ids.numpy()
    s = np.ones(len(a)) if scale is None else f64(scale)
    want = O.apply_adapters(x, a, b, i, s, None if base is None else f64(base))
    out = str(got.dtype)[6:]
    # u = A x: a sum of din exact products in float32 (each addition counted as two
    # roundings), then scaled; the two 16-bit parts of u keep it to 2^-16 (bfloat16) or to
    # 2^-22 of the token's largest (float16), three to 2^-24
    ok = (i >= 0) & (i < len(a))
    err, size = np.zeros_like(want), np.zeros_like(want)
    for r in np.flatnonzero(ok):
        U_, V = np.abs(a[i[r]]) @ np.abs(x[r]), np.abs(a[i[r]] @ x[r])
        du = (2 * -(-x.shape[1] // 16) + 34) * 2 * U * U_ + 2 * U * V
        # (the float32 sum behind u may differ from the float64 one by du itself)
        du = du + (V + du) * (2.0 ** -16 if X.dtype == torch.bfloat16 and out != "float32" else 2.0 ** -23) + 2.0 ** -22 * V.max()
        err[r] = s[i[r]] * (np.abs(b[i[r]]) @ du)
        size[r] = s[i[r]] * (np.abs(b[i[r]]) @ V)
    # the expansion's sum over rank (and parts), the addition, one rounding
    err = 1.01 * (err + (2 * a.shape[1] / 16 * 3 + 12 + a.shape[1] * (len(x) <= 64)) * 2 * U * size) + 2 * U * np.abs(np.nan_to_num(want))
    near(got, want, err + HALF[out] * 1.01 * np.abs(want) + float(torch.finfo(got.dtype).tiny) * HALF[out])
    if base is not None:
        assert torch.equal(got[ids.cuda() < 0], base.cuda()[ids.cuda() < 0])
    return got


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("ydtype", [None, "float32"])
@pytest.mark.parametrize("n,din,dout,rank,m", [(1, 8, 8, 8, 1), (1, 4096, 1000, 16, 3), (2, 100, 33, 24, 2), (5, 513, 257, 128, 4),
                                               (48, 1024, 300, 16, 32), (64, 72, 520, 40, 7), (65, 72, 520, 40, 7), (100, 64, 64, 8, 1),
                                               (130, 1000, 1343, 16, 50), (300, 513, 100, 32, 3), (257, 256, 301, 64, 9),
                                               (80, 2048, 96, 128, 5), (1000, 96, 160, 16, 200), (2100, 512, 128, 48, 6)])
def test_adapters(jarq, dtype, ydtype, n, din, dout, rank, m):
    rng = np.random.default_rng(n + din + rank)
    for order in ("any", "runs"):
        args = inputs(rng, n, din, dout, rank, m, dtype, ydtype, order)
        check(jarq, *args)
    X, A, B, ids, scale, _ = args
    check(jarq, X, A, B, ids, None, None, dtype=ydtype)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("n", [3, 90])
@pytest.mark.parametrize("px,py,ox,oy", [(101, 203, 0, 0), (104, 208, 8, 8), (112, 209, 1, 3)])
def test_strides_alignment_and_in_place(jarq, dtype, n, px, py, ox, oy):
    rng = np.random.default_rng(px)
    X, A, B, ids, scale, base = inputs(rng, n, 101, 203, 16, 4, dtype)
    x, y = device(X, px, ox), device(base, py, oy)
    a = torch.empty(A.numel() + 1, dtype=A.dtype, device="cuda")[1:].view(A.shape).copy_(A)
    b = torch.empty(B.numel() + 1, dtype=B.dtype, device="cuda")[1:].view(B.shape).copy_(B)
    flat = y._base
    gaps = torch.ones_like(flat, dtype=torch.bool)
    torch.as_strided(gaps, y.shape, y.stride(), y.storage_offset()).fill_(False)
    got = check(jarq, X, A, B, ids, scale, base, (x, a, b, ids.cuda(), scale.cuda(), y), out=y)
    assert got.data_ptr() == y.data_ptr() and flat[gaps].isnan().all()


@pytest.mark.parametrize("n", [4, 40, 200])
def test_tokens_without_an_adapter_and_of_one_that_is_not_there(jarq, n):
    rng = np.random.default_rng(n)
    X, A, B, ids, scale, base = inputs(rng, n, 64, 96, 16, 3, "float16")
    ids[1], ids[2], ids[3] = -7, 3, 2 ** 31 - 1
    got = check(jarq, X, A, B, ids, scale, base)
    assert got[2].isnan().all() and got[3].isnan().all()
    none = torch.full((n,), -1, dtype=torch.int32)
    assert torch.equal(check(jarq, X, A, B, none, scale, base), base.cuda())
    assert (check(jarq, X, A, B, none, scale, None) == 0).all()
    # no adapters at all
    got = jarq.apply_adapters(X.cuda(), A[:0].cuda(), B[:0].cuda(), none.cuda(), base=base.cuda())
    assert torch.equal(got, base.cuda())


@pytest.mark.parametrize("n", [6, 200])
def test_values_that_are_not_finite_stay_with_their_tokens(jarq, n):
    rng = np.random.default_rng(n)
    X, A, B, ids, scale, base = inputs(rng, n, 64, 96, 16, 4, "bfloat16")
    ids[:] = torch.as_tensor(rng.integers(0, 3, n).astype(np.int32))
    ids[5] = 3
    X[4, 7] = float("nan")
    A[3, 1, 2] = float("nan")
    B[3, :, 0] = float("inf")
    got = jarq.apply_adapters(X.cuda(), A.cuda(), B.cuda(), ids.cuda(), scale=scale.cuda(), base=base.cuda())
    bad = got.isnan().any(1).nonzero().flatten().tolist()
    assert bad == [4, 5]
    keep = [r for r in range(n) if r not in (4, 5)]
    want = O.apply_adapters(f64(X[keep]), f64(A[:3]), f64(B[:3]), ids[keep].numpy(), f64(scale), f64(base[keep]))
    near(got[keep], want, HALF["bfloat16"] * 1.01 * np.abs(want) + 1e-3)


@pytest.mark.parametrize("size", [1e-4, 300.0])
@pytest.mark.parametrize("n", [3, 100])
def test_float16_sums_past_its_range(jarq, size, n):
    """A x far above and below float16's numbers, expanded by small and large B."""
    rng = np.random.default_rng(n)
    X, A, B, ids, scale, base = inputs(rng, n, 512, 64, 16, 2, "float16", "float32")
    X, A = (X.float() * size).half(), (A.float() * size * 20).half()
    B = (B.float() / size).half()
    check(jarq, X, A, B, ids, scale, base * size)


def test_a_token_does_not_depend_on_the_others(jarq):
    rng = np.random.default_rng(9)
    for n in (40, 400):
        X, A, B, ids, scale, base = (t.cuda() for t in inputs(rng, n, 256, 192, 16, 5, "bfloat16"))
        want = jarq.apply_adapters(X, A, B, ids, scale=scale, base=base)
        for seed in range(3):
            p = torch.randperm(n, generator=torch.Generator(device="cuda").manual_seed(seed), device="cuda")
            got = jarq.apply_adapters(X[p].contiguous(), A, B, ids[p].contiguous(), scale=scale, base=base[p].contiguous())
            assert torch.equal(got, want[p])


def test_beside_an_integer_layer_after_a_norm(jarq):
    """The operators as they are used together: norm with the residual and 8-bit rows, a
    quantized projection and the adapters beside it, in a graph on a stream of its own."""
    rng = np.random.default_rng(10)
    n, din, dout = 70, 256, 384
    X, A, B, ids, scale, _ = (t.cuda() for t in inputs(rng, n, din, dout, 16, 3, "float16"))
    res, gain = randn(rng, n, din, "float16").cuda(), randn(rng, 1, din, "float16")[0].cuda()
    C = torch.as_tensor(rng.integers(-7, 8, (dout, din)).astype(np.int8)).cuda()
    ws = torch.as_tensor(rng.uniform(0.01, 0.02, (dout, 2)).astype(np.float32)).cuda()

    def layer():
        r = jarq.rms_norm(X, gain, residual=res, codes=True)
        y = jarq.integer_product(r.codes, r.scale, C, ws, 128, dtype="float16")
        return r, y.clone(), jarq.apply_adapters(r.y, A, B, ids, scale=scale, base=y, out=y)

    layer()
    stream, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.graph(graph, stream=stream):
        r, y, z = layer()
    for seed in (1, 2):
        X.copy_(randn(np.random.default_rng(seed), n, din, "float16"))
        graph.replay()
        torch.cuda.synchronize()
        e, ey, ez = layer()
        assert torch.equal(e.codes, r.codes) and torch.equal(ey, y) and torch.equal(ez, z)
        # the projection of the norm, in float64, by the integers' half steps
        v = f64(e.codes) * f64(e.scale)[:, None]
        want = (v.reshape(n, 2, 128)[:, None] * (f64(C).reshape(dout, 2, 128) * f64(ws)[:, :, None])).sum((2, 3))
        near(ey, want, 2 ** -11 * 1.01 * np.abs(want) + 1e-4)
        near(f64(e.y), v, (f64(e.scale) * 0.5)[:, None] * 1.001 + 2 ** -11 * 1.01 * np.abs(v))
        check(jarq, e.y.cpu(), A.cpu(), B.cpu(), ids.cpu(), scale.cpu(), ey.cpu())
    assert jarq.async_status() == jarq.JARQ_OK
