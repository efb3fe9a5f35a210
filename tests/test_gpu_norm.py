"""The root-mean-square norm of rows and its gradient on the GPU against the float64
reference: the sum with the residual and the 8-bit integers exactly, the rest within
bounds counted from the float32 operations."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")

pytestmark = [pytest.mark.gpu,
              pytest.mark.skipif(not torch.cuda.is_available(), reason="needs a CUDA GPU")]

from oracle import jarq_tuning as O  # noqa: E402

DT = {"float32": torch.float32, "float16": torch.float16, "bfloat16": torch.bfloat16}
U = 2.0 ** -24
HALF = {t: torch.finfo(d).eps / 2 for t, d in DT.items()}


@pytest.fixture(scope="module")
def jarq():
    from paper_2609_38599_gb300 import jarq as J
    return J


def device(x, pitch=None, offset=0):
    """The matrix x on the GPU, its rows `pitch` apart, NaN between them."""
    n, d = x.shape
    pitch = pitch or d
    flat = torch.full((offset + max(0, n - 1) * pitch + d,), float("nan"), dtype=x.dtype, device="cuda")
    out = torch.as_strided(flat, (n, d), (pitch, 1), offset)
    return out.copy_(x)


def randn(rng, n, d, dtype, scale=1.0):
    return torch.as_tensor((rng.standard_normal((n, d)) * scale).astype(np.float32)).to(DT[dtype])


def f64(x):
    return x.detach().double().cpu().numpy()


def near(got, want, bound):
    """Equal where not finite, else within the bound."""
    got = f64(got) if torch.is_tensor(got) else np.asarray(got)
    fine = np.isfinite(want)
    assert np.array_equal(np.isnan(got), np.isnan(want))
    assert np.array_equal(got[~fine & ~np.isnan(want)], want[~fine & ~np.isnan(want)])
    over = np.abs(np.where(fine, got - np.where(fine, want, 0), 0)) - np.broadcast_to(bound, want.shape)
    assert not (over[fine] > 0).any(), f"{over[fine].max()} over the bound"


def terms(d):
    """Most terms that one thread adds up, and the levels that join threads."""
    return max(32, d / 1024 + 8) + 12


def check(jarq, x, gain, eps=1e-5, residual=None, args=None, **kw):
    """The norm of host rows x; `args`: the same on the device."""
    dtype = str(x.dtype)[6:]
    dx, dr, dg = args or (x.cuda(), None if residual is None else residual.cuda(), None if gain is None else gain.cuda())
    r = jarq.rms_norm(dx, dg, eps=eps, residual=dr, codes=True, **kw)
    h = x if residual is None else (x.float() + residual.float()).to(x.dtype)
    assert torch.equal(torch.nan_to_num(r.h.cpu().float(), 7.0, 8.0, 9.0), torch.nan_to_num(h.float(), 7.0, 8.0, 9.0))
    ref = O.rms_norm(f64(h), None if gain is None else f64(gain), eps)
    # the sum of squares, of which half reaches rstd; the mean, eps, root and quotient
    rel = (0.5 * terms(x.shape[1]) + 4) * U * 1.01
    near(r.rstd, ref["rstd"], rel * np.abs(ref["rstd"]) + 1e-45)
    assert np.array_equal(r.codes.cpu().numpy(), ref["codes"])
    near(r.scale, ref["scale"], (rel + 2 * U) * np.abs(ref["scale"]) + 1e-45)
    if r.y is not None:
        # v and v rstd rounded to float32, then to the type (absolutely below its normal numbers)
        tiny = float(torch.finfo(x.dtype).tiny) * HALF[dtype]
        near(r.y, ref["y"], (rel + 2 * U + HALF[dtype]) * 1.01 * np.abs(ref["y"]) + tiny)
    return r, ref


@pytest.mark.parametrize("dtype", list(DT))
@pytest.mark.parametrize("n,d", [(1, 1), (3, 2), (1, 7), (2, 33), (9, 129), (1, 4096), (5, 1000), (160, 1001), (200, 4096),
                                 (3, 14336), (300, 520), (155, 8200), (154, 16384), (2, 20000), (160, 40003)])
def test_norm(jarq, dtype, n, d):
    rng = np.random.default_rng(n + d)
    gain = randn(rng, 1, d, dtype)[0]
    check(jarq, randn(rng, n, d, dtype, 3.0), gain)
    check(jarq, randn(rng, n, d, dtype), gain.float(), residual=randn(rng, n, d, dtype, 2.0))
    check(jarq, randn(rng, n, d, dtype), None, residual=randn(rng, n, d, dtype))


@pytest.mark.parametrize("dtype", list(DT))
@pytest.mark.parametrize("pitch,offset", [(None, 1), (1003, 0), (1010, 3), (1024, 8)])
@pytest.mark.parametrize("n", [5, 170])
def test_strides_and_alignment(jarq, dtype, pitch, offset, n):
    rng = np.random.default_rng(offset)
    x, r, g = randn(rng, n, 1001, dtype), randn(rng, n, 1001, dtype), randn(rng, 1, 1001, dtype)[0]
    dr = device(r, pitch, offset)
    base = dr._base if dr._base is not None else dr
    gaps = torch.ones_like(base, dtype=torch.bool)
    torch.as_strided(gaps, dr.shape, dr.stride(), dr.storage_offset()).fill_(False)
    args = (device(x, pitch, offset), dr, device(g[None], None, offset)[0])
    check(jarq, x, g, residual=r, args=args, h=dr)           # the residual stream in place
    assert base[gaps].isnan().all()                          # and nothing between its rows


@pytest.mark.parametrize("dtype", list(DT))
def test_zero_tiny_and_huge_rows(jarq, dtype):
    rng = np.random.default_rng(4)
    d = 300
    x = randn(rng, 8, d, dtype)
    x[0] = 0
    x[1] = float(torch.finfo(DT[dtype]).tiny)
    x[2] = float(torch.finfo(DT[dtype]).max)
    x[3, 5] = float(torch.finfo(DT[dtype]).min)
    x[4] = 1e-30 if dtype != "float16" else 6e-8
    gain = randn(rng, 1, d, dtype)[0]
    gain[:] = 0.5
    r, ref = check(jarq, x, gain, eps=1e-6)
    assert (r.codes[0] == 0).all() and r.scale[0] == 0 and (r.y[0] == 0).all()
    assert r.y[2].float().sub(0.5).abs().max() < 0.01         # squares past float32's range


@pytest.mark.parametrize("dtype", list(DT))
@pytest.mark.parametrize("value", [float("nan"), float("inf"), -float("inf")])
@pytest.mark.parametrize("n,d", [(3, 100), (160, 4096)])
def test_rows_that_are_not_finite_stay_alone(jarq, dtype, value, n, d):
    rng = np.random.default_rng(5)
    x = randn(rng, n, d, dtype)
    x[1, d // 2] = value
    r, ref = check(jarq, x, None)
    assert r.scale[1].isnan() and (r.codes[1] == 0).all() and not r.scale[0].isnan() and not r.y[2].isnan().any()


def check_grad(jarq, h, gain, rstd, dy, dh, args=None, **kw):
    dtype = str(h.dtype)[6:]
    dx, dgain = jarq.rms_norm_grad(*(args or [None if x is None else x.cuda() for x in (h, gain, rstd, dy, dh)]), **kw)
    g = None if gain is None else f64(gain)
    H, Y, r = f64(h), f64(dy), f64(rstd)
    wx, wg = O.rms_norm_grad(H, g, r, Y, None if dh is None else f64(dh))
    n, d = H.shape
    u = np.abs(Y * (1.0 if g is None else g))
    mean = (u * np.abs(H)).sum(1) / d
    # u and each product rounded, the sum's terms, then four operations to rstd^2 mean
    along = (terms(d) + 2 + 5) * U * r ** 2 * mean
    err = r[:, None] * (3 * U * u + np.abs(H) * (along + 2 * U * r ** 2 * mean)[:, None])
    err += 2 * U * (np.abs(wx) + (0 if dh is None else np.abs(f64(dh))))
    if dx is not None:
        near(dx, wx, 1.01 * err + HALF[dtype] * 1.01 * np.abs(wx) + float(torch.finfo(h.dtype).tiny) * HALF[dtype])
    if dgain is not None:
        # rows that one block adds up, blocks that one warp does, and the warps; two products a term
        count = n / 608 + 1 + n / 8 / 32 * (d > 8192) + 19 + 8 + 5 + 2
        near(dgain, wg, count * U * 1.01 * np.abs(Y * H * r[:, None]).sum(0) + 1e-45)
    return dx, dgain


def _grad_inputs(rng, n, d, dtype):
    h = randn(rng, n, d, dtype, 2.0)
    rstd = torch.as_tensor(O.rms_norm(f64(h), None, 1e-5)["rstd"]).float()
    return h, randn(rng, 1, d, dtype)[0], rstd, randn(rng, n, d, dtype, 0.1), randn(rng, n, d, dtype, 0.1)


@pytest.mark.parametrize("dtype", list(DT))
@pytest.mark.parametrize("n,d", [(1, 1), (2, 3), (7, 129), (48, 1000), (700, 257), (1300, 64), (65, 4096), (3, 14336), (2, 20000),
                                 (50, 40003)])
def test_gradient(jarq, dtype, n, d):
    rng = np.random.default_rng(n * d)
    h, gain, rstd, dy, dh = _grad_inputs(rng, n, d, dtype)
    check_grad(jarq, h, gain, rstd, dy, dh)
    check_grad(jarq, h, gain.float(), rstd, dy, None)
    assert check_grad(jarq, h, None, rstd, dy, None, gains=False)[1] is None
    assert check_grad(jarq, h, gain, rstd, dy, None, rows=False)[0] is None


@pytest.mark.parametrize("dtype", list(DT))
@pytest.mark.parametrize("pitch,offset", [(1003, 0), (1010, 3), (1024, 8)])
def test_gradient_strides(jarq, dtype, pitch, offset):
    rng = np.random.default_rng(offset)
    h, gain, rstd, dy, dh = _grad_inputs(rng, 13, 1001, dtype)
    args = (device(h, pitch, offset), gain.cuda(), rstd.cuda(), device(dy, pitch, offset), device(dh, pitch, offset))
    check_grad(jarq, h, gain, rstd, dy, dh, args=args)


@pytest.mark.parametrize("d", [512, 20000])
@pytest.mark.parametrize("which", ["dy", "dh"])
def test_gradient_in_place(jarq, d, which):
    """dX over the gradient that came in, also where the gains' sums read it apart."""
    rng = np.random.default_rng(d)
    h, gain, rstd, dy, dh = _grad_inputs(rng, 40, d, "float32")
    want, wg = check_grad(jarq, h, gain, rstd, dy, dh)
    y, s = dy.cuda(), dh.cuda()
    out = y if which == "dy" else s
    dx, dgain = jarq.rms_norm_grad(h.cuda(), gain.cuda(), rstd.cuda(), y, dh=s, out=out)
    assert dx.data_ptr() == out.data_ptr() and torch.equal(dx, want) and torch.equal(dgain, wg)


def test_gradient_against_differences(jarq):
    """The gradient of the library's own norm, by differences of its float32 rows."""
    rng = np.random.default_rng(9)
    n, d, step = 3, 40, 2.0 ** -6
    h, gain, _, dy, _ = _grad_inputs(rng, n, d, "float32")
    r = jarq.rms_norm(h.cuda(), gain.cuda(), eps=1e-3)
    dx, dgain = jarq.rms_norm_grad(h.cuda(), gain.cuda(), r.rstd, dy.cuda())
    total = lambda x, g: (f64(jarq.rms_norm(x.cuda(), g.cuda(), eps=1e-3).y) * f64(dy)).sum()
    for r_, k in ((0, 0), (1, 17), (2, 39)):
        hi, lo = h.clone(), h.clone()
        hi[r_, k] += step
        lo[r_, k] -= step
        # third derivatives (below 30 |dy| for rows of unit size) times step^2 / 6, and the rows' rounding
        assert abs((total(hi, gain) - total(lo, gain)) / float(hi[r_, k] - lo[r_, k]) - dx[r_, k].item()) < 1e-3
    hi = gain.clone()
    hi[5] += 0.5
    assert abs((total(h, hi) - total(h, gain)) / 0.5 - dgain[5].item()) < 1e-4


def test_no_rows(jarq):
    x = torch.zeros(0, 64, device="cuda")
    r = jarq.rms_norm(x, codes=True)
    assert r.y.shape == (0, 64) and r.codes.shape == (0, 64)
    dx, dgain = jarq.rms_norm_grad(x, None, r.rstd, x)
    assert dx.shape == (0, 64) and (dgain == 0).all()


def test_same_bits_whatever_the_batch_and_again(jarq):
    """A row's outputs do not depend on the other rows where the threads that share
    it are the same; the gains' sums are always added in the same order."""
    rng = np.random.default_rng(11)
    x, r = randn(rng, 400, 4096, "bfloat16").cuda(), randn(rng, 400, 4096, "bfloat16").cuda()
    gain = randn(rng, 1, 4096, "bfloat16")[0].cuda()
    a = jarq.rms_norm(x, gain, residual=r, codes=True)
    for at in (slice(100, 300), slice(7, 8), slice(300, 400)):
        b = jarq.rms_norm(x[at], gain, residual=r[at], codes=True)
        for name in ("h", "y", "codes", "scale", "rstd"):
            assert torch.equal(getattr(a, name)[at], getattr(b, name))
        for dh in (r, None):
            full = jarq.rms_norm_grad(a.h, gain, a.rstd, x, dh=dh)[0]
            assert torch.equal(full[at], jarq.rms_norm_grad(b.h, gain, b.rstd, x[at], dh=None if dh is None else dh[at])[0])
    one = jarq.rms_norm_grad(a.h, gain, a.rstd, x, dh=r)
    for _ in range(3):
        two = jarq.rms_norm_grad(a.h, gain, a.rstd, x, dh=r)
        assert torch.equal(one[0], two[0]) and torch.equal(one[1], two[1])


def test_graph_and_other_stream(jarq):
    rng = np.random.default_rng(12)
    x, res, gain = randn(rng, 64, 1024, "float16").cuda(), randn(rng, 64, 1024, "float16").cuda(), None
    dy = randn(rng, 64, 1024, "float16").cuda()
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.stream(stream):
        with torch.cuda.graph(graph, stream=stream):
            r = jarq.rms_norm(x, gain, residual=res, codes=True)
            dx, dgain = jarq.rms_norm_grad(r.h, gain, r.rstd, dy)
    for seed in (1, 2):
        x.copy_(randn(np.random.default_rng(seed), 64, 1024, "float16"))
        graph.replay()
        want = jarq.rms_norm(x, gain, residual=res, codes=True)
        assert torch.equal(want.y, r.y) and torch.equal(want.codes, r.codes)
        wx, wg = jarq.rms_norm_grad(want.h, gain, want.rstd, dy)
        assert torch.equal(wx, dx) and torch.equal(wg, dgain)
