"""Linear layers in 8-bit integers on the GPU against the float64 reference:
row quantization (bit-exact), the integer codes of a refined layer (exact) and
the product with token, channel and group scales (within derived bounds)."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")

pytestmark = [pytest.mark.gpu,
              pytest.mark.skipif(not torch.cuda.is_available(), reason="needs a CUDA GPU")]

from oracle import jarq_inference as O  # noqa: E402

DT = {"float32": torch.float32, "float16": torch.float16, "bfloat16": torch.bfloat16}
# unit roundoff and half the smallest subnormal step of the output types
UNIT = {"float32": (2.0 ** -24, 2.0 ** -150), "float16": (2.0 ** -11, 2.0 ** -25), "bfloat16": (2.0 ** -8, 2.0 ** -134)}


@pytest.fixture(scope="module")
def jarq():
    from paper_2609_38599_gb300 import jarq as J
    return J


def _rows(a, pitch=None, offset=0):
    """Device copy of a matrix with rows `pitch` elements apart, `offset`
    elements into its storage."""
    t = torch.as_tensor(a)
    n, d = t.shape
    pitch = pitch or d
    flat = torch.zeros(offset + max(0, n - 1) * pitch + d, dtype=t.dtype, device="cuda")
    v = torch.as_strided(flat, (n, d), (pitch, 1), offset)
    v.copy_(t)
    return v


# ---------------------------------------------------------------- rows to integers

@pytest.mark.parametrize("dtype", list(DT))
@pytest.mark.parametrize("n,d,pitch,offset", [(1, 1, None, 0), (3, 7, None, 0), (5, 64, None, 1), (9, 255, 300, 3),
                                              (33, 1001, None, 0), (17, 1792, None, 0), (2, 4096, 4100, 5),
                                              (7, 14337, None, 0), (2, 40000, None, 2)])
def test_quantize_rows_bit_exact(jarq, dtype, n, d, pitch, offset):
    rng = np.random.default_rng(n * d)
    X = torch.as_tensor((rng.standard_normal((n, d)) * np.exp(rng.standard_normal((n, 1)) * 3)).astype(np.float32)).to(DT[dtype])
    x = _rows(X, pitch, offset)
    q, s = jarq.quantize_rows(x)
    q0, s0 = O.quantize_rows(X.float().numpy())
    assert np.array_equal(s.cpu().numpy(), s0)
    assert np.array_equal(q.cpu().numpy(), q0)


def test_quantize_rows_special_rows(jarq):
    X = torch.zeros(6, 100)
    X[1, 3] = float("inf")
    X[2, 99] = float("nan")
    X[3, 0] = 2.0 ** -126
    X[4, 5] = torch.finfo(torch.float32).max
    X[5, :] = 2.0 ** -120
    q, s = jarq.quantize_rows(X.cuda())
    q0, s0 = O.quantize_rows(X.numpy())
    assert np.array_equal(s.cpu().numpy(), s0, equal_nan=True) and np.array_equal(q.cpu().numpy(), q0)
    assert q0[5].min() == 127 and q0[4, 5] == 127 and (q0[:4] == 0).all()


# ---------------------------------------------------------------- codes of a refined layer

@pytest.mark.parametrize("dout,din,g,bits,offset", [(5, 192, 64, 3, 0), (130, 384, 128, 7, 0), (3, 96, 32, 4, 1), (7, 30, 10, 1, 0)])
def test_integer_codes_exact(jarq, dout, din, g, bits, offset):
    rng = np.random.default_rng(din)
    Q = rng.integers(0, 1 << bits, (dout, din), dtype=np.uint8)
    Z = rng.integers(0, 1 << bits, (dout, din // g)).astype(np.int32)
    q = torch.zeros(offset + dout * din, dtype=torch.uint8, device="cuda")[offset:].view(dout, din)
    q.copy_(torch.as_tensor(Q))
    C = jarq.integer_codes(q, torch.as_tensor(Z).cuda(), g, bits)
    assert np.array_equal(C.cpu().numpy(), Q.astype(np.int64) - np.repeat(Z, g, axis=1))


def test_integer_codes_refuses_bad_codes(jarq):
    Q = torch.full((4, 64), 8, dtype=torch.uint8, device="cuda")
    Z = torch.zeros(4, 1, dtype=torch.int32, device="cuda")
    with pytest.raises(jarq.JarqError) as e:
        jarq.integer_codes(Q, Z, 64, 3)
    assert e.value.status == jarq.JARQ_ERR_ARG


# ---------------------------------------------------------------- the product

def _codes(rng, n, d, most=127):
    return rng.integers(-most, most + 1, (n, d)).astype(np.int8)


def _check(y, X, xs, C, ws, g, bias, dtype):
    """Every output within the bound of the operator's roundings.  G = 1: the
    exact sum, its product with the channel's scale and the last
    multiply-add are each rounded to float32, then to the output type.  Groups:
    one rounding a term, on partial sums of at most the terms' magnitudes, and
    as many again where parts of K are joined (at most 8)."""
    Y, M = O.integer_product(X, xs, C, ws, g, bias)
    u, tiny = UNIT[dtype]
    terms = 3 if not g else X.shape[1] // g + 3 + 8
    B = 0 if bias is None else np.abs(bias)
    bound = terms * 2.0 ** -24 * (M + B) * 1.01 + u * np.abs(Y) * 1.01 + tiny + 2.0 ** -149
    err = np.abs(y.double().cpu().numpy() - Y)
    assert err.shape == bound.shape and (err <= bound).all(), float((err / bound).max())


SHAPES = [(1, 1, 1), (1, 64, 17), (2, 1000, 130), (3, 4096, 512), (5, 77, 33), (8, 2048, 1024), (9, 1344, 300),
          (16, 512, 257), (17, 1001, 64), (33, 11008, 200), (64, 4096, 640), (65, 130, 1000), (100, 640, 128),
          (129, 256, 129), (200, 1088, 384), (257, 3000, 511), (300, 4096, 1500), (600, 448, 260), (1025, 129, 1029)]


@pytest.mark.parametrize("n,din,dout", SHAPES)
def test_product_one_scale_a_channel(jarq, n, din, dout):
    rng = np.random.default_rng(n + din + dout)
    X, C = _codes(rng, n, din), _codes(rng, dout, din)
    xs, ws = rng.random(n).astype(np.float32) * 0.1, (rng.standard_normal(dout) * 0.01).astype(np.float32)
    bias = rng.standard_normal(dout).astype(np.float32) if n % 2 else None
    dtype = list(DT)[(n + dout) % 3]
    t = lambda a: None if a is None else torch.as_tensor(a).cuda()
    y = jarq.integer_product(t(X), t(xs), t(C), t(ws), bias=t(bias), dtype=dtype)
    assert y.dtype == DT[dtype]
    _check(y, X, xs, C, ws, 0, bias, dtype)


@pytest.mark.parametrize("g", [64, 128])
@pytest.mark.parametrize("n,din,dout", [(1, 128, 5), (1, 4096, 700), (4, 1408, 130), (7, 384, 64), (11, 11008, 129),
                                        (40, 896, 300), (64, 4096, 256), (130, 1280, 513), (300, 2304, 640),
                                        (515, 256, 1100), (1030, 640, 400)])
def test_product_with_group_scales(jarq, n, din, dout, g):
    rng = np.random.default_rng(n * din + dout + g)
    X, C = _codes(rng, n, din), _codes(rng, dout, din, 15)
    xs, ws = rng.random(n).astype(np.float32), (rng.standard_normal((dout, din // g)) * 0.01).astype(np.float32)
    bias = rng.standard_normal(dout).astype(np.float32) if dout % 2 else None
    dtype = list(DT)[(n + dout) % 3]
    t = lambda a: None if a is None else torch.as_tensor(a).cuda()
    y = jarq.integer_product(t(X), t(xs), t(C), t(ws), g, t(bias), dtype)
    _check(y, X, xs, C, ws, g, bias, dtype)


@pytest.mark.parametrize("n", [1, 6, 20, 70, 300])
@pytest.mark.parametrize("xp,xo,cp,co", [(1001, 0, 1001, 0), (1040, 0, 1056, 0), (1041, 3, 1008, 0), (1008, 16, 1003, 5)])
def test_product_strides_and_alignment(jarq, n, xp, xo, cp, co):
    """Rows at any pitch and offset, an output that is a slice; nothing is read
    or written between the rows."""
    din, dout = 1001, 150
    rng = np.random.default_rng(n + xp)
    X, C = _codes(rng, n, din), _codes(rng, dout, din)
    xs, ws = rng.random(n).astype(np.float32), rng.random(dout).astype(np.float32)
    out = torch.full((n, dout + 7), 3.0, device="cuda")
    y = jarq.integer_product(_rows(X, xp, xo), torch.as_tensor(xs).cuda(), _rows(C, cp, co), torch.as_tensor(ws).cuda(),
                             dtype="float32", out=out[:, 3:3 + dout])
    _check(y, X, xs, C, ws, 0, None, "float32")
    assert (out[:, :3] == 3).all() and (out[:, 3 + dout:] == 3).all()


@pytest.mark.parametrize("n", [1, 8, 64, 260])
@pytest.mark.parametrize("a,b", [(-128, -128), (-128, 127), (127, 127)])
def test_largest_sums_are_exact(jarq, n, a, b):
    """Codes of the largest magnitude over the longest rows: the sum is exact,
    so one scale of a power of two gives the rounded integer."""
    din, dout = 65536, 130
    X = torch.full((n, din), a, dtype=torch.int8, device="cuda")
    C = torch.full((dout, din), b, dtype=torch.int8, device="cuda")
    X[:, 5] = 1
    C[:, 7] = 3
    want = a * b * (din - 2) + b + 3 * a
    y = jarq.integer_product(X, torch.ones(n, device="cuda"), C, torch.ones(dout, device="cuda"), dtype="float32")
    assert (y == torch.tensor(float(np.float32(want)), device="cuda")).all()


@pytest.mark.parametrize("n", [2, 12, 100, 400])
def test_result_does_not_depend_on_the_batch(jarq, n):
    """One scale a channel: the integer sums are exact, so a token's outputs are
    the same bits alone and in any batch."""
    rng = np.random.default_rng(n)
    t = lambda a: torch.as_tensor(a).cuda()
    X, C = t(_codes(rng, n, 2080)), t(_codes(rng, 333, 2080))
    xs, ws = t(rng.random(n).astype(np.float32)), t(rng.random(333).astype(np.float32))
    whole = jarq.integer_product(X, xs, C, ws, dtype="float32")
    for i in (0, n // 2, n - 1):
        assert torch.equal(whole[i:i + 1], jarq.integer_product(X[i:i + 1], xs[i:i + 1], C, ws, dtype="float32"))


def test_scales_of_nan_and_zero(jarq):
    rng = np.random.default_rng(0)
    X, C = _codes(rng, 20, 256), _codes(rng, 40, 256)
    t = lambda a: torch.as_tensor(a).cuda()
    xs = torch.ones(20, device="cuda")
    xs[3], xs[4] = float("nan"), 0.0
    y = jarq.integer_product(t(X), xs, t(C), torch.ones(40, device="cuda"), bias=torch.ones(40, device="cuda"), dtype="float32")
    assert torch.isnan(y[3]).all() and (y[4] == 1).all() and torch.isfinite(y[5:]).all()


@pytest.mark.parametrize("n", [2, 50])
def test_rows_past_two_to_the_31(jarq, n):
    """Weights whose last rows lie more than 2^31 bytes into their storage."""
    din, dout, pitch = 64, 1100, 1 << 21
    rng = np.random.default_rng(5)
    X, C = _codes(rng, n, din), _codes(rng, dout, din)
    c = _rows(C, pitch)
    xs, ws = np.ones(n, np.float32), np.ones(dout, np.float32)
    y = jarq.integer_product(torch.as_tensor(X).cuda(), torch.as_tensor(xs).cuda(), c, torch.as_tensor(ws).cuda(), dtype="float32")
    _check(y, X, xs, C, ws, 0, None, "float32")


def test_empty_batch(jarq):
    e = lambda *s, dtype=torch.float32: torch.zeros(*s, dtype=dtype, device="cuda")
    y = jarq.integer_product(e(0, 64, dtype=torch.int8), e(0), e(5, 64, dtype=torch.int8), e(5))
    assert y.shape == (0, 5)
    assert jarq.integer_linear(e(0, 64), e(5, 64, dtype=torch.int8), e(5)).shape == (0, 5)
    assert jarq.quantize_rows(e(0, 64))[0].shape == (0, 64)


@pytest.mark.parametrize("xdtype", list(DT))
@pytest.mark.parametrize("n,din,dout,g", [(1, 4096, 300, 0), (1, 768, 130, 128), (3, 1001, 77, 0), (4, 11008, 64, 64), (50, 1024, 300, 64), (300, 999, 200, 0)])
def test_linear_is_quantization_then_product(jarq, xdtype, n, din, dout, g):
    """integer_linear gives the bits of its two halves."""
    rng = np.random.default_rng(din)
    t = lambda a: torch.as_tensor(a).cuda()
    X = t((rng.standard_normal((n, din)) * 3).astype(np.float32)).to(DT[xdtype])
    if n > 2:
        X[1] = 0
    C, ws = t(_codes(rng, dout, din, 7)), t(rng.standard_normal((dout, din // g if g else 1)).astype(np.float32))
    bias = t(rng.standard_normal(dout).astype(np.float32))
    q, xs = jarq.quantize_rows(X)
    want = jarq.integer_product(q, xs, C, ws, g, bias, "float32")
    y = jarq.integer_linear(X, C, ws, g, bias, "float32")
    Y, M = O.integer_product(q.cpu().numpy(), xs.cpu().numpy(), C.cpu().numpy(), ws.cpu().numpy(), g, bias.cpu().numpy())
    assert (np.abs(y.double().cpu().numpy() - Y) <= (din // (g or din) + 12) * 2.0 ** -24 * 1.02 * (M + np.abs(Y) + 5)).all()
    if not g:
        assert torch.equal(y, want)
    assert jarq.integer_linear(X, C, ws, g, bias).dtype == DT[xdtype]


def test_other_stream_and_graph(jarq):
    """Work goes to torch's current stream only, and a call can be captured."""
    rng = np.random.default_rng(3)
    t = lambda a: torch.as_tensor(a).cuda()
    for n in (1, 6, 40, 300):
        X = t(rng.standard_normal((n, 1024)).astype(np.float32))
        C, ws = t(_codes(rng, 500, 1024)), t(rng.random(500).astype(np.float32))
        want = jarq.integer_linear(X, C, ws)
        s = torch.cuda.Stream()
        s.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(s):
            other = jarq.integer_linear(X, C, ws)
        s.synchronize()
        assert torch.equal(want, other)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            y = jarq.integer_linear(X, C, ws)
        X.copy_(X.flip(0) * 2)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(y, jarq.integer_linear(X, C, ws))
    assert jarq.async_status() == jarq.JARQ_OK


def test_a_refined_layer_runs_in_integers(jarq):
    """The scales and codes of a refined layer are the operator's weights as
    they are: its product is that of the dequantized weights."""
    from synth import tiny_layer
    lay = tiny_layer()
    t = lambda a: torch.as_tensor(a).cuda()
    W, S, Q, Z = t(lay.W), t(lay.S0).clone(), t(lay.Q0).clone(), t(lay.Z)
    hess = jarq.prepare(t(lay.H), lay.g)
    jarq.refine(hess, W, S, Q, Z, lay.bits, max_iters=2)
    hess.close()
    C = jarq.integer_codes(Q, Z, lay.g, lay.bits)
    X = torch.randn(40, lay.din, device="cuda", generator=torch.Generator("cuda").manual_seed(1))
    q, xs = jarq.quantize_rows(X)
    y = jarq.integer_linear(X, C, S, lay.g, dtype="float32").double()
    what = jarq.dequantize(S, Q, Z, lay.g, lay.bits, "float32").double()
    want = (q.double() * xs[:, None].double()) @ what.T
    # one float32 rounding a weight there, one a term here: G + 12 units
    bound = (lay.din // lay.g + 12) * 2.0 ** -24 * ((q.double().abs() * xs[:, None].double()) @ what.abs().T) + 1e-30
    assert ((y - want).abs() <= bound).all()


def test_refusals(jarq):
    dev = dict(device="cuda")
    X, C = torch.zeros(4, 128, dtype=torch.int8, **dev), torch.zeros(8, 128, dtype=torch.int8, **dev)
    xs, ws = torch.zeros(4, **dev), torch.zeros(8, **dev)
    for bad in (lambda: jarq.integer_product(X.cpu(), xs, C, ws), lambda: jarq.integer_product(X, xs[:3], C, ws),
                lambda: jarq.integer_product(X.float(), xs, C, ws), lambda: jarq.integer_product(X, xs, C, ws, 64),
                lambda: jarq.integer_product(X.t(), xs, C, ws), lambda: jarq.integer_linear(X, C, ws),
                lambda: jarq.quantize_rows(X), lambda: jarq.integer_product(X, xs, C, ws, bias=xs)):
        with pytest.raises(TypeError):
            bad()
    with pytest.raises(ValueError):
        jarq.integer_product(X[:, :64], xs, C, ws)
    with pytest.raises(jarq.JarqError) as e:        # a group size that the kernels do not have
        jarq.integer_product(X, xs, C, torch.zeros(8, 4, **dev), 32)
    assert e.value.status == jarq.JARQ_ERR_ARG
    with pytest.raises(jarq.JarqError) as e:        # one row of storage for all tokens
        jarq.integer_product(X[:1].expand(4, 128), xs, C, ws)
    assert e.value.status == jarq.JARQ_ERR_ARG
    # the C entry: host pointers, too small a workspace, a misaligned output
    lib, p = jarq.library(), lambda t: t.data_ptr()
    f, out = torch.zeros(4, 128, **dev), torch.zeros(4 * 8 + 1, **dev)
    work = torch.zeros(lib.jarq_integer_linear_workspace(4, 128), dtype=torch.uint8, **dev)
    def linear(x=p(f), y=p(out), w=p(work), size=work.numel()):
        return lib.jarq_integer_linear(x, 0, 128, p(C), 128, p(ws), 0, None, 4, 8, 128, 0, y, 8, w, size, None)
    assert linear() == jarq.JARQ_OK
    for got in (linear(x=f.cpu().data_ptr()), linear(size=work.numel() - 1), linear(y=p(out) + 2), linear(w=None),
                linear(w=p(work) + 4), linear(x=None)):
        assert got == jarq.JARQ_ERR_ARG
    torch.cuda.synchronize()


def test_a_wait_that_gives_up_is_reported_once(jarq):
    """The product's form whose issuer stops early: its waits run out, the call
    reports it, and the next products are right."""
    assert jarq.async_status() == jarq.JARQ_OK
    assert jarq.selftest_stalled_kernel("integer_product") == jarq.JARQ_ERR_TIMEOUT
    assert jarq.async_status() == jarq.JARQ_OK
    rng = np.random.default_rng(8)
    X, C = _codes(rng, 300, 1024), _codes(rng, 700, 1024)
    xs, ws = rng.random(300).astype(np.float32), rng.random(700).astype(np.float32)
    t = lambda a: torch.as_tensor(a).cuda()
    _check(jarq.integer_product(t(X), t(xs), t(C), t(ws), dtype="float32"), X, xs, C, ws, 0, None, "float32")


# every form of the product: tiles of 32 to 256 tokens, K split over a cluster or
# not, one or several tiles a cluster, rows on 16-byte boundaries or not
@pytest.mark.parametrize("pitch", [0, 1])
@pytest.mark.parametrize("g", [0, 64, 128])
@pytest.mark.parametrize("n,din,dout", [(3, 512, 300), (20, 2048, 140), (30, 256, 20000), (50, 1152, 200), (60, 384, 20500),
                                        (110, 2560, 300), (128, 256, 20000), (250, 4096, 260), (700, 384, 2900),
                                        (1500, 256, 5000)])
def test_linear_in_every_form(jarq, n, din, dout, g, pitch):
    rng = np.random.default_rng(n + g)
    C = _codes(rng, dout, din, 15)
    X = torch.as_tensor((rng.standard_normal((n, din)) * 2).astype(np.float32)).cuda().half()
    ws = rng.standard_normal((dout, din // g if g else 1)).astype(np.float32)
    c, w = _rows(C, din + 16 * (1 - pitch) + pitch), torch.as_tensor(ws).cuda()
    q, xs = jarq.quantize_rows(X)
    y = jarq.integer_linear(X, c, w, g, dtype="float32")
    # in 64 bits on the device; the bound of _check
    x64, c64 = q.double() * xs.double()[:, None], c.double()
    w64 = w.double().repeat_interleave(g or din, dim=1)
    want = x64 @ (c64 * w64).T
    if g:
        size = sum((x64[:, i * g:(i + 1) * g] @ (c64 * w64)[:, i * g:(i + 1) * g].T).abs() for i in range(din // g))
    else:
        size = want.abs()
    terms = din // g + 11 if g else 3
    assert ((y.double() - want).abs() <= terms * 2.0 ** -24 * 1.01 * size + 2.0 ** -24 * want.abs() + 1e-12 * x64.abs().max() * din).all()
    p = jarq.integer_product(q, xs, c, w, g, dtype="float32")
    assert ((p.double() - want).abs() <= terms * 2.0 ** -24 * 1.01 * size + 2.0 ** -24 * want.abs() + 1e-12 * x64.abs().max() * din).all()


# groups of 64 with many tokens: an odd number of groups, one and several tiles a
# cluster, K split or not; every output against 64 bits on the device.  The bound is
# _check's: G products and G - 1 additions in float32, and the three roundings of
# the token's scale, the bias and the output.
@pytest.mark.parametrize("n,din,dout", [(600, 64, 2900), (1500, 192, 5000), (700, 1088, 1300), (2100, 320, 5003), (513, 4160, 520),
                                        (4000, 576, 9000)])
def test_odd_numbers_of_groups(jarq, n, din, dout):
    g = 64
    rng = np.random.default_rng(n + din)
    c = _rows(_codes(rng, dout, din, 15))
    w = torch.as_tensor(rng.standard_normal((dout, din // g)).astype(np.float32)).cuda()
    X = torch.as_tensor((rng.standard_normal((n, din)) * 2).astype(np.float32)).cuda().half()
    q, xs = jarq.quantize_rows(X)
    y = jarq.integer_linear(X, c, w, g, dtype="float32").double()
    want, size = torch.zeros_like(y), torch.zeros_like(y)
    for i in range(din // g):
        part = (q[:, i * g:(i + 1) * g].double() @ c[:, i * g:(i + 1) * g].double().T) * w[:, i].double()
        want += part
        size += part.abs()
    want *= xs.double()[:, None]
    size *= xs.double()[:, None]
    bound = (2 * (din // g) + 3) * 2.0 ** -24 * 1.01 * size + 1e-30
    assert ((y - want).abs() <= bound).all()
    assert torch.equal(y, jarq.integer_linear(X, c, w, g, dtype="float32").double())


# a single token, which shorter rows' blocks quantize for themselves: the same bits
# as quantization and product apart, on both sides of the change, at lengths that
# are no multiple of 16, from any alignment, and with rows that hold no number
@pytest.mark.parametrize("xdtype", list(DT))
@pytest.mark.parametrize("din,dout,g,offset", [(1, 1, 0, 0), (17, 5, 0, 1), (1001, 1343, 0, 3), (4096, 2500, 64, 0), (6143, 40, 0, 2),
                                               (6144, 700, 128, 1), (6145, 40, 0, 0), (6272, 300, 128, 0)])
def test_single_token(jarq, xdtype, din, dout, g, offset):
    rng = np.random.default_rng(din)
    c = _rows(_codes(rng, dout, din, 15), din + offset, offset)
    w = torch.as_tensor(rng.standard_normal((dout, din // g if g else 1)).astype(np.float32)).cuda()
    x = torch.as_tensor(rng.standard_normal((1, din)).astype(np.float32)).to(DT[xdtype])
    for last in (None, 0.0, float("inf"), float("nan")):
        if last is not None:
            x[0, -1] = last
            if last == 0.0:
                x.zero_()
        X = _rows(x, None, offset)
        q, xs = jarq.quantize_rows(X)
        y = jarq.integer_linear(X, c, w, g, dtype="float32")
        assert torch.equal(y.view(torch.int32), jarq.integer_product(q, xs, c, w, g, dtype="float32").view(torch.int32))
