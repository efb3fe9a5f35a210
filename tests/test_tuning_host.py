"""Host code of the norm, the head's loss and the adapters, on the CPU: what is refused
before any CUDA work, the stream they work on, with nothing waited for or allocated on
the device, and a late failure reported by each (linked to a CUDA runtime without a
device)."""
import ctypes

import pytest

torch = pytest.importorskip("torch")

from test_host_paths import STREAM, dev, lib  # noqa: F401  (fixtures)
from test_operators_arguments import FakeCuda, calls, jarq  # noqa: F401  (fixtures)
from test_operators_late_failure import word  # noqa: F401  (fixture)

F32, F16, BF16 = 0, 1, 2
ARG, TIMEOUT = 1, 5
MOST = 2 ** 31 - 4096


def norm(L, n=0, d=64, ldx=64, R=None, ldr=64, H=None, ldh=64, gain=None, gtype=F16, eps=1e-5, Y=None, ldy=64, Q=None, ldq=64,
         scale=None, rstd=None, dtype=F16, X=None):
    return L.jarq_rms_norm(X, dtype, n, d, ldx, R, ldr, H, ldh, gain, gtype, eps, Y, ldy, Q, ldq, scale, rstd, None)


def norm_grad(L, n=0, d=64, ldh=64, gain=None, gtype=F16, ldy=64, dH=None, lds=64, dX=1, ldx=64, dgain=None, dtype=F16, dY=None):
    return L.jarq_rms_norm_grad(None, dtype, n, d, ldh, gain, gtype, None, dY, ldy, dH, lds, dX, ldx, dgain, None, 0, None)


def loss(L, n=0, d=64, ldx=64, vocab=100, ldw=64, dtype=F16):
    return L.jarq_cross_entropy(None, dtype, n, d, ldx, None, vocab, ldw, None, None, None, None, 0, None)


def loss_grad(L, n=0, d=64, ldx=64, vocab=100, ldw=64, dX=1, lddx=64, dW=None, lddw=64, dtype=F16):
    return L.jarq_cross_entropy_grad(None, dtype, n, d, ldx, None, vocab, ldw, None, None, None, dX, lddx, dW, lddw, None, 0, None)


def adapt(L, n=0, din=64, dout=32, rank=16, m=4, ldx=64, Y0=None, ldy0=32, ldy=32, dtype=F16, ytype=F16, Y=None):
    return L.jarq_apply_adapters(None, dtype, ldx, None, None, None, m, rank, None, n, din, dout, Y0, ldy0, Y, ldy, ytype, None, 0, None)


def test_empty_batches_return_ok_without_cuda_work(jarq):  # noqa: F811
    L = jarq.library()
    for call in (norm, norm_grad, loss, loss_grad, adapt):
        assert call(L) == 0, call.__name__


def test_sizes_are_checked_first(jarq):  # noqa: F811
    L = jarq.library()
    bad = [norm(L, n=-1), norm(L, n=MOST + 1), norm(L, d=0), norm(L, d=MOST + 1, ldx=MOST + 1), norm(L, ldx=63), norm(L, dtype=3),
           norm(L, eps=0.0), norm(L, eps=-1.0), norm(L, eps=float("inf")), norm(L, eps=float("nan")), norm(L, R=64), norm(L, H=64),
           norm(L, R=64, H=128, ldr=63), norm(L, R=64, H=128, ldh=63), norm(L, Y=64, ldy=63), norm(L, Q=64), norm(L, scale=64),
           norm(L, Q=64, scale=128, ldq=63), norm(L, gain=64, gtype=BF16), norm(L, n=2, R=64, H=64, ldh=65), norm(L, n=1),
           norm_grad(L, n=-1), norm_grad(L, n=MOST + 1), norm_grad(L, d=0), norm_grad(L, ldh=63), norm_grad(L, ldy=63), norm_grad(L, dtype=-1),
           norm_grad(L, dX=None), norm_grad(L, dH=64, lds=63), norm_grad(L, ldx=63), norm_grad(L, gain=64, gtype=BF16),
           norm_grad(L, n=2, dX=64, dY=64, ldx=65), norm_grad(L, n=2, dX=64, dH=64, ldx=65), norm_grad(L, n=1),
           loss(L, n=-1), loss(L, n=2 ** 22 + 1), loss(L, d=0), loss(L, ldx=63), loss(L, ldw=63), loss(L, vocab=0),
           loss(L, vocab=2 ** 30 + 1), loss(L, d=2 ** 20 + 1, ldx=2 ** 21, ldw=2 ** 21), loss(L, dtype=F32), loss(L, n=1),
           loss_grad(L, n=-1), loss_grad(L, vocab=0), loss_grad(L, dX=None), loss_grad(L, lddx=63), loss_grad(L, dW=64, lddw=63),
           loss_grad(L, dtype=F32), loss_grad(L, n=1), loss_grad(L, ldw=63),
           adapt(L, n=-1), adapt(L, n=2 ** 30 + 1), adapt(L, din=0), adapt(L, dout=0), adapt(L, ldx=63), adapt(L, ldy=31),
           adapt(L, Y0=64, ldy0=31), adapt(L, rank=4), adapt(L, rank=12), adapt(L, rank=136), adapt(L, m=-1), adapt(L, m=8193),
           adapt(L, dtype=F32), adapt(L, ytype=BF16), adapt(L, n=2, Y0=64, Y=64, ldy0=33), adapt(L, n=1),
           adapt(L, din=2 ** 20 + 1, ldx=2 ** 21), adapt(L, dout=2 ** 20 + 1, ldy=2 ** 21)]
    assert bad == [ARG] * len(bad)
    assert adapt(L, dtype=BF16, ytype=F32) == 0 and norm(L, gain=64, gtype=F32) == 0 and loss(L, dtype=BF16) == 0


def test_workspaces_of_sizes_that_are_refused(jarq):  # noqa: F811
    L = jarq.library()
    assert L.jarq_rms_norm_grad_workspace(-1, 64) == 0 and L.jarq_rms_norm_grad_workspace(4, 0) == 0
    assert L.jarq_rms_norm_grad_workspace(200, 64) == 200 * 64 * 4 and L.jarq_rms_norm_grad_workspace(10 ** 6, 64) == 608 * 64 * 4
    assert L.jarq_rms_norm_grad_workspace(152, 64) == 0 and L.jarq_adapters_workspace(64, 64, 16, 1) == 0 < L.jarq_adapters_workspace(65, 64, 16, 1)
    assert L.jarq_cross_entropy_workspace(0, 64, 100, 1) == 0 and L.jarq_cross_entropy_workspace(2 ** 22 + 1, 64, 100, 1) == 0
    assert L.jarq_adapters_workspace(0, 64, 16, 1) == 0 and L.jarq_adapters_workspace(8, 64, 20, 1) == 0
    # room for copies of rows that are not on 16-byte boundaries
    a, b = (L.jarq_cross_entropy_workspace(10, 65, 1000, k) for k in (1, 0))
    assert b - a >= 2 * 72 * 1010
    both, x, w = (L.jarq_cross_entropy_grad_workspace(300, 128, 5000, 1, *k) for k in ((1, 1), (1, 0), (0, 1)))
    assert both >= max(x, w) and min(x, w) >= 300 * 5000 * 2


def test_a_piece_of_the_vocabulary_at_a_time(jarq):  # noqa: F811
    """The gradient's workspace does not grow with the vocabulary beyond 512 MB of it."""
    L = jarq.library()
    size = lambda n, v: L.jarq_cross_entropy_grad_workspace(n, 64, v, 1, 1, 0)
    assert size(8192, 10 ** 6) < (512 << 20) * 1.1 + 16 * 4 * 8192 * 64
    assert size(8192, 10 ** 6) < 8192 * 10 ** 6 / 8
    assert size(2 ** 20, 10 ** 6) < 2 ** 20 * 5000 * 2 + 16 * 4 * 2 ** 20 * 64


def _calls(d):
    L, s, i64, cf = d.lib, ctypes.c_void_p(STREAM), ctypes.c_int64, ctypes.c_float
    for f in ("jarq_rms_norm_grad_workspace", "jarq_cross_entropy_workspace", "jarq_cross_entropy_grad_workspace", "jarq_adapters_workspace"):
        getattr(L, f).restype = ctypes.c_size_t
    n, w, v, m, r, o = 300, 256, 1000, 3, 16, 96
    x, y, z, q = (d.buf(4 * n * w) for _ in range(4))
    f, gain, tok, ids = d.buf(4 * n), d.buf(4 * w), d.buf(8 * n), d.buf(4 * n)
    W, A, B, out = d.buf(2 * v * w), d.buf(2 * m * r * w), d.buf(2 * m * r * o), d.buf(4 * n * o)
    size = ctypes.c_size_t(64 << 20)
    work = d.buf(size.value)
    return {
        "norm": lambda: L.jarq_rms_norm(x, F16, n, w, i64(w), y, i64(w), z, i64(w), gain, F32, cf(1e-5), y, i64(w), q, i64(w), f, f, s),
        "one row": lambda: L.jarq_rms_norm(x, F32, 1, w, i64(w), None, i64(w), None, i64(w), None, F32, cf(1e-5), y, i64(w), None, i64(w), None, None, s),
        "norm_grad": lambda: L.jarq_rms_norm_grad(x, BF16, n, w, i64(w), gain, F32, f, y, i64(w), None, i64(w), z, i64(w), gain, work, size, s),
        "loss": lambda: L.jarq_cross_entropy(x, F16, n, w, i64(w), W, v, i64(w), tok, f, f, work, size, s),
        "unaligned loss": lambda: L.jarq_cross_entropy(x, F16, n, 250, i64(251), W, v, i64(253), tok, f, None, work, size, s),
        "loss_grad": lambda: L.jarq_cross_entropy_grad(x, F16, n, w, i64(w), W, v, i64(w), tok, f, f, y, i64(w), W, i64(w), work, size, s),
        "adapters": lambda: L.jarq_apply_adapters(x, BF16, i64(w), A, B, f, m, r, ids, n, w, o, out, i64(o), out, i64(o), F32, work, size, s),
        "few adapters": lambda: L.jarq_apply_adapters(x, F16, i64(w), A, B, None, m, r, ids, 5, w, o, None, i64(o), out, i64(o), F16, work, size, s),
    }


def test_calls_only_enqueue_on_their_stream(dev):  # noqa: F811
    made = _calls(dev)
    for name, call in made.items():
        before, live = len(dev.log()), dev.lib.fake_live()
        assert call() == 0, name
        new = [e for e in dev.log()[before:] if e[0] != "attribute"]
        assert {e[0] for e in new} == {"launch"} and {e[1] for e in new} == {str(STREAM)}, (name, new)
        assert dev.lib.fake_live() == live, name


def test_every_call_reports_a_failure_until_it_is_asked_for(dev, word):  # noqa: F811
    made = _calls(dev)
    for name, call in made.items():
        assert call() == 0, name
    word[0] = 1
    before = len(dev.log())
    assert {name: call() for name, call in made.items()} == dict.fromkeys(made, TIMEOUT)
    assert len(dev.log()) == before                     # and nothing is enqueued
    assert dev.lib.jarq_async_status(ctypes.c_void_p(STREAM)) == TIMEOUT
    for name, call in made.items():
        assert call() == 0, name


def test_pointers_and_workspaces_are_checked(dev):  # noqa: F811
    """Host memory, misaligned memory and a workspace that is too small are refused, and
    nothing is enqueued."""
    L, s, i64, cf = dev.lib, ctypes.c_void_p(STREAM), ctypes.c_int64, ctypes.c_float
    _calls(dev)
    host = ctypes.addressof(ctypes.create_string_buffer(1 << 16))
    x, W, tok, f, work = dev.buf(1 << 16), dev.buf(1 << 16), dev.buf(1 << 12), dev.buf(1 << 12), dev.buf(1 << 20)
    odd = lambda p, k: ctypes.c_void_p(p.value + k)
    size = L.jarq_cross_entropy_workspace(8, 64, 100, 1)
    gsize = L.jarq_cross_entropy_grad_workspace(8, 64, 100, 1, 1, 1)
    asize = L.jarq_adapters_workspace(100, 64, 16, 2)
    z = ctypes.c_size_t
    made = [
        lambda X=x, T=tok, F=f, w=work, k=size: L.jarq_cross_entropy(X, F16, 8, 64, i64(64), W, 100, i64(64), T, F, f, w, z(k), s),
        lambda X=x, T=tok, F=f, w=work, k=gsize: L.jarq_cross_entropy_grad(X, F16, 8, 64, i64(64), W, 100, i64(64), T, F, f, x, i64(64), W, i64(64), w, z(k), s),
        lambda X=x, T=tok, F=f, w=work, k=asize: L.jarq_apply_adapters(X, F16, i64(64), W, W, F, 2, 16, T, 100, 64, 32, x, i64(32), x, i64(32), F16, w, z(k), s),
        lambda X=x, T=tok, F=f, w=work, k=200 * 64 * 4: L.jarq_rms_norm_grad(X, F16, 200, 64, i64(64), None, F16, F, x, i64(64), None, i64(64), W, i64(64), T, w, z(k), s),
    ]
    for call in made:
        assert call() == 0
    before = len(dev.log())
    for i, call in enumerate(made):
        for wrong in (dict(X=host), dict(X=odd(x, 1)), dict(X=None), dict(T=host), dict(T=odd(tok, 2)), dict(F=odd(f, 2)),
                      dict(w=None), dict(w=odd(work, 8)), dict(w=host)):
            assert call(**wrong) == ARG, (i, wrong)
        assert call(k=(size, gsize, asize, 200 * 64 * 4)[i] - 1) == ARG, i
    assert len(dev.log()) == before


# ---- the Python entries, with a library that notes its calls

def fake(shape, dtype=torch.float16, **kw):
    return FakeCuda(shape, dtype, **kw)


def test_python_entries_refuse_what_does_not_fit(jarq, calls):  # noqa: F811
    x, g = fake((6, 64)), fake((64,))
    rstd, dy = fake((6,), torch.float32), fake((6, 64))
    W, tok = fake((100, 64)), fake((6,), torch.int64)
    A, B, ids = fake((3, 16, 64)), fake((3, 32, 16)), fake((6,), torch.int32)
    lse = fake((6,), torch.float32)
    for wrong in (lambda: jarq.rms_norm(fake((6, 64), torch.float64)), lambda: jarq.rms_norm(x, fake((63,))),
                  lambda: jarq.rms_norm(x, fake((64,), torch.bfloat16)), lambda: jarq.rms_norm(x, residual=fake((5, 64))),
                  lambda: jarq.rms_norm(x, residual=fake((6, 64), torch.bfloat16)), lambda: jarq.rms_norm(x, h=dy),
                  lambda: jarq.rms_norm(x, residual=dy, h=fake((6, 65))), lambda: jarq.rms_norm(torch.zeros(6, 64)),
                  lambda: jarq.rms_norm_grad(x, g, fake((5,), torch.float32), dy), lambda: jarq.rms_norm_grad(x, g, rstd, fake((6, 63))),
                  lambda: jarq.rms_norm_grad(x, g, rstd, dy, dh=fake((6, 64), torch.float32)),
                  lambda: jarq.rms_norm_grad(x, g, rstd, dy, rows=False, out=dy),
                  lambda: jarq.cross_entropy(x, fake((100, 63)), tok), lambda: jarq.cross_entropy(x, fake((100, 64), torch.bfloat16), tok),
                  lambda: jarq.cross_entropy(fake((6, 64), torch.float32), fake((100, 64), torch.float32), tok),
                  lambda: jarq.cross_entropy(x, W, fake((6,), torch.int32)), lambda: jarq.cross_entropy(x, W, fake((5,), torch.int64)),
                  lambda: jarq.cross_entropy_grad(x, W, tok, fake((5,), torch.float32), lse),
                  lambda: jarq.cross_entropy_grad(x, W, tok, lse, fake((6,))),
                  lambda: jarq.apply_adapters(x, fake((3, 16, 63)), B, ids), lambda: jarq.apply_adapters(x, A, fake((3, 32, 8)), ids),
                  lambda: jarq.apply_adapters(x, A, fake((2, 32, 16)), ids), lambda: jarq.apply_adapters(x, fake((16, 64)), B, ids),
                  lambda: jarq.apply_adapters(x, A, B, fake((6,), torch.int64)), lambda: jarq.apply_adapters(x, A, B, fake((5,), torch.int32)),
                  lambda: jarq.apply_adapters(x, A, B, ids, scale=fake((2,), torch.float32)),
                  lambda: jarq.apply_adapters(x, A, B, ids, base=fake((6, 31))),
                  lambda: jarq.apply_adapters(x, A, B, ids, base=fake((6, 32), torch.bfloat16)),
                  lambda: jarq.apply_adapters(x, A, B, ids, base=fake((6, 32)), dtype="float32"),
                  lambda: jarq.apply_adapters(x, A, B, ids, dtype="bfloat16")):
        with pytest.raises((TypeError, ValueError)):
            wrong()
    assert not calls
