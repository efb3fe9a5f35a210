"""Host code of the operators that only enqueue, on the CPU: argument checks
that return before any CUDA work, and (linked to a CUDA runtime without a
device) the stream they work on, with nothing waited for or allocated."""
import ctypes

import pytest

from test_host_paths import STREAM, dev, lib  # noqa: F401  (fixtures)


@pytest.fixture(scope="module")
def jarq():
    from paper_2609_38599_gb300 import jarq as mod
    return mod


F32, F16 = 0, 1


def test_empty_batches_return_ok_without_cuda_work(jarq):
    L = jarq.library()
    assert L.jarq_quantize_rows(None, F16, 0, 64, 64, None, 64, None, None) == 0
    assert L.jarq_integer_codes(None, None, 0, 64, 64, 3, None, 64, None) == 0
    assert L.jarq_integer_product(None, 64, None, None, 64, None, 0, None, 0, 8, 64, F16, None, 8, None) == 0
    assert L.jarq_integer_linear(None, F16, 64, None, 64, None, 0, None, 0, 8, 64, F16, None, 8, None, 0, None) == 0
    assert L.jarq_token_logprobs(None, F16, 0, 100, 100, None, 1, 5, None, None, None, None, None, None) == 0
    assert L.jarq_token_logprobs_grad(None, F16, 0, 100, 100, None, 1, None, None, None, None, None, 100, None) == 0


def test_sizes_are_checked_first(jarq):
    L, bad = jarq.library(), jarq.JARQ_ERR_ARG

    def quantize(n=1, d=64, ldx=64, ldq=64, dtype=F16):
        return L.jarq_quantize_rows(None, dtype, n, d, ldx, None, ldq, None, None)

    def codes(bits=3, g=64, din=64, ldc=64, dout=0):
        return L.jarq_integer_codes(None, None, dout, din, g, bits, None, ldc, None)

    def product(n=0, dout=8, din=128, g=0, ldx=128, ldc=128, ldy=8, dtype=F16):
        return L.jarq_integer_product(None, ldx, None, None, ldc, None, g, None, n, dout, din, dtype, None, ldy, None)

    def scores(n=0, v=100, ld=100, t=1, k=5, dtype=F16):
        return L.jarq_token_logprobs(None, dtype, n, v, ld, None, t, k, None, None, None, None, None, None)

    def grad(n=0, v=100, ld=100, t=1, ldd=100, dtype=F16):
        return L.jarq_token_logprobs_grad(None, dtype, n, v, ld, None, t, None, None, None, None, None, ldd, None)

    for got in (quantize(n=-1), quantize(d=0), quantize(ldx=63), quantize(ldq=63), quantize(dtype=3), quantize(),
                codes(bits=8), codes(bits=0), codes(g=48), codes(ldc=63), codes(dout=-1), codes(dout=1),
                product(n=-1), product(dout=0), product(din=0), product(din=65537, ldx=65537, ldc=65537),
                product(g=32), product(g=128, din=192, ldx=192, ldc=192), product(ldx=127), product(ldc=127),
                product(ldy=7), product(dtype=-1), product(n=1),
                scores(n=-1), scores(v=0), scores(ld=99), scores(t=257), scores(t=-1), scores(k=33), scores(k=-1),
                scores(v=4, k=5), scores(dtype=7), scores(n=1),
                grad(n=-1), grad(t=0), grad(ldd=99), grad(t=257), grad(n=1)):
        assert got == bad
    for got in (product(g=64), product(g=128), scores(), scores(k=0, t=0), grad()):
        assert got == jarq.JARQ_OK


def test_workspace_covers_padded_codes_and_scales(jarq):
    size = jarq.library().jarq_integer_linear_workspace
    assert size(1, 1) >= 16 + 4 and size(3, 17) >= 3 * (32 + 4)
    assert size(0, 64) == 0 and size(-1, 64) == 0 and size(4, 0) == 0
    assert size(70000, 65536) > 2 ** 32


def test_operators_enqueue_on_their_stream_and_wait_for_nothing(dev):  # noqa: F811
    """Launches on the caller's stream; no copy, fill, synchronisation or
    device allocation."""
    L, s = dev.lib, ctypes.c_void_p(STREAM)
    L.jarq_integer_linear_workspace.restype = ctypes.c_size_t
    i64, n, din, dout, v = ctypes.c_int64, 5, 256, 96, 1000
    x, q, xs = dev.buf(4 * n * din), dev.buf(n * din), dev.buf(4 * n)
    C, ws, y = dev.buf(dout * din), dev.buf(4 * dout * 4), dev.buf(4 * n * dout)
    size = L.jarq_integer_linear_workspace(n, din)
    work = dev.buf(size)
    logits, tok, f, out = dev.buf(4 * n * v), dev.buf(8 * n), dev.buf(4 * n), dev.buf(4 * n * v)
    top, ids = dev.buf(4 * n * 8), dev.buf(4 * n * 8)
    before, live = len(dev.log()), L.fake_live()
    calls = [
        lambda: L.jarq_quantize_rows(x, F32, n, din, i64(din), q, i64(din), xs, s),
        lambda: L.jarq_integer_product(q, i64(din), xs, C, i64(din), ws, 64, None, n, dout, din, F32, y, i64(dout), s),
        lambda: L.jarq_integer_linear(x, F32, i64(din), C, i64(din), ws, 0, None, n, dout, din, F16, y, i64(dout), work,
                                      ctypes.c_size_t(size), s),
        lambda: L.jarq_token_logprobs(logits, F32, n, v, i64(v), tok, 1, 8, f, f, f, top, ids, s),
        lambda: L.jarq_token_logprobs_grad(logits, F32, n, v, i64(v), tok, 1, f, f, f, f, out, i64(v), s),
    ]
    for call in calls:
        assert call() == 0
    log = [e for e in dev.log()[before:] if e[0] != "attribute"]
    assert {e[0] for e in log} == {"launch"} and {e[1] for e in log} == {str(STREAM)}
    assert len(log) >= len(calls) + 1                  # the linear layer has two halves
    assert L.fake_live() == live
    assert L.jarq_async_status(s) == 0
    assert dev.log()[-1][0] == "sync"
