"""A device wait that gave up is reported by every later call of the operators that
run and score a quantized model until it has been asked for: the library's host code
on the CPU, linked to a CUDA runtime without a device, with the word that a kernel
would set written by the test."""
import ctypes

import pytest

from test_host_paths import STREAM, dev, lib  # noqa: F401  (fixtures)

F32, TIMEOUT = 0, 5


@pytest.fixture
def word(dev):  # noqa: F811
    """The word in which kernels report a wait that gave up; cleared at the end."""
    f = getattr(dev.lib, "_ZN4jarq10async_wordEv")       # jarq::async_word()
    f.restype = ctypes.POINTER(ctypes.c_int)
    p = f()
    assert p and p[0] == 0
    yield p
    p[0] = 0


def _calls(dev):  # noqa: F811
    L, s, i64 = dev.lib, ctypes.c_void_p(STREAM), ctypes.c_int64
    L.jarq_integer_linear_workspace.restype = ctypes.c_size_t
    n, din, dout, v, g = 3, 256, 96, 1000, 64
    x, q, xs = dev.buf(4 * n * din), dev.buf(n * din), dev.buf(4 * n)
    Q, Z, C = dev.buf(dout * din), dev.buf(4 * dout * 4), dev.buf(dout * din)
    ws, y = dev.buf(4 * dout * 4), dev.buf(4 * n * dout)
    size = L.jarq_integer_linear_workspace(n, din)
    work = dev.buf(size)
    logits, tok, f, out = dev.buf(4 * n * v), dev.buf(8 * n), dev.buf(4 * n), dev.buf(4 * n * v)
    return {
        "quantize_rows": lambda: L.jarq_quantize_rows(x, F32, n, din, i64(din), q, i64(din), xs, s),
        "integer_codes": lambda: L.jarq_integer_codes(Q, Z, dout, din, g, 3, C, i64(din), s),
        "integer_product": lambda: L.jarq_integer_product(q, i64(din), xs, C, i64(din), ws, g, None, n, dout, din, F32, y,
                                                          i64(dout), s),
        "one token": lambda: L.jarq_integer_product(q, i64(din), xs, C, i64(din), ws, g, None, 1, dout, din, F32, y, i64(dout), s),
        "integer_linear": lambda: L.jarq_integer_linear(x, F32, i64(din), C, i64(din), ws, g, None, n, dout, din, F32, y,
                                                        i64(dout), work, ctypes.c_size_t(size), s),
        "token_logprobs": lambda: L.jarq_token_logprobs(logits, F32, n, v, i64(v), tok, 1, 0, f, f, f, None, None, s),
        "token_logprobs_grad": lambda: L.jarq_token_logprobs_grad(logits, F32, n, v, i64(v), tok, 1, f, f, f, f, out, i64(v), s),
    }


def test_every_call_reports_a_failure_until_it_is_asked_for(dev, word):  # noqa: F811
    L, s = dev.lib, ctypes.c_void_p(STREAM)
    calls = _calls(dev)
    for name, call in calls.items():
        assert call() == 0, name
    word[0] = 1
    before = len(dev.log())
    assert {name: call() for name, call in calls.items()} == dict.fromkeys(calls, TIMEOUT)
    assert len(dev.log()) == before                     # and nothing is enqueued
    assert L.jarq_async_status(s) == TIMEOUT
    assert L.jarq_async_status(s) == 0
    for name, call in calls.items():
        assert call() == 0, name


def test_wrong_arguments_are_reported_as_such_beside_a_failure(dev, word):  # noqa: F811
    L, s, i64 = dev.lib, ctypes.c_void_p(STREAM), ctypes.c_int64
    word[0] = 1
    q = dev.buf(64)
    assert L.jarq_quantize_rows(q, F32, 1, 16, i64(15), q, i64(16), q, s) == 1
    assert L.jarq_integer_codes(q, q, 1, 64, 64, 8, q, i64(64), s) == 1
    assert L.jarq_quantize_rows(None, F32, 0, 16, i64(16), None, i64(16), None, s) == 0      # an empty batch
