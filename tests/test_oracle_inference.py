"""The float64 reference of the integer products and token scores, against
closed forms, central differences and planted mistakes."""
import numpy as np
import pytest

from oracle import jarq_inference as O


def test_quantize_rows_by_hand():
    X = np.array([[0.0, 127.0, -63.5, 0.5], [0, 0, 0, 0], [1, np.inf, 0, 0], [2.0 ** -130, 0, 0, 0]])
    q, s = O.quantize_rows(X)
    assert q.tolist() == [[0, 127, -64, 0], [0] * 4, [0] * 4, [0] * 4]     # -63.5 and 0.5: half to even
    assert s[0] == 1 and s[1] == 0 and np.isnan(s[2]) and s[3] == 0


def test_quantize_rows_is_within_half_a_step():
    X = np.random.default_rng(0).standard_normal((40, 333)).astype(np.float32)
    q, s = O.quantize_rows(X)
    assert np.abs(X - q * s[:, None].astype(np.float64)).max() <= 0.5001 * s.max()
    assert (np.abs(q).max(1) == 127).all()


def test_integer_product_equals_the_dequantized_product():
    rng = np.random.default_rng(1)
    X, C = rng.integers(-127, 128, (5, 192)), rng.integers(-15, 16, (7, 192))
    xs, ws, b = rng.random(5), rng.standard_normal((7, 3)), rng.standard_normal(7)
    Y, M = O.integer_product(X, xs, C, ws, 64, b)
    W = C * np.repeat(ws, 64, axis=1)
    assert np.allclose(Y, (X * xs[:, None]) @ W.T + b, rtol=1e-12, atol=1e-12)
    assert (np.abs(Y - b) <= M * (1 + 1e-12)).all()


def test_uniform_logits_have_the_closed_form():
    for v in (1, 2, 1000):
        r = O.token_logprobs(np.full((1, v), -3.25), np.array([[0, v - 1, -1]]), top=min(v, 4))
        assert r["logprob"][0] == pytest.approx([-np.log(v), -np.log(v), 0])
        assert r["entropy"][0] == pytest.approx(np.log(v)) and r["lse"][0] == pytest.approx(np.log(v) - 3.25)
        assert r["top_token"][0].tolist() == list(range(min(v, 4)))


def test_masked_rows():
    x = np.array([[-np.inf, 2.0, -np.inf, 2.0], [-np.inf] * 4, [0, np.nan, 0, 0]])
    r = O.token_logprobs(x, np.array([[0, 1], [0, -1], [0, 4]]), top=3)
    assert r["logprob"][0].tolist() == [-np.inf, -np.log(2)] and r["top_token"][0].tolist() == [1, 3, -1]
    assert r["lse"][1] == -np.inf and r["entropy"][1] == 0 and r["logprob"][1].tolist() == [-np.inf, 0]
    assert np.isnan(r["logprob"][2]).all() and r["top_token"][2].tolist() == [-1, -1, -1]


def _value(x, tok, g, gh):
    r = O.token_logprobs(x, tok)
    return float((g * r["logprob"]).sum() + (gh * r["entropy"]).sum())


@pytest.mark.parametrize("seed", range(3))
def test_gradient_equals_central_differences(seed):
    rng = np.random.default_rng(seed)
    n, v, t = 3, 9, 3
    x = rng.standard_normal((n, v)) * 2
    x[0, 4] = -np.inf
    tok = rng.integers(0, v, (n, t))
    tok[0] = [1, 1, -1]
    tok[tok == 4] = 5
    g, gh = rng.standard_normal((n, t)), rng.standard_normal(n)
    r = O.token_logprobs(x, tok)
    dx = O.token_logprobs_grad(x, tok, r["lse"], g, r["entropy"], gh)
    h = 1e-5
    for i in range(n):
        for j in range(v):
            if x[i, j] == -np.inf:
                assert dx[i, j] == 0
                continue
            up, down = x.copy(), x.copy()
            up[i, j] += h
            down[i, j] -= h
            # truncation h^2 / 6 f''' and rounding 2^-52 |f| / h: both below 1e-9
            assert dx[i, j] == pytest.approx((_value(up, tok, g, gh) - _value(down, tok, g, gh)) / (2 * h), abs=1e-8)


def test_planted_mistakes_are_seen():
    """The checks above tell a gradient without the softmax term, with a dropped
    duplicate or with the entropy's sign turned from the right one."""
    rng = np.random.default_rng(7)
    x, tok = rng.standard_normal((1, 6)), np.array([[2, 2]])
    g, gh = np.array([[0.7, 0.4]]), np.array([0.3])
    r = O.token_logprobs(x, tok)
    dx = O.token_logprobs_grad(x, tok, r["lse"], g, r["entropy"], gh)
    once = O.token_logprobs_grad(x, np.array([[2, -1]]), r["lse"], g, r["entropy"], gh)
    turned = O.token_logprobs_grad(x, tok, r["lse"], g, r["entropy"], -gh)
    no_soft = np.zeros((1, 6))
    no_soft[0, 2] = g.sum()
    for wrong in (once, turned, no_soft):
        assert np.abs(wrong - dx).max() > 1e-2
    assert dx.sum() == pytest.approx(0, abs=1e-12)      # a softmax does not see a shift
