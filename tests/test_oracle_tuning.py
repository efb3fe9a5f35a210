"""The float64 forms of the norm, the head's loss and the adapters against closed
forms, differences and planted mistakes."""
import numpy as np
import pytest

from oracle import jarq_tuning as O


def _difference(f, x, at, step=1e-6):
    """Central differences of the number f(x) by the elements `at` of x."""
    out = []
    for i in at:
        hi, lo = x.copy(), x.copy()
        hi[i] += step
        lo[i] -= step
        out.append((f(hi) - f(lo)) / (2 * step))
    return np.array(out)


def test_norm_of_equal_and_single_elements():
    r = O.rms_norm(np.array([[3.0, -3.0, 3.0, -3.0], [0.0, 0.0, 8.0, 0.0]]), None, 0.0)
    assert np.allclose(r["y"], [[1, -1, 1, -1], [0, 0, 2, 0]])
    assert (r["codes"] == [[127, -127, 127, -127], [0, 0, 127, 0]]).all()
    assert np.allclose(r["codes"] * r["scale"][:, None], r["y"])


def test_integers_do_not_depend_on_the_row_s_factor():
    rng = np.random.default_rng(0)
    h, g = rng.standard_normal((5, 64)), 0.5 + rng.random(64)
    a, b = O.rms_norm(h, g, 1e-6), O.rms_norm(h * 4.0, g, 1e-6)
    assert (a["codes"] == b["codes"]).all() and np.allclose(a["y"], b["y"], rtol=1e-5)


@pytest.mark.parametrize("gain", [False, True])
def test_norm_gradient_is_the_norm_s(gain):
    rng = np.random.default_rng(1)
    h, dy, dh = rng.standard_normal((3, 3, 17))
    g = 0.5 + rng.random(17) if gain else None
    rstd = O.rms_norm(h, g, 1e-3)["rstd"]
    dx, dgain = O.rms_norm_grad(h, g, rstd, dy, dh)
    at = [(r, k) for r in range(3) for k in range(0, 17, 4)]
    loss = lambda x: (O.rms_norm(x, g, 1e-3)["y"] * dy).sum() + (x * dh).sum()
    assert np.allclose(_difference(loss, h, at), [dx[i] for i in at], atol=1e-7)
    ones = np.ones(17) if g is None else g
    at = [(k,) for k in range(17)]
    assert np.allclose(_difference(lambda w: (O.rms_norm(h, w, 1e-3)["y"] * dy).sum(), ones, at), dgain, atol=1e-7)
    # the projection along h and the residual's gradient are both needed
    assert not np.allclose(rstd[:, None] * dy * ones + dh, dx, atol=1e-3) and not np.allclose(dx - dh, dx, atol=1e-3)


def test_loss_of_equal_logits_and_ignored_tokens():
    X, W = np.ones((3, 2)), np.zeros((10, 2))
    loss, lse = O.cross_entropy(X, W, np.array([4, -1, 10]))
    assert np.allclose(lse, np.log(10)) and np.isclose(loss[0], np.log(10)) and loss[1] == 0 and np.isnan(loss[2])


def test_loss_gradient_is_the_loss_s():
    rng = np.random.default_rng(2)
    X, W = rng.standard_normal((4, 6)), rng.standard_normal((9, 6))
    tok, g = np.array([0, 8, -1, 3]), rng.standard_normal(4)
    lse = O.cross_entropy(X, W, tok)[1]
    dX, dW = O.cross_entropy_grad(X, W, tok, lse, g)
    total = lambda x, w: (O.cross_entropy(x, w, tok)[0] * g).sum()
    at = [(i, j) for i in range(4) for j in range(6)]
    assert np.allclose(_difference(lambda x: total(x, W), X, at), [dX[i] for i in at], atol=1e-7)
    at = [(i, j) for i in range(9) for j in range(6)]
    assert np.allclose(_difference(lambda w: total(X, w), W, at), [dW[i] for i in at], atol=1e-7)
    assert (dX[2] == 0).all()
    D = O.logit_gradient(X, W, tok, lse, g)
    assert np.allclose(D.sum(axis=1), 0)                 # softmax and one-hot both sum to one
    D[np.arange(2), tok[:2]] += g[:2]
    assert not np.allclose(D @ W, dX, atol=1e-3)         # the one-hot left out


def test_adapters_of_a_row_alone():
    rng = np.random.default_rng(3)
    X, A, B = rng.standard_normal((4, 5)), rng.standard_normal((2, 3, 5)), rng.standard_normal((2, 7, 3))
    base, scale = rng.standard_normal((4, 7)), np.array([0.5, -2.0])
    Y = O.apply_adapters(X, A, B, [1, -1, 0, 2], scale, base)
    assert np.allclose(Y[0], base[0] - 2.0 * (B[1] @ A[1]) @ X[0]) and (Y[1] == base[1]).all()
    assert np.allclose(Y[2], base[2] + 0.5 * (B[0] @ A[0]) @ X[2]) and np.isnan(Y[3]).all()
