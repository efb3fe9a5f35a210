"""Norms, the loss of an output head and adapters in float64 NumPy, from their
definitions.

Test infrastructure for the operators that run and score a quantized model:
the root-mean-square norm of rows with its 8-bit integers and its gradient, the
softmax cross entropy of hidden states under a head with its gradient, and low-rank
adapters of many requests.
"""
from __future__ import annotations

import numpy as np


def rms_norm(h, gain, eps):
    """dict of rstd, y (float64) and the codes and scale of v = h gain, which are
    defined in float32 up to the row's own factor."""
    h = np.asarray(h, dtype=np.float64)
    g = np.ones(h.shape[1]) if gain is None else np.asarray(gain, dtype=np.float64)
    with np.errstate(all="ignore"):
        rstd = 1.0 / np.sqrt((h * h).mean(axis=1) + eps)
        v32 = h.astype(np.float32) * g.astype(np.float32)
        codes = np.zeros(h.shape, dtype=np.int8)
        scale = np.zeros(h.shape[0])
        for r, v in enumerate(v32):
            a = np.max(np.abs(v))
            if not np.isfinite(v).all():
                scale[r] = np.nan
            elif a >= np.float32(2.0) ** -120:
                scale[r] = np.float64(a) / 127.0 * rstd[r]
                codes[r] = np.rint(v * (np.float32(127) / a)).astype(np.int8)
        return {"rstd": rstd, "y": h * g * rstd[:, None], "codes": codes, "scale": scale}


def rms_norm_grad(h, gain, rstd, dy, dh=None):
    """(dx, dgain) from the given rstd."""
    h, dy, r = (np.asarray(x, dtype=np.float64) for x in (h, dy, rstd))
    g = np.ones(h.shape[1]) if gain is None else np.asarray(gain, dtype=np.float64)
    u = dy * g
    dx = r[:, None] * (u - h * (r ** 2 * (u * h).mean(axis=1))[:, None])
    if dh is not None:
        dx = dx + np.asarray(dh, dtype=np.float64)
    return dx, (dy * h * r[:, None]).sum(axis=0)


def cross_entropy(X, W, tokens):
    """(loss, lse) of every row; negative tokens are ignored, others past the
    vocabulary give NaN."""
    logits = np.asarray(X, dtype=np.float64) @ np.asarray(W, dtype=np.float64).T
    loss, lse = np.zeros(len(tokens)), np.zeros(len(tokens))
    for r, (row, t) in enumerate(zip(logits, tokens)):
        m = row.max()
        lse[r] = m + np.log(np.exp(row - m).sum())
        loss[r] = 0.0 if t < 0 else np.nan if t >= row.size else lse[r] - row[t]
    return loss, lse


def logit_gradient(X, W, tokens, lse, g_loss):
    """D[r][v] = g_r (exp(l_rv - lse_r) - [v = token_r]), 0 where the token is ignored."""
    D = np.exp(np.asarray(X, dtype=np.float64) @ np.asarray(W, dtype=np.float64).T - np.asarray(lse, np.float64)[:, None])
    for r, t in enumerate(tokens):
        if t < 0:
            D[r] = 0.0
        elif t >= D.shape[1]:
            D[r] = np.nan
        else:
            D[r, t] -= 1.0
            D[r] *= float(g_loss[r])
    return D


def cross_entropy_grad(X, W, tokens, lse, g_loss):
    """(dX, dW) of sum(g_loss loss)."""
    D = logit_gradient(X, W, tokens, lse, g_loss)
    return D @ np.asarray(W, dtype=np.float64), D.T @ np.asarray(X, dtype=np.float64)


def apply_adapters(X, A, B, ids, scale=None, base=None):
    """base + scale_i B_i (A_i x) for every row's adapter i = ids[row]; none for a
    negative one, NaN for one that there is not."""
    X, A, B = (np.asarray(x, dtype=np.float64) for x in (X, A, B))
    Y = np.zeros((X.shape[0], B.shape[1])) if base is None else np.array(base, dtype=np.float64)
    for r, i in enumerate(ids):
        if i >= A.shape[0]:
            Y[r] = np.nan
        elif i >= 0:
            Y[r] += (1.0 if scale is None else float(scale[i])) * (B[i] @ (A[i] @ X[r]))
    return Y
