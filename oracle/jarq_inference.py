"""Integer products and token scores in float64 NumPy, from their definitions.

Test infrastructure for the operators that run and score a quantized model:
rows of activations to 8-bit integers, the product of such integers with scales
for each token, channel and group, log probabilities of tokens under a softmax
with its entropy and most probable tokens, and their gradient.
"""
from __future__ import annotations

import numpy as np


def quantize_rows(X):
    """(codes int8, scale float32): scale = a / 127 and rint(x (127 / a)), a the
    row's largest magnitude, every quotient and product rounded to float32."""
    X = np.asarray(X, dtype=np.float32)
    codes = np.zeros(X.shape, dtype=np.int8)
    scale = np.zeros(X.shape[0], dtype=np.float32)
    for r, x in enumerate(X):
        a = np.max(np.abs(x))
        if not np.isfinite(x).all():
            scale[r] = np.nan
        elif a >= np.float32(2.0) ** -120:
            scale[r] = a / np.float32(127)
            codes[r] = np.rint(x * (np.float32(127) / a)).astype(np.int8)
    return codes, scale


def integer_product(X, xs, C, ws, group_size=0, bias=None):
    """(Y, sum of the terms' magnitudes) in float64; the group sums exact."""
    X, C = np.asarray(X, dtype=np.int64), np.asarray(C, dtype=np.int64)
    n, d = X.shape
    g = group_size or d
    ws = np.asarray(ws, dtype=np.float64).reshape(C.shape[0], -1)
    xs = np.asarray(xs, dtype=np.float64)[:, None]
    Y, M = np.zeros((n, C.shape[0])), np.zeros((n, C.shape[0]))
    for i in range(d // g):
        s = slice(i * g, (i + 1) * g)
        term = xs * (X[:, s].astype(np.float64) @ C[:, s].T.astype(np.float64)) * ws[:, i]
        Y += term
        M += np.abs(term)
    if bias is not None:
        Y = Y + np.asarray(bias, dtype=np.float64)
    return Y, M


def token_logprobs(x, tokens, top=0):
    """dict of logprob, entropy, lse, top_logprob, top_token of every row.
    Negative tokens are ignored (0); -inf masks a token; a row with a NaN or
    +inf is NaN throughout, with tokens -1."""
    x = np.asarray(x, dtype=np.float64)
    n, vocab = x.shape
    out = {"logprob": np.zeros(tokens.shape), "entropy": np.zeros(n), "lse": np.zeros(n),
           "top_logprob": np.full((n, top), -np.inf), "top_token": np.full((n, top), -1)}
    for r in range(n):
        row = x[r]
        live = np.flatnonzero(row > -np.inf)
        bad = np.isnan(row).any() or (row == np.inf).any()
        if bad:
            lse = ent = np.nan
            lp = np.full(vocab, np.nan)
            out["top_logprob"][r] = np.nan
        elif live.size == 0:
            lse, ent, lp = -np.inf, 0.0, np.full(vocab, -np.inf)
        else:
            m = row[live].max()
            d = row[live] - m
            z = np.exp(d).sum()
            lse, ent = m + np.log(z), np.log(z) - (np.exp(d) * d).sum() / z
            lp = np.full(vocab, -np.inf)
            lp[live] = d - np.log(z)
            order = live[np.lexsort((live, -row[live]))][:top]
            out["top_token"][r, :order.size] = order
            out["top_logprob"][r, :order.size] = lp[order]
        out["lse"][r], out["entropy"][r] = lse, ent
        for j, t in enumerate(tokens[r]):
            out["logprob"][r, j] = 0.0 if t < 0 else np.nan if t >= vocab else lp[t]
    return out


def token_logprobs_grad(x, tokens, lse, g_logprob, entropy=None, g_entropy=None):
    """Gradient of sum(g_logprob logprob) + sum(g_entropy entropy) with respect
    to the logits, from given lse and entropy."""
    x = np.asarray(x, dtype=np.float64)
    n, vocab = x.shape
    dx = np.zeros((n, vocab))
    for r in range(n):
        live = x[r] > -np.inf
        lp = x[r][live] - lse[r]
        p = np.exp(lp)
        d = np.zeros(vocab)
        total = 0.0
        for t, g in zip(tokens[r], g_logprob[r]):
            if t >= vocab:
                total = np.nan
            elif t >= 0:
                d[t] += g
                total += g
        d[live] -= total * p
        if g_entropy is not None:
            d[live] -= g_entropy[r] * np.where(p > 0, p * (lp + entropy[r]), 0.0)
        dx[r] = np.where(live, d, 0.0)
    return dx
