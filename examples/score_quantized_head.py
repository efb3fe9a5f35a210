"""Quantizes an output projection, runs it in integers and scores what it answers.

A synthetic output head ``logits = X W^T`` is quantized to 3 bits by the
round-to-nearest host, refined on the calibration Hessian of its inputs, and both
states are run on held-out inputs in 8-bit integers (``integer_linear``: one
scale a token, one a channel and group).  ``token_logprobs`` scores the tokens
that the full-precision head draws, which is what a perplexity is the exponential
of, and ``token_logprobs_grad`` fits a bias of the refined head to them.

    python examples/score_quantized_head.py
"""
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

from paper_2609_38599_gb300 import jarq  # noqa: E402
from synth import activations_torch, rtn_host_torch  # noqa: E402


def main(vocab=4000, din=512, group=128, bits=3, tokens=4096, steps=8, device="cuda"):
    gen = torch.Generator(device=device).manual_seed(0)
    # calibration and held-out inputs: correlated, with a few outlier channels
    X = activations_torch(2 * tokens, din, rank=16, n_out=2, out_scale=8.0, D_lo=0.05, seed=3, device=device)
    calib, held = X[:tokens].contiguous(), X[tokens:].contiguous()
    W = torch.randn(vocab, din, generator=gen, device=device)
    W *= 2.5 / (held.float() @ W.T).std()

    # quantize: calibration Hessian, host state, refinement
    H = jarq.accumulate_hessian(calib, scale=1.0 / tokens)
    nu2 = 0.01 * float(H.diagonal().mean())
    S0, Q0, Z = rtn_host_torch(W, bits, group)
    S, Q = S0.clone(), Q0.clone()
    hess = jarq.prepare(H, group, nu2)
    jarq.refine(hess, W, S, Q, Z, bits, max_iters=5, collect_stats=False)
    hess.close()

    # the tokens that the full-precision head draws
    full = held.float() @ W.T
    drawn = torch.multinomial(torch.softmax(full, 1), 1, generator=gen)[:, 0]
    result = {"full": jarq.token_logprobs(full, drawn).logprob.mean().item()}

    # run both quantized heads in integers and score the tokens
    heads = {"host": (jarq.integer_codes(Q0, Z, group, bits), S0), "refined": (jarq.integer_codes(Q, Z, group, bits), S)}
    for name, (codes, scales) in heads.items():
        logits = jarq.integer_linear(held, codes, scales, group, dtype="float32")
        scores = jarq.token_logprobs(logits, drawn, top=5)
        result[name] = scores.logprob.mean().item()
        result[name + " in top 5"] = (scores.top_token == drawn[:, None]).any(1).float().mean().item()
    assert jarq.async_status() == jarq.JARQ_OK

    # a bias of the refined head, by gradient ascent on the tokens' log probability
    codes, scales = heads["refined"]
    bias = torch.zeros(vocab, device=device)
    weight = torch.full((tokens,), 1.0 / tokens, device=device)
    for _ in range(steps):
        logits = jarq.integer_linear(held, codes, scales, group, bias=bias, dtype="float32")
        scores = jarq.token_logprobs(logits, drawn)
        grad = jarq.token_logprobs_grad(logits, drawn, scores.lse, weight, out=logits)
        bias += 100.0 * grad.sum(0)
    logits = jarq.integer_linear(held, codes, scales, group, bias=bias, dtype="float32")
    result["refined with a bias"] = jarq.token_logprobs(logits, drawn).logprob.mean().item()
    return result


if __name__ == "__main__":
    for name, value in main().items():
        print(f"{name:22s} {value:9.4f}")
