"""Performance cases of the operators that run and score a quantized model:

``linear``  a linear layer in 8-bit integers: every token's activations are
            quantized to int8 with a scale of their own, multiplied with int8
            weight codes and scaled by token and by channel (or by channel and
            group, the form of a refined layer);
``score``   log probabilities of given tokens under logits, with the entropy and
            the most probable alternatives;
``grad``    the gradient of those log probabilities and entropies with respect
            to the logits.

``run`` computes each in plain torch operations in 32 bits (``own`` false) or
through the library's entry points (``own`` true).  ``exact`` is the same from
the definitions in 64 bits.  Layer widths are those of ``synth/layers.py`` and
the benchmark, and ranges around them; vocabularies are generic.  Inputs are
drawn on the GPU from the seed alone.
"""
import math

import torch

own = False

DEV = "cuda"
TYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
BYTES = {"f32": 4, "f16": 2, "bf16": 2}


# ---------------------------------------------------------------- the cases

def _linear(name, n, din, dout, g, x, y, bias=False, pad=0):
    """``g``: group size of the weight scales, 0 for one a channel; ``pad``:
    columns by which the rows of activations and codes lie further apart."""
    return {"name": name, "kind": "linear", "n": n, "din": din, "dout": dout, "g": g, "x": x,
            "y": y, "bias": bias, "pad": pad}


def _score(name, n, vocab, x, t, top, mask):
    """``t``: given tokens a row; ``top``: alternatives; ``mask``: of the logits."""
    return {"name": name, "kind": "score", "n": n, "vocab": vocab, "x": x, "t": t, "top": top,
            "mask": mask}


def _grad(name, n, vocab, x, t, entropy, mask):
    return {"name": name, "kind": "grad", "n": n, "vocab": vocab, "x": x, "t": t,
            "entropy": entropy, "mask": mask}


def listed():
    return [
        # one token through an up projection: generation for a single user
        _linear("linear_token", 1, 4096, 11008, 0, "f16", "f16"),
        # one step of generation for a batch of users, through a refined
        # (group-scaled) down projection
        _linear("linear_batch", 24, 11008, 4096, 128, "bf16", "bf16"),
        # an odd layer in 32 bits with a bias, rows not on 16-byte boundaries
        _linear("linear_ragged", 333, 1001, 1343, 0, "f32", "f32", bias=True),
        # one calibration sequence through a refined attention projection with
        # groups of 64; activations are a slice of a wider tensor
        _linear("linear_sequence", 2048, 4096, 4096, 64, "f16", "f16", pad=64),
        # two sequences through the widest gate projection, groups of 128
        _linear("linear_gate", 4096, 4096, 14336, 128, "f16", "f16"),
        # evaluation of four sequences through a down projection
        _linear("linear_eval", 8192, 11008, 4096, 0, "bf16", "bf16"),
        # the token just generated and its alternatives
        _score("score_token", 1, 128000, "f32", 1, 8, "none"),
        # four candidate answers at each place, constrained vocabulary, many
        # alternatives, odd vocabulary
        _score("score_choices", 48, 50001, "f16", 4, 20, "rows"),
        # perplexity of four sequences of 2048 tokens
        _score("score_eval", 8192, 32000, "bf16", 1, 0, "none"),
        # perplexity and alternatives over a large vocabulary in 32 bits
        _score("score_wide", 2048, 131072, "f32", 1, 5, "none"),
        # a small batch with an entropy term, odd constrained vocabulary
        _grad("grad_small", 16, 32001, "f16", 2, True, "rows"),
        # a training step's loss over four sequences, padded vocabulary
        _grad("grad_train", 8192, 32000, "bf16", 1, False, "tail"),
    ]


def _log_uniform(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


_MOST_FLOPS = 2 * 8192 * 11008 * 4096
_MOST_BYTES = 4 * 2048 * 131072


def draw(rng):
    kind = rng.choice(["linear", "linear", "score", "grad"])
    x = rng.choice(["f32", "f16", "bf16"])
    while True:
        if kind == "linear":
            g = rng.choice([0, 64, 128])
            din = _log_uniform(rng, 128, 14336)
            if g:
                din = max(g, din // g * g)
            c = _linear("", _log_uniform(rng, 1, 8192), din, _log_uniform(rng, 64, 14336), g, x,
                        rng.choice([x, "f32"]), bias=rng.random() < 0.3, pad=rng.choice([0, 0, 16, 24, 1]))
            fits = 2 * c["n"] * c["din"] * c["dout"] <= _MOST_FLOPS and 4 * c["n"] * c["dout"] <= _MOST_BYTES
        elif kind == "score":
            c = _score("", _log_uniform(rng, 1, 8192), _log_uniform(rng, 1000, 131072), x, rng.choice([1, 1, 2, 4]),
                       rng.choice([0, 1, 5, 8, 20, 32]), rng.choice(["none", "rows", "tail"]))
            fits = BYTES[x] * c["n"] * c["vocab"] <= _MOST_BYTES // 2
        else:
            c = _grad("", _log_uniform(rng, 1, 8192), _log_uniform(rng, 1000, 131072), x, rng.choice([1, 1, 2, 4]),
                      rng.random() < 0.5, rng.choice(["none", "rows", "tail"]))
            fits = 2 * BYTES[x] * c["n"] * c["vocab"] <= _MOST_BYTES
        if fits:
            del c["name"]
            return c


def work(case):
    if case["kind"] == "linear":
        n, din, dout, g = case["n"], case["din"], case["dout"], case["g"]
        return {"bytes": n * din * BYTES[case["x"]] + dout * din + 4 * dout * (din // g if g else 1)
                + (4 * dout if case["bias"] else 0) + n * dout * BYTES[case["y"]],
                "flops": 2 * n * din * dout}
    n, v, t = case["n"], case["vocab"], case["t"]
    b = BYTES[case["x"]]
    if case["kind"] == "score":
        return {"bytes": n * v * b + n * (12 * t + 8 + 8 * case["top"]), "flops": 5 * n * v}
    return {"bytes": 2 * n * v * b + n * (12 * t + 4 + (8 if case["entropy"] else 0)), "flops": 4 * n * v}


# ---------------------------------------------------------------- inputs

def _rows(n, d, pad, dtype):
    """[n][d], rows ``d + pad`` elements apart."""
    return torch.zeros(n, d + pad, dtype=dtype, device=DEV)[:, :d]


def _prepare_linear(case, gen):
    n, din, dout, g, pad = (case[k] for k in ("n", "din", "dout", "g", "pad"))
    randn = lambda *s: torch.randn(*s, generator=gen, device=DEV)
    rand = lambda *s: torch.rand(*s, generator=gen, device=DEV)
    # activations: channels of different size with a few outliers, tokens too
    ch = 0.2 + rand(din)
    ch[torch.randperm(din, generator=gen, device=DEV)[:max(1, din // 256)]] *= 20.0
    X = _rows(n, din, pad, TYPES[case["x"]])
    X.copy_(randn(n, din) * ch * torch.exp(0.5 * randn(n, 1)))
    if n > 8:
        X[n // 2] = 0                      # a padding token
    W = randn(dout, din) * 0.02
    C = _rows(dout, din, pad, torch.int8)
    if g:
        # a refined layer: 4-bit codes minus the group's zero point, signed scales
        Wg = W.view(dout, din // g, g)
        lo, hi = Wg.amin(2), Wg.amax(2)
        ws = (hi - lo) / 15.0
        z = torch.round(-lo / ws).clamp(0, 15)
        q = (torch.round(Wg / ws[:, :, None]) + z[:, :, None]).clamp(0, 15)
        flip = rand(dout, din // g) < 0.02
        ws = torch.where(flip, -ws, ws)
        C.copy_((q - z[:, :, None]).reshape(dout, din))
    else:
        ws = W.abs().amax(1) / 127.0
        C.copy_(torch.round(W / ws[:, None]).clamp(-127, 127))
    bias = randn(dout) * 0.1 if case["bias"] else None
    return {"X": X, "C": C, "ws": ws.contiguous(), "bias": bias}


def _logits(case, gen):
    n, v = case["n"], case["vocab"]
    x = torch.randn(n, v, generator=gen, device=DEV) * 2.5
    # a confident head: some rows have a token far above the others
    real = v - v // 100 if case["mask"] == "tail" else v
    best = torch.randint(0, real, (n,), generator=gen, device=DEV)
    lift = 14.0 * torch.rand(n, generator=gen, device=DEV)
    x.scatter_add_(1, best[:, None], lift[:, None])
    tok = torch.randint(0, real, (n, case["t"]), generator=gen, device=DEV)
    tok[:, 0] = torch.where(torch.rand(n, generator=gen, device=DEV) < 0.5, best, tok[:, 0])
    if case["mask"] == "tail":             # entries that pad the vocabulary
        x[:, real:] = torch.finfo(TYPES[case["x"]]).min
    elif case["mask"] == "rows":           # tokens that a row may not take
        x[torch.rand(n, v, generator=gen, device=DEV) < 0.1] = -math.inf
        x[3::16, 3:] = -math.inf           # three tokens left
        x[5::32] = -math.inf               # none
    if n > 4:
        tok[2::16, 0] = -1                 # places that do not count
    return x.to(TYPES[case["x"]]), tok


def prepare(case, seed):
    gen = torch.Generator(device=DEV).manual_seed(1000003 * int(seed) + 17)
    if case["kind"] == "linear":
        return {"case": case, **_prepare_linear(case, gen)}
    x, tok = _logits(case, gen)
    s = {"case": case, "x": x, "tok": tok}
    if case["kind"] == "grad":
        _, lse, ent = _stats64(x)
        s["lse"], s["entropy"] = lse.float(), ent.float()
        n = case["n"]
        s["g_logprob"] = torch.randn(n, case["t"], generator=gen, device=DEV) / n
        s["g_entropy"] = torch.randn(n, generator=gen, device=DEV) * (0.1 / n) if case["entropy"] else None
    return s


# ---------------------------------------------------------------- plain forms

def _codes(X):
    """int8 codes of every row as float32 integers, and its scale: with a the
    row's largest magnitude, scale a / 127 and round(x (127 / a)), each quotient
    rounded once (a number as a divisor or dividend is not: torch multiplies by
    its reciprocal)."""
    x = X.float()
    a = x.abs().amax(1, keepdim=True)
    live = a > 0
    c = torch.full_like(a, 127.0)
    q = torch.round(x * (c / torch.where(live, a, 1.0)))
    return torch.where(live, q, 0.0), (a / c)[:, 0]


def _plain_linear(s):
    c = s["case"]
    q, xs = _codes(s["X"])
    w = s["C"].float()
    if c["g"]:
        w = (w.reshape(c["dout"], -1, c["g"]) * s["ws"][:, :, None]).reshape(c["dout"], c["din"])
        y = (q @ w.t()) * xs[:, None]
    else:
        y = (q @ w.t()) * xs[:, None] * s["ws"]
    if s["bias"] is not None:
        y = y + s["bias"]
    return {"y": y.to(TYPES[c["y"]])}


def _plain_score(s):
    c, tok = s["case"], s["tok"]
    x = s["x"].float()
    m = x.amax(1, keepdim=True)
    empty = m == -math.inf
    d = x - torch.where(empty, 0.0, m)
    e = torch.exp(d)
    z = e.sum(1, keepdim=True)
    zs = torch.where(empty, 1.0, z)
    logz = torch.log(zs)
    r = {"lse": torch.where(empty, -math.inf, m + logz)[:, 0],
         "entropy": (logz - torch.where(e > 0, e * d, 0.0).sum(1, keepdim=True) / zs)[:, 0]}
    lp = d - logz
    r["logprob"] = torch.where(tok < 0, 0.0, lp.gather(1, tok.clamp(min=0)))
    k = c["top"]
    if k:
        # order: larger logits first, of equal ones the lower token
        b = (x + 0.0).view(torch.int32)
        key = torch.where(b < 0, b ^ 0x7FFFFFFF, b).long() * (1 << 32)
        key += (1 << 31) - torch.arange(x.shape[1], device=x.device)
        i = key.topk(k, dim=1).indices
        v = lp.gather(1, i)
        r["top_logprob"] = v
        r["top_token"] = torch.where(v == -math.inf, -1, i).int()
    return r


def _plain_grad(s):
    tok, x = s["tok"], s["x"].float()
    live = x > -math.inf
    lp = torch.where(live, x - s["lse"][:, None], -math.inf)
    p = torch.exp(lp)
    g = torch.where(tok < 0, 0.0, s["g_logprob"])
    dx = -g.sum(1, keepdim=True) * p
    if s["g_entropy"] is not None:
        dx -= s["g_entropy"][:, None] * torch.where(p > 0, p * (lp + s["entropy"][:, None]), 0.0)
    dx.scatter_add_(1, tok.clamp(min=0), g)
    return {"dx": torch.where(live, dx, 0.0).to(s["x"].dtype)}


def run(state):
    kind = state["case"]["kind"]
    if not own:
        return {"linear": _plain_linear, "score": _plain_score, "grad": _plain_grad}[kind](state)
    from paper_2609_38599_gb300 import jarq
    c = state["case"]
    if kind == "linear":
        return {"y": jarq.integer_linear(state["X"], state["C"], state["ws"], group_size=c["g"],
                                         bias=state["bias"], dtype=str(TYPES[c["y"]])[6:])}
    if kind == "score":
        r = jarq.token_logprobs(state["x"], state["tok"], top=c["top"])
        out = {"lse": r.lse, "entropy": r.entropy, "logprob": r.logprob}
        if c["top"]:
            out.update(top_logprob=r.top_logprob, top_token=r.top_token)
        return out
    return {"dx": jarq.token_logprobs_grad(state["x"], state["tok"], state["lse"], state["g_logprob"],
                                           entropy=state["entropy"], g_entropy=state["g_entropy"])}


# ---------------------------------------------------------------- 64 bits

def _stats64(x):
    """Largest logit, log sum of exponentials and entropy of every row, in 64
    bits, a few rows at a time."""
    out = []
    for part in x.split(max(1, (1 << 26) // x.shape[1])):
        v = part.double()
        m = v.max(1).values
        m0 = torch.where(m > -math.inf, m, torch.zeros_like(m))
        w = torch.exp(v - m0[:, None])
        z = w.sum(1)
        lse = m0 + torch.log(z)                                   # log 0 = -inf: an empty row
        u = torch.where(w > 0, w * (v - m0[:, None]), torch.zeros_like(v)).sum(1)
        ent = torch.where(z > 0, torch.log(z) - u / z, torch.zeros_like(z))
        out.append(torch.stack([m0, lse, ent]))
    return torch.cat(out, 1)


def exact(case, seed):
    s = prepare(case, seed)
    if case["kind"] == "linear":
        # the codes are defined in 32 bits, everything after them is not
        X = s["X"].to(torch.float32)
        top = X.abs().max(1).values
        full = torch.full_like(top, 127.0)
        inv = torch.where(top > 0, torch.div(full, top), torch.zeros_like(top))
        q = (X * inv[:, None]).round().double() * torch.div(top, full).double()[:, None]
        C = s["C"].double()
        ws = s["ws"].double().reshape(case["dout"], -1)
        W = C * ws.repeat_interleave(case["din"] // ws.shape[1], dim=1)
        y = q @ W.t()
        return {"y": y if s["bias"] is None else y + s["bias"].double()}
    x, tok = s["x"], s["tok"]
    if case["kind"] == "score":
        m, lse, ent = _stats64(x)
        empty = lse == -math.inf
        ref = torch.where(empty, torch.zeros_like(lse), lse)[:, None]
        at = x.gather(1, tok.clamp(min=0)).double() - ref
        r = {"lse": lse, "entropy": ent, "logprob": torch.where(tok < 0, torch.zeros_like(at), at)}
        if case["top"]:
            # the values alone: sorted, whatever the order of equal ones
            r["top_logprob"] = torch.stack([part.double().sort(descending=True).values[:case["top"]]
                                            for part in x]) - ref
            r["top_token"] = None
        return r
    lse, ent = s["lse"].double(), s["entropy"].double()
    out = torch.empty(x.shape, dtype=torch.float64, device=x.device)
    step = max(1, (1 << 26) // x.shape[1])
    for a in range(0, case["n"], step):
        b = min(case["n"], a + step)
        v, t = x[a:b].double(), tok[a:b]
        ref = torch.where(lse[a:b] == -math.inf, torch.zeros_like(lse[a:b]), lse[a:b])[:, None]
        p = torch.exp(v - ref)
        onehot = torch.zeros_like(p)
        weight = torch.where(t < 0, torch.zeros_like(s["g_logprob"][a:b]), s["g_logprob"][a:b]).double()
        onehot.scatter_add_(1, t.clamp(min=0), weight)
        d = onehot - p * weight.sum(1, keepdim=True)
        if s["g_entropy"] is not None:
            h = torch.where(p > 0, p * (v - ref + ent[a:b, None]), torch.zeros_like(p))
            d = d - s["g_entropy"][a:b, None].double() * h
        out[a:b] = torch.where(v == -math.inf, torch.zeros_like(d), d)
    return {"dx": out}
