"""Performance cases of the operators around a quantized model's layers:

``norm``        root-mean-square norm of rows with the residual's addition, as
                values, as 8-bit integers with a scale a row, or both;
``norm_grad``   its gradient;
``loss``        softmax cross entropy of an output head's hidden states, in
                pieces of the vocabulary, without keeping the logits;
``loss_grad``   the same with its gradients, as a training step calls it;
``adapt``       low-rank adapters of many requests added to a shared
                projection's outputs.

``run`` computes each in plain torch operations in 32 bits (``own`` false) or
through the library's entry points (``own`` true).  ``exact`` is the same from
the definitions in 64 bits.  Layer widths are those of ``synth/layers.py`` and
the benchmark, and ranges around them; vocabularies, ranks and numbers of
requests are generic.  Inputs are drawn on the GPU from the seed alone.
"""
import math

import torch

own = False

DEV = "cuda"
TYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
BYTES = {"f32": 4, "f16": 2, "bf16": 2}
EPS = 1e-5


# ---------------------------------------------------------------- the cases

def _norm(name, n, d, x, residual, out, pad=0):
    """``out``: "y" values, "q" 8-bit integers with scales, "yq" both; ``pad``:
    columns by which the rows of the activations lie further apart."""
    return {"name": name, "kind": "norm", "n": n, "d": d, "x": x, "residual": residual, "out": out, "pad": pad}


def _norm_grad(name, n, d, x, residual, pad=0):
    """``residual``: a gradient arrives at the sum beside the norm's."""
    return {"name": name, "kind": "norm_grad", "n": n, "d": d, "x": x, "residual": residual, "pad": pad}


def _loss(name, n, d, vocab, x, pad=0):
    return {"name": name, "kind": "loss", "n": n, "d": d, "vocab": vocab, "x": x, "pad": pad}


def _loss_grad(name, n, d, vocab, x, grads, pad=0):
    """``grads``: "x" of the hidden states (a frozen head), "w" of the head, "xw"."""
    return {"name": name, "kind": "loss_grad", "n": n, "d": d, "vocab": vocab, "x": x, "grads": grads, "pad": pad}


def _adapt(name, n, din, dout, rank, adapters, x, y, order):
    """``order``: the tokens' adapters: "runs" a run of tokens a request, "each"
    one token a request, in any order."""
    return {"name": name, "kind": "adapt", "n": n, "din": din, "dout": dout, "rank": rank, "adapters": adapters,
            "x": x, "y": y, "order": order}


def listed():
    return [
        # generation for a single user: the norm before a projection
        _norm("norm_token", 1, 4096, "f16", True, "y"),
        # odd rows in 32 bits, not on 16-byte boundaries, values and integers
        _norm("norm_ragged", 333, 1001, "f32", False, "yq"),
        # prompts of 8192 tokens before a refined layer in 8-bit integers
        _norm("norm_prompts", 8192, 4096, "bf16", True, "q"),
        # tuning on a few short answers, the width of a down projection's input
        _norm_grad("norm_grad_small", 48, 11008, "f16", False),
        # a training step over four sequences
        _norm_grad("norm_grad_train", 8192, 4096, "bf16", True),
        # candidate answers scored, odd vocabulary
        _loss("loss_answers", 48, 2048, 50001, "f16"),
        # perplexity of one sequence
        _loss("loss_eval", 2048, 4096, 32000, "bf16"),
        # tuning below a frozen head, odd vocabulary, hidden states a slice of a wider tensor
        _loss_grad("loss_grad_frozen", 1000, 1344, 50001, "f16", "x", pad=64),
        # a training step over four sequences
        _loss_grad("loss_grad_train", 8192, 4096, 32000, "bf16", "xw"),
        # the token of one user beside an up projection
        _adapt("adapt_token", 1, 4096, 11008, 16, 4, "f16", "f16", "each"),
        # one step of generation for many users beside a down projection
        _adapt("adapt_batch", 48, 11008, 4096, 16, 32, "bf16", "bf16", "each"),
        # the prompts of a few users beside an attention projection
        _adapt("adapt_prompts", 8192, 4096, 4096, 16, 6, "bf16", "bf16", "runs"),
    ]


def _log_uniform(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


_MOST = {"norm": 8192 * 4096, "norm_grad": 8192 * 4096, "loss": 8192 * 4096 * 32000,
         "loss_grad": 8192 * 4096 * 32000, "adapt": 8192 * 8192}


def draw(rng):
    kind = rng.choice(["norm", "norm_grad", "loss", "loss_grad", "adapt"])
    x = rng.choice(["f32", "f16", "bf16"] if kind in ("norm", "norm_grad") else ["f16", "bf16"])
    pad = rng.choice([0, 0, 0, 16, 24, 1])
    while True:
        n = _log_uniform(rng, 1, 8192)
        if kind in ("norm", "norm_grad"):
            d = _log_uniform(rng, 64, 14336)
            c = (_norm("", n, d, x, rng.random() < 0.6, rng.choice(["y", "q", "yq"]), pad) if kind == "norm"
                 else _norm_grad("", n, d, x, rng.random() < 0.6, pad))
            size = n * d * BYTES[x] // 2
        elif kind in ("loss", "loss_grad"):
            # most heads are of a width that is a multiple of eight
            d = _log_uniform(rng, 64, 8192)
            d = d if rng.random() < 0.2 else (d + 7) // 8 * 8
            v = _log_uniform(rng, 1000, 131072)
            c = (_loss("", n, d, v, x, pad) if kind == "loss"
                 else _loss_grad("", n, d, v, x, rng.choice(["x", "w", "xw"]), pad))
            size = max(n * d * v, 64 * n * v, 64 * d * v)
        else:
            din, dout = _log_uniform(rng, 64, 14336), _log_uniform(rng, 64, 14336)
            c = _adapt("", n, din, dout, rng.choice([8, 16, 32, 64]), _log_uniform(rng, 1, 64), x,
                       rng.choice([x, "f32"]), rng.choice(["runs", "each"]))
            size = n * (din + dout * BYTES[c["y"]] // 2)
        if size <= _MOST[kind]:
            del c["name"]
            return c


def work(case):
    kind, n = case["kind"], case["n"]
    b = BYTES[case["x"]]
    if kind == "norm":
        d, size = case["d"], b * (3 if case["residual"] else 1)
        size += (b if "y" in case["out"] else 0) + (1 if "q" in case["out"] else 0)
        return {"bytes": n * d * size + b * d + n * (4 + (4 if "q" in case["out"] else 0)), "flops": 6 * n * d}
    if kind == "norm_grad":
        d = case["d"]
        return {"bytes": n * d * b * (4 if case["residual"] else 3) + (b + 4) * d + 4 * n, "flops": 10 * n * d}
    if kind == "loss":
        d, v = case["d"], case["vocab"]
        return {"bytes": (n + v) * d * b + 16 * n, "flops": 2 * n * v * d}
    if kind == "loss_grad":
        d, v = case["d"], case["vocab"]
        grads = (n if "x" in case["grads"] else 0) + (v if "w" in case["grads"] else 0)
        return {"bytes": (n + v + grads) * d * b + 20 * n, "flops": 2 * n * v * d * (1 + len(case["grads"]))}
    din, dout, r = case["din"], case["dout"], case["rank"]
    used = min(case["adapters"], n)
    return {"bytes": n * (din * b + 2 * dout * BYTES[case["y"]] + 4) + used * (r * (din + dout) * b + 4),
            "flops": 2 * n * r * (din + dout)}


# ---------------------------------------------------------------- inputs

def _rows(x, pad, dtype):
    """The matrix ``x`` in ``dtype``, its rows ``pad`` elements further apart."""
    n, d = x.shape
    out = torch.zeros(n, d + pad, dtype=dtype, device=DEV)[:, :d]
    return out.copy_(x)


def _activations(n, d, gen):
    """Channels of different size with a few outliers, tokens too."""
    ch = 0.2 + torch.rand(d, generator=gen, device=DEV)
    ch[torch.randperm(d, generator=gen, device=DEV)[:max(1, d // 256)]] *= 20.0
    x = torch.randn(n, d, generator=gen, device=DEV) * ch
    return x * torch.exp(0.5 * torch.randn(n, 1, generator=gen, device=DEV))


def _prepare_norm(case, gen):
    n, d, pad, t = case["n"], case["d"], case["pad"], TYPES[case["x"]]
    x = _rows(_activations(n, d, gen), pad, t)
    gain = (0.3 + torch.rand(d, generator=gen, device=DEV)).to(t)
    if case["kind"] == "norm":
        if n > 8:
            x[n // 2] = 0                          # a padding token
        r = _rows(4.0 * torch.randn(n, d, generator=gen, device=DEV), pad, t) if case["residual"] else None
        if r is not None and n > 8:
            r[n // 2] = 0
        return {"x": x, "gain": gain, "r": r}
    rstd = (x.double().square().mean(1) + EPS).rsqrt().float()
    dy = _rows(torch.randn(n, d, generator=gen, device=DEV) * 1e-2, pad, t)
    dh = _rows(torch.randn(n, d, generator=gen, device=DEV) * 1e-2, pad, t) if case["residual"] else None
    return {"h": x, "gain": gain, "rstd": rstd, "dy": dy, "dh": dh}


def _prepare_loss(case, gen):
    n, d, v, pad, t = case["n"], case["d"], case["vocab"], case["pad"], TYPES[case["x"]]
    w = (torch.randn(v, d, generator=gen, device=DEV) * (2.5 / math.sqrt(d))).to(t)
    tok = torch.randint(0, v, (n,), generator=gen, device=DEV)
    # a head that has learnt something: the token's logit is lifted by up to 14
    lift = 14.0 / 6.25 * torch.rand(n, 1, generator=gen, device=DEV)
    x = _rows(torch.randn(n, d, generator=gen, device=DEV) + lift * w[tok].float(), pad, t)
    if n > 4:
        tok[2::16] = -1                            # places that do not count
    s = {"x": x, "w": w, "tok": tok}
    if case["kind"] == "loss_grad":
        s["g"] = torch.rand(n, generator=gen, device=DEV) / n
    return s


def _prepare_adapt(case, gen):
    n, din, dout, r, m = (case[k] for k in ("n", "din", "dout", "rank", "adapters"))
    t = TYPES[case["x"]]
    randn = lambda *s: torch.randn(*s, generator=gen, device=DEV)
    ids = torch.randint(0, m, (n,), generator=gen, device=DEV, dtype=torch.int32)
    if case["order"] == "runs":
        ids = ids[torch.randint(0, n, (min(m, n),), generator=gen, device=DEV).sort().values]
        cut = torch.randint(0, n, (ids.numel(),), generator=gen, device=DEV)
        ids = ids[torch.bucketize(torch.arange(n, device=DEV), cut.sort().values).clamp(max=ids.numel() - 1)]
    if n > 8:
        ids[n // 2: n // 2 + max(1, n // 16)] = -1     # a request without an adapter
    return {"x": _activations(n, din, gen).to(t), "a": (randn(m, r, din) / math.sqrt(din)).to(t),
            "b": (randn(m, dout, r) * 0.2).to(t), "scale": 0.5 + torch.rand(m, generator=gen, device=DEV),
            "ids": ids.contiguous(), "base": randn(n, dout).to(TYPES[case["y"]])}


def prepare(case, seed):
    gen = torch.Generator(device=DEV).manual_seed(1000003 * int(seed) + 29)
    kind = case["kind"]
    made = (_prepare_norm if kind.startswith("norm") else _prepare_loss if kind.startswith("loss") else _prepare_adapt)
    return {"case": case, **made(case, gen)}


# ---------------------------------------------------------------- plain forms

def _plain_norm(s):
    c, x = s["case"], s["x"].float()
    t, out = s["x"].dtype, {}
    if s["r"] is not None:
        h = (x + s["r"].float()).to(t)             # the sum as the next layer reads it
        out["h"], x = h, h.float()
    rstd = 1.0 / torch.sqrt((x * x).mean(1, keepdim=True) + EPS)
    out["rstd"] = rstd[:, 0]
    v = x * s["gain"].float()
    if "y" in c["out"]:
        out["y"] = (v * rstd).to(t)
    if "q" in c["out"]:
        # the row's own factor goes into its scale, so the integers are those of
        # v: with a the row's largest magnitude, round(v (127 / a)), each
        # quotient and product rounded once to 32 bits
        a = v.abs().amax(1, keepdim=True)
        full, live = torch.full_like(a, 127.0), a > 0
        q = torch.where(live, torch.round(v * (full / torch.where(live, a, 1.0))), 0.0)
        out["q"] = q * (a / full * rstd)
    return out


def _plain_norm_grad(s):
    h, dy, r = s["h"].float(), s["dy"].float(), s["rstd"][:, None]
    u = dy * s["gain"].float()
    dx = r * (u - h * (r * r * (u * h).mean(1, keepdim=True)))
    if s["dh"] is not None:
        dx = dx + s["dh"].float()
    return {"dx": dx.to(s["h"].dtype), "dgain": (dy * h * r).sum(0)}


def _plain_loss(s):
    x, w, tok = s["x"].float(), s["w"].float(), s["tok"]
    logits = x @ w.t()
    m = logits.amax(1, keepdim=True)
    e = torch.exp(logits - m)
    z = e.sum(1, keepdim=True)
    at = logits.gather(1, tok.clamp(min=0)[:, None])
    out = {"loss": torch.where(tok < 0, 0.0, (torch.log(z) + (m - at))[:, 0]), "lse": (m + torch.log(z))[:, 0]}
    if s["case"]["kind"] == "loss_grad":
        g = torch.where(tok < 0, 0.0, s["g"])[:, None]
        e *= g / z
        e.scatter_add_(1, tok.clamp(min=0)[:, None], -g)
        if "x" in s["case"]["grads"]:
            out["dx"] = (e @ w).to(s["x"].dtype)
        if "w" in s["case"]["grads"]:
            out["dw"] = (e.t() @ x).to(s["x"].dtype)
    return out


def _plain_adapt(s):
    n, r, m = s["case"]["n"], s["case"]["rank"], s["case"]["adapters"]
    a, b = s["a"].float(), s["b"].float()
    # every adapter for every token; of these a token keeps its own
    u = (s["x"].float() @ a.reshape(m * r, -1).t()).reshape(n, m, r)
    mine = s["ids"][:, None] == torch.arange(m, device=DEV)
    u = u * torch.where(mine, s["scale"], 0.0)[:, :, None]
    y = s["base"].float() + u.reshape(n, m * r) @ b.transpose(1, 2).reshape(m * r, -1)
    return {"y": y.to(s["base"].dtype)}


def run(state):
    c = state["case"]
    kind = c["kind"]
    if not own:
        return {"norm": _plain_norm, "norm_grad": _plain_norm_grad, "loss": _plain_loss,
                "loss_grad": _plain_loss, "adapt": _plain_adapt}[kind](state)
    from paper_2609_38599_gb300 import jarq
    if kind == "norm":
        r = jarq.rms_norm(state["x"], state["gain"], eps=EPS, residual=state["r"], values="y" in c["out"],
                          codes="q" in c["out"])
        out = {} if state["r"] is None else {"h": r.h}
        out["rstd"] = r.rstd
        if "y" in c["out"]:
            out["y"] = r.y
        if "q" in c["out"]:
            out["q"] = r.codes * r.scale[:, None]          # what the integers stand for
        return out
    if kind == "norm_grad":
        dx, dgain = jarq.rms_norm_grad(state["h"], state["gain"], state["rstd"], state["dy"], dh=state["dh"])
        return {"dx": dx, "dgain": dgain}
    if kind in ("loss", "loss_grad"):
        loss, lse = jarq.cross_entropy(state["x"], state["w"], state["tok"])
        out = {"loss": loss, "lse": lse}
        if kind == "loss_grad":
            dx, dw = jarq.cross_entropy_grad(state["x"], state["w"], state["tok"], lse, state["g"],
                                             hidden="x" in c["grads"], head="w" in c["grads"])
            out.update({k: v for k, v in (("dx", dx), ("dw", dw)) if v is not None})
        return out
    return {"y": jarq.apply_adapters(state["x"], state["a"], state["b"], state["ids"], scale=state["scale"],
                                     base=state["base"])}


# ---------------------------------------------------------------- 64 bits

def _exact_norm(s):
    out, h = {}, s["x"].double()
    if s["r"] is not None:
        out["h"] = h + s["r"].double()
        h = out["h"].to(s["x"].dtype).double()     # the norm is defined on the rounded sum
    out["rstd"] = torch.pow(h.pow(2).sum(1) / h.shape[1] + EPS, -0.5)
    v = h * s["gain"].double()
    if "y" in s["case"]["out"]:
        out["y"] = v * out["rstd"][:, None]
    if "q" in s["case"]["out"]:
        # the integers are defined in 32 bits, what they stand for is not
        v = v.float()
        top = v.abs().max(1).values
        inv = torch.where(top > 0, torch.div(torch.full_like(top, 127.0), top), torch.zeros_like(top))
        out["q"] = (v * inv[:, None]).round().double() * (top.double() / 127.0 * out["rstd"])[:, None]
    return out


def _exact_norm_grad(s):
    h, dy, r = s["h"].double(), s["dy"].double(), s["rstd"].double()
    gained = dy * s["gain"].double()
    along = torch.einsum("td,td->t", gained, h) / h.shape[1]
    dx = r[:, None] * gained - (r.pow(3) * along)[:, None] * h
    if s["dh"] is not None:
        dx = dx + s["dh"].double()
    return {"dx": dx, "dgain": torch.einsum("td,td,t->d", dy, h, r)}


def _exact_loss(s):
    c, x, w, tok = s["case"], s["x"].double(), s["w"].double(), s["tok"]
    counts = tok >= 0
    logits = torch.matmul(x, w.transpose(0, 1))
    lse = torch.logsumexp(logits, 1)
    mine = logits[torch.arange(len(tok), device=DEV), torch.where(counts, tok, 0)]
    out = {"loss": torch.where(counts, lse - mine, 0.0), "lse": lse}
    if c["kind"] == "loss_grad":
        p = logits.sub_(lse[:, None]).exp_()
        p[counts.nonzero()[:, 0], tok[counts]] -= 1.0
        p *= torch.where(counts, s["g"], 0.0).double()[:, None]
        if "x" in c["grads"]:
            out["dx"] = torch.matmul(p, w)
        if "w" in c["grads"]:
            out["dw"] = torch.matmul(p.transpose(0, 1), x)
    return out


def _exact_adapt(s):
    y = s["base"].double().clone()
    for i in range(s["case"]["adapters"]):
        at = (s["ids"] == i).nonzero()[:, 0]
        if len(at):
            u = torch.matmul(s["x"][at].double(), s["a"][i].double().T)
            y[at] += s["scale"][i].double() * torch.matmul(u, s["b"][i].double().T)
    return {"y": y}


def exact(case, seed):
    kind, s = case["kind"], prepare(case, seed)
    return {"norm": _exact_norm, "norm_grad": _exact_norm_grad, "loss": _exact_loss,
            "loss_grad": _exact_loss, "adapt": _exact_adapt}[kind](s)
