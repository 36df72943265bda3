"""Cases for measuring the operators at the two ends of a language model's step:
token embedding, normalisation and token loss, each with its gradient.

They stand around the linear modules whose inputs and output gradients the
library compresses: the embedding begins the forward pass, a normalisation
writes the input of most modules, and the loss gradient begins the backward
pass. Every operator works on B examples of T tokens; `lengths` leaves the
positions from lengths[b] on out (padding), whatever they hold.

`run` computes them in elementary torch operations in 32 bits, or, with `own`
set, through the library's calls.
"""
import math

import numpy as np
import torch

own = False

_TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
_SIZES = {"f32": 4, "bf16": 2}
IGNORE = -100


# ------------------------------------------------------------------- cases
def listed():
    return [
        # one token of a model being served: a table row and its position's row
        dict(name="embed_token", op="embed", B=1, T=1, V=50_000, d=768, dtype="bf16", index="i64", pos=True,
             scale=1.0, ragged=False),
        # the batch of the 4096-wide stack that is compressed at a time, examples of several lengths
        dict(name="embed_batch", op="embed", B=32, T=2048, V=100_000, d=4096, dtype="bf16", index="i64", pos=False,
             scale=64.0, ragged=True),
        # the embedding's gradient for one example, odd length and width, 32-bit model
        dict(name="embed_grad_example", op="embed_grad", B=1, T=509, V=32_001, d=770, dtype="f32", grad="f32",
             index="i32", scale=1.0, ragged=False),
        # a training batch of the 768-wide stack (512 examples of up to 512 tokens)
        dict(name="embed_grad_batch", op="embed_grad", B=512, T=512, V=50_000, d=768, dtype="bf16", grad="f32",
             index="i64", scale=1.0, ragged=True),
        # one token of a model being served
        dict(name="norm_token", op="norm", B=1, T=1, d=4096, dtype="bf16", kind="rms", ragged=False),
        # the input of a module of the 4096-wide stack, one batch
        dict(name="norm_batch", op="norm", B=32, T=2048, d=4096, dtype="bf16", kind="layer", ragged=False),
        # backward through one normalisation for a single example, odd width, 32-bit model
        dict(name="norm_grad_example", op="norm_grad", B=1, T=511, d=770, dtype="f32", kind="layer",
             per_example=False, ragged=False),
        # backward for one batch of the 4096-wide stack
        dict(name="norm_grad_batch", op="norm_grad", B=32, T=2048, d=4096, dtype="bf16", kind="rms",
             per_example=False, ragged=False),
        # backward for one batch of the 768-wide stack, with each example's own weight gradient
        dict(name="norm_grad_each", op="norm_grad", B=512, T=512, d=768, dtype="bf16", kind="layer",
             per_example=True, ragged=True),
        # the loss of a short answer alone, 32-bit logits over an odd vocabulary
        dict(name="loss_answer", op="loss", B=1, T=37, V=50_001, dtype="f32", index="i64", gradient=False,
             weighted=False, masked=0, prompt=0, ragged=False),
        # one example's loss and the gradient that starts its backward pass, odd vocabulary
        dict(name="loss_example", op="loss", B=1, T=511, V=50_001, dtype="bf16", index="i64", gradient=True,
             weighted=False, masked=0, prompt=64, ragged=False),
        # a training batch of conversations: prompts not counted, several lengths, a vocabulary padded with masked columns
        dict(name="loss_batch", op="loss", B=4, T=2048, V=100_096, dtype="bf16", index="i64", gradient=True,
             weighted=True, masked=96, prompt=256, ragged=True),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _width(rng, lo, hi):
    """Model widths: mostly multiples of 64, some of 8, some odd."""
    d = _log(rng, lo, hi)
    step = rng.choice([64, 64, 64, 8, 1])
    return max(step, d // step * step)


def _batch(rng, most):
    """B and T with at most `most` tokens, from a single one on."""
    tokens = _log(rng, 1, most)
    T = min(tokens, _log(rng, 1, 4096))
    return max(1, tokens // T), T


def draw(rng):
    op = rng.choice(["embed", "embed_grad", "norm", "norm_grad", "loss"])
    dtype = rng.choice(["bf16", "bf16", "f32"])
    c = dict(op=op, dtype=dtype, ragged=rng.random() < 0.5)
    es = _SIZES[dtype]
    if op == "loss":
        V = _log(rng, 1000, 131_072)
        gradient = rng.random() < 0.75
        B, T = _batch(rng, min(65_536, max(1, int(1.2e9 / (V * es * (2 if gradient else 1))))))
        c.update(B=B, T=T, V=V, index=rng.choice(["i64", "i32"]), gradient=gradient, weighted=rng.random() < 0.5,
                 masked=rng.choice([0, V // 50]), prompt=rng.choice([0, T // 4]))
        return c
    d = _width(rng, 64, 8192)
    B, T = _batch(rng, min(262_144, max(1, int(5e8 / (d * es)))))
    c.update(B=B, T=T, d=d)
    if op in ("embed", "embed_grad"):
        c.update(V=min(_log(rng, 500, 131_072), int(4e8 / d)), index=rng.choice(["i64", "i32"]),
                 scale=rng.choice([1.0, math.sqrt(d)]))
        c.update(dict(pos=rng.random() < 0.5) if op == "embed" else dict(grad=rng.choice(["f32", "f32", dtype])))
    else:
        c.update(kind=rng.choice(["layer", "rms"]))
        if op == "norm_grad":
            c.update(per_example=rng.random() < 0.5)
    return c


def _lengths(c):
    """Tokens kept of each example: all, or from none to all of them, spread evenly; the seed only orders them."""
    B, T = c["B"], c["T"]
    if not c["ragged"]:
        return [T] * B
    return [T if b == 0 else 0 if b == 1 else max(1, round(T * (0.25 + 0.75 * ((b * 0.6180339887) % 1.0))))
            for b in range(B)]


# ------------------------------------------------------------------ inputs
def _gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def _tokens(c, g, V):
    """Token numbers with the frequencies of text: rank r about as often as 1/r, the ranks spread over the table."""
    u = torch.rand((c["B"], c["T"]), generator=g, device="cuda", dtype=torch.float64)
    rank = torch.exp(u * math.log(V + 1)).long().sub_(1).clamp_(0, V - 1)
    step = next(s for s in range(V // 3 | 1, 2 * V + 3, 2) if math.gcd(s, V) == 1) if V > 1 else 1
    tok = (rank * step + 17) % V
    return tok.to(torch.int32 if c["index"] == "i32" else torch.int64)


def _hidden(c, g):
    """A residual stream: unit scale, tokens of different size, a few channels much larger, an offset."""
    x = torch.randn((c["B"], c["T"], c["d"]), generator=g, device="cuda")
    x.mul_(0.5 + 2.0 * torch.rand((c["B"], c["T"], 1), generator=g, device="cuda"))
    gain = torch.ones(c["d"], device="cuda")
    gain[:: max(1, c["d"] // 6)] = 12.0
    return x.mul_(gain).add_(0.2).to(_TYPES[c["dtype"]])


def _pad(x, st, value):
    """Positions past an example's length hold what was there before."""
    if st["keep"] is not None:
        x.masked_fill_(~st["keep"][..., None], value)
    return x


def prepare(case, seed):
    c, g = case, _gen(seed)
    st = dict(case=c, lengths=None, keep=None)
    ln = _lengths(c)
    if c["ragged"]:
        order = torch.randperm(c["B"], generator=g, device="cuda")
        st["lengths"] = torch.tensor(ln, dtype=torch.int32, device="cuda")[order].contiguous()
        st["keep"] = torch.arange(c["T"], device="cuda")[None] < st["lengths"][:, None]
    op, dt = c["op"], _TYPES[c["dtype"]]
    if op == "embed":
        st["tokens"] = _tokens(c, g, c["V"])
        st["table"] = (0.02 * torch.randn((c["V"], c["d"]), generator=g, device="cuda")).to(dt)
        st["pos"] = (0.01 * torch.randn((c["T"], c["d"]), generator=g, device="cuda")).to(dt) if c["pos"] else None
    elif op == "embed_grad":
        st["tokens"] = _tokens(c, g, c["V"])
        st["dout"] = _pad((1e-3 * torch.randn((c["B"], c["T"], c["d"]), generator=g, device="cuda")).to(dt), st,
                          float("nan"))
    elif op in ("norm", "norm_grad"):
        st["x"] = _pad(_hidden(c, g), st, float("nan"))
        st["weight"] = (1.0 + 0.2 * torch.randn(c["d"], generator=g, device="cuda")).to(dt)
        st["bias"] = (0.1 * torch.randn(c["d"], generator=g, device="cuda")).to(dt) if c["kind"] == "layer" else None
        if op == "norm_grad":
            st["dy"] = _pad((1e-2 * torch.randn((c["B"], c["T"], c["d"]), generator=g, device="cuda")).to(dt), st,
                            float("inf"))
            _, st["mean"], st["rstd"] = _norm(st)
    else:
        V = c["V"]
        x = torch.randn((c["B"], c["T"], V), generator=g, device="cuda").mul_(2.5)
        tgt = torch.randint(0, V - c["masked"], (c["B"], c["T"]), generator=g, device="cuda")
        sure = 12.0 * torch.rand((c["B"], c["T"], 1), generator=g, device="cuda")
        x.scatter_add_(2, tgt[..., None], sure)
        if c["masked"]:
            x[..., V - c["masked"]:] = float("-inf")
        st["logits"] = _pad(x.to(dt), st, float("nan"))
        tgt[:, : c["prompt"]] = IGNORE
        st["targets"] = tgt.to(torch.int32 if c["index"] == "i32" else torch.int64)
        st["weights"] = 0.5 + torch.rand((c["B"], c["T"]), generator=g, device="cuda") if c["weighted"] else None
    return st


# -------------------------------------------------------------- plain forms
def _kept(st, v, other=0.0):
    return v if st["keep"] is None else torch.where(st["keep"][..., None] if v.dim() == 3 else st["keep"], v, other)


def _embed(st):
    c = st["case"]
    out = st["table"][st["tokens"].long()].float() * c["scale"]
    if st["pos"] is not None:
        out = out + st["pos"].float()
    return _kept(st, out).to(st["table"].dtype)


def _embed_grad(st):
    c = st["case"]
    rows = _kept(st, st["dout"].float()).reshape(-1, c["d"])
    grad = torch.zeros((c["V"], c["d"]), device="cuda")
    grad.index_add_(0, st["tokens"].reshape(-1).long(), rows)
    return (grad * c["scale"]).to(_TYPES[c["grad"]])


def _eps(c):
    return 1e-5 if c["kind"] == "layer" else 1e-6


def _norm(st):
    c = st["case"]
    x = st["x"].float()
    mean = x.mean(-1) if c["kind"] == "layer" else None
    xc = x if mean is None else x - mean[..., None]
    rstd = 1.0 / torch.sqrt((xc * xc).mean(-1) + _eps(c))
    y = xc * rstd[..., None] * st["weight"].float()
    if st["bias"] is not None:
        y = y + st["bias"].float()
    return _kept(st, y).to(st["x"].dtype), None if mean is None else _kept(st, mean), _kept(st, rstd)


def _norm_grad(st):
    c = st["case"]
    dy, x, rstd = _kept(st, st["dy"].float()), _kept(st, st["x"].float()), st["rstd"][..., None]
    xhat = (x if st["mean"] is None else x - st["mean"][..., None]) * rstd
    g = dy * st["weight"].float()
    t = g - xhat * (g * xhat).mean(-1, keepdim=True)
    if c["kind"] == "layer":
        t = t - g.mean(-1, keepdim=True)
    over = (1,) if c["per_example"] else (0, 1)
    dw = (dy * xhat).sum(over)
    db = dy.sum(over) if c["kind"] == "layer" else None
    return _kept(st, t * rstd).to(st["x"].dtype), dw, db


def _loss(st):
    c = st["case"]
    counted = st["targets"] != IGNORE
    if st["keep"] is not None:
        counted = counted & st["keep"]
    tgt = torch.where(counted, st["targets"].long(), 0)
    x = torch.where(counted[..., None], st["logits"].float(), 0.0)
    top = x.amax(-1, keepdim=True)
    e = torch.exp(x - top)
    s = e.sum(-1, keepdim=True)
    lse = (top + torch.log(s))[..., 0]
    w = counted.float() if st["weights"] is None else torch.where(counted, st["weights"], 0.0)
    loss = w * (lse - x.gather(-1, tgt[..., None])[..., 0])
    lse = torch.where(counted, lse, 0.0)
    if not c["gradient"]:
        return loss, lse
    e.mul_((w[..., None] / s))
    e.scatter_add_(-1, tgt[..., None], -w[..., None])
    return loss, lse, e.to(st["logits"].dtype)


def run(state):
    st, c = state, state["case"]
    if not own:
        return {"embed": _embed, "embed_grad": _embed_grad, "norm": _norm, "norm_grad": _norm_grad,
                "loss": _loss}[c["op"]](st)
    from paper_2609_37842_gb300 import eogp as E
    op = c["op"]
    if op == "embed":
        return E.embed(st["tokens"], st["table"], scale=c["scale"], pos=st["pos"], lengths=st["lengths"])
    if op == "embed_grad":
        return E.embed_grad(st["tokens"], st["dout"], c["V"], scale=c["scale"], lengths=st["lengths"],
                            dtype=_TYPES[c["grad"]])
    kind = E.NORM_RMS if c.get("kind") == "rms" else E.NORM_LAYER
    if op == "norm":
        return E.norm(st["x"], st["weight"], st["bias"], kind=kind, eps=_eps(c), lengths=st["lengths"])
    if op == "norm_grad":
        return E.norm_grad(st["dy"], st["x"], st["mean"], st["rstd"], st["weight"], kind=kind,
                           lengths=st["lengths"], per_example=c["per_example"], want_dbias=c["kind"] == "layer")
    loss, lse, dlogits = E.cross_entropy(st["logits"], st["targets"], weights=st["weights"], lengths=st["lengths"],
                                         ignore_index=IGNORE, want_grad=c["gradient"])
    return (loss, lse, dlogits) if c["gradient"] else (loss, lse)


# --------------------------------------------------------------------- work
def _distinct(n, V):
    """Expected number of different tokens among n of _tokens'."""
    r = np.arange(1, V + 1, dtype=np.float64)
    p = np.log1p(1.0 / r) / math.log(V + 1)
    return float(np.sum(-np.expm1(n * np.log1p(-np.minimum(p, 1 - 1e-12)))))


def work(case):
    c = case
    op, es = c["op"], _SIZES[c["dtype"]]
    M, n = c["B"] * c["T"], sum(_lengths(c))
    ix = 4 if c.get("index") == "i32" else 8
    if op == "embed":
        rows = _distinct(n, c["V"]) + (max(_lengths(c)) if c["pos"] else 0)
        return {"bytes": n * ix + (rows + M) * c["d"] * es, "flops": n * c["d"] * (2 if c["pos"] else 1)}
    if op == "embed_grad":
        return {"bytes": n * ix + n * c["d"] * es + c["V"] * c["d"] * _SIZES[c["grad"]], "flops": n * c["d"]}
    layer = c.get("kind") == "layer"
    if op == "norm":
        return {"bytes": (n + M) * c["d"] * es + M * (8 if layer else 4) + c["d"] * es * (2 if layer else 1),
                "flops": n * c["d"] * (8 if layer else 4)}
    if op == "norm_grad":
        sums = (c["B"] if c["per_example"] else 1) * c["d"] * 4 * (2 if layer else 1)
        return {"bytes": (2 * n + M) * c["d"] * es + n * (8 if layer else 4) + c["d"] * es + sums,
                "flops": n * c["d"] * (13 if layer else 9)}
    m = sum(max(0, t - c["prompt"]) for t in _lengths(c))
    g = M * c["V"] * es if c["gradient"] else 0
    return {"bytes": m * c["V"] * es + g + n * ix + M * 8 + (m * 4 if c["weighted"] else 0),
            "flops": m * c["V"] * (6 if c["gradient"] else 4)}


# ------------------------------------------------------------------ 64 bits
def exact(case, seed):
    st, c = prepare(case, seed), case
    op = c["op"]
    keep = st["keep"] if st["keep"] is not None else torch.ones((c["B"], c["T"]), dtype=torch.bool, device="cuda")
    if op == "embed":
        out = torch.zeros((c["B"], c["T"], c["d"]), dtype=torch.float64, device="cuda")
        b, t = keep.nonzero(as_tuple=True)
        rows = st["table"].double().index_select(0, st["tokens"][b, t].long()) * c["scale"]
        out[b, t] = rows if st["pos"] is None else rows + st["pos"].double()[t]
        return out
    if op == "embed_grad":
        # sorted by token, each token's sum is a difference of the running sum
        tok = st["tokens"][keep].long()
        tok, order = torch.sort(tok, stable=True)
        run_sum = torch.zeros((tok.numel() + 1, c["d"]), dtype=torch.float64, device="cuda")
        run_sum[1:] = st["dout"][keep][order].double()
        torch.cumsum(run_sum, 0, out=run_sum)
        ends = torch.searchsorted(tok, torch.arange(c["V"] + 1, device="cuda"))
        grad = run_sum[ends[1:]]
        grad -= run_sum[ends[:-1]]
        return grad.mul_(c["scale"])
    if op in ("norm", "norm_grad"):
        x = st["x"].double().masked_fill(~keep[..., None], 1.0).requires_grad_(op == "norm_grad")
        groups = c["B"] if c.get("per_example") else 1
        w = st["weight"].double().expand(groups, c["d"]).clone().requires_grad_(op == "norm_grad")
        v, m = torch.var_mean(x, -1, unbiased=False)
        if c["kind"] == "layer":
            r = torch.rsqrt(v + _eps(c))
            xhat = (x - m[..., None]) * r[..., None]
        else:
            r = torch.rsqrt(torch.linalg.vector_norm(x, dim=-1) ** 2 / c["d"] + _eps(c))
            xhat = x * r[..., None]
        if op == "norm":
            y = xhat * w[0]
            if st["bias"] is not None:
                y = y + st["bias"].double()
            zero = (~keep).double() * 0 + keep.double()
            return (y * zero[..., None], m * zero if c["kind"] == "layer" else None, r * zero)
        dy = st["dy"].double().masked_fill(~keep[..., None], 0.0)
        (xhat * w[:, None] * dy).sum().backward()
        over = (1,) if c["per_example"] else (0, 1)
        db = dy.sum(over) if c["kind"] == "layer" else None
        return x.grad, w.grad if c["per_example"] else w.grad[0], db
    counted = keep & (st["targets"] != IGNORE)
    b, t = counted.nonzero(as_tuple=True)
    tgt = st["targets"][b, t].long()
    wt = torch.ones(b.numel(), dtype=torch.float64, device="cuda") if st["weights"] is None else \
        st["weights"][b, t].double()
    loss = torch.zeros((c["B"], c["T"]), dtype=torch.float64, device="cuda")
    lse = torch.zeros_like(loss)
    grad = torch.zeros((c["B"], c["T"], c["V"]), dtype=torch.float64, device="cuda") if c["gradient"] else None
    step = max(1, int(2e8 / c["V"]))
    for i in range(0, b.numel(), step):
        s = slice(i, i + step)
        x = st["logits"][b[s], t[s]].double()
        z = torch.logsumexp(x, -1)
        lse[b[s], t[s]] = z
        loss[b[s], t[s]] = wt[s] * (z - x.gather(1, tgt[s, None])[:, 0])
        if grad is not None:
            p = torch.softmax(x, -1)
            p[torch.arange(p.shape[0], device="cuda"), tgt[s]] -= 1.0
            grad[b[s], t[s]] = p * wt[s, None]
    return (loss, lse, grad) if c["gradient"] else (loss, lse)
