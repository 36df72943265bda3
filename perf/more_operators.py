"""Cases for measuring two losses that begin a language model's backward pass,
beside the token loss on given logits: the token loss through the output matrix,
which keeps no logits, and distillation from a teacher's top logits, each with its
gradient.

Both work on B examples of T tokens; positions from lengths[b] on are padding and
hold what was there before. `run` computes them in elementary torch operations in
32 bits, or, with `own` set, through the library's calls.
"""
import math

import torch

own = False

_TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
_SIZES = {"f32": 4, "bf16": 2}
IGNORE = -100


# ------------------------------------------------------------------- cases
def listed():
    return [
        # one token of an answer scored while it is served
        dict(name="head_token", op="head", B=1, T=1, d=768, V=50_000, dtype="bf16", index="i64", gradient=False,
             grad="bf16", scale=1.0, weighted=False, prompt=0, ragged=False),
        # one example of an odd vocabulary: its loss and the gradient that its codes are made from
        dict(name="head_example", op="head", B=1, T=511, d=768, V=50_001, dtype="bf16", index="i64", gradient=True,
             grad="bf16", scale=1.0, weighted=False, prompt=64, ragged=False),
        # the same for a 32-bit model of odd width
        dict(name="head_example_f32", op="head", B=1, T=509, d=770, V=32_001, dtype="f32", index="i32", gradient=True,
             grad="f32", scale=770 ** -0.5, weighted=False, prompt=0, ragged=False),
        # the losses alone of the examples a store is evaluated on, 2048-wide model
        dict(name="head_evaluation", op="head", B=16, T=1024, d=2048, V=100_000, dtype="bf16", index="i64",
             gradient=False, grad="bf16", scale=1.0, weighted=False, prompt=0, ragged=False),
        # a training batch of the 768-wide stack, several lengths, gradient of a tied table in 32 bits
        dict(name="head_batch_small", op="head", B=64, T=512, d=768, V=50_000, dtype="bf16", index="i64",
             gradient=True, grad="f32", scale=1.0, weighted=False, prompt=0, ragged=True),
        # a training batch of conversations for the 4096-wide stack: prompts not counted, several lengths
        dict(name="head_batch", op="head", B=4, T=2048, d=4096, V=100_000, dtype="bf16", index="i64", gradient=True,
             grad="bf16", scale=1.0, weighted=True, prompt=256, ragged=True),
        # how far a short answer is from a teacher's, 32-bit logits over an odd vocabulary
        dict(name="distill_answer", op="distill", B=1, T=37, V=50_001, K=20, dtype="f32", teacher="f32", index="i64",
             gradient=False, tail=False, temperature=1.0, weighted=False, fewer=False, ragged=False),
        # one example of a distilled model, the teacher's remaining mass as one more class
        dict(name="distill_example", op="distill", B=1, T=511, V=50_001, K=64, dtype="bf16", teacher="f32",
             index="i32", gradient=True, tail=True, temperature=1.0, weighted=False, fewer=True, ragged=False),
        # a training batch of the 768-wide stack from short lists
        dict(name="distill_lists", op="distill", B=32, T=512, V=50_000, K=8, dtype="bf16", teacher="bf16",
             index="i32", gradient=True, tail=True, temperature=1.0, weighted=False, fewer=False, ragged=True),
        # a training batch of conversations, softened, the lists renormalised
        dict(name="distill_batch", op="distill", B=4, T=2048, V=100_096, K=128, dtype="bf16", teacher="f32",
             index="i64", gradient=True, tail=False, temperature=2.0, weighted=True, fewer=False, ragged=True),
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
    tokens = _log(rng, 1, max(1, most))
    T = min(tokens, _log(rng, 1, 4096))
    return max(1, tokens // T), T


def draw(rng):
    op = rng.choice(["head", "head", "distill"])
    dtype = rng.choice(["bf16", "bf16", "f32"])
    c = dict(op=op, dtype=dtype, ragged=rng.random() < 0.5, weighted=rng.random() < 0.5,
             gradient=rng.random() < 0.75, index=rng.choice(["i64", "i32"]))
    V = _log(rng, 1000, 131_072)
    if op == "head":
        d = _width(rng, 64, 4096)
        # as many multiplications as the largest batch at most, or as the 32-bit example four times
        products = 1.6e12 if dtype == "bf16" else 5.0e10
        B, T = _batch(rng, min(65_536, int(products / (V * d)), int(1.6e9 / V)))
        c.update(B=B, T=T, d=d, V=V, grad="f32" if dtype == "f32" else rng.choice(["bf16", "bf16", "f32"]),
                 scale=rng.choice([1.0, d ** -0.5]), prompt=rng.choice([0, T // 4]))
        return c
    B, T = _batch(rng, min(65_536, max(1, int(1.2e9 / (V * _SIZES[dtype] * (2 if c["gradient"] else 1))))))
    c.update(B=B, T=T, V=V, K=_log(rng, 1, 256), teacher=rng.choice(["f32", "bf16"]), tail=rng.random() < 0.5,
             temperature=rng.choice([1.0, 1.0, 2.0, 0.7]), fewer=rng.random() < 0.5)
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


def _index(c, t):
    return t.to(torch.int32 if c["index"] == "i32" else torch.int64)


def prepare(case, seed):
    c, g = case, _gen(seed)
    B, T, V, dt = c["B"], c["T"], c["V"], _TYPES[c["dtype"]]
    st = dict(case=c, lengths=None, keep=None)

    def normal(*shape):
        return torch.randn(shape, generator=g, device="cuda")

    def uniform(*shape):
        return torch.rand(shape, generator=g, device="cuda")

    if c["ragged"]:
        order = torch.randperm(B, generator=g, device="cuda")
        st["lengths"] = torch.tensor(_lengths(c), dtype=torch.int32, device="cuda")[order].contiguous()
        st["keep"] = torch.arange(T, device="cuda")[None] < st["lengths"][:, None]
    st["weights"] = 0.5 + uniform(B, T) if c["weighted"] else None

    def pad(x, value):
        return x if st["keep"] is None else x.masked_fill_(~st["keep"][..., None], value)

    if c["op"] == "head":
        # the last normalisation's output: unit scale, a few channels much larger, a part of it along the
        # target's row, so that targets are found with all degrees of certainty
        d = c["d"]
        w = normal(V, d).mul_(2.5 / (math.sqrt(d) * c["scale"]))
        st["weight"] = w.to(dt)
        tgt = torch.randint(0, V, (B, T), generator=g, device="cuda")
        x = normal(B, T, d)
        x[..., :: max(1, d // 6)] *= 4.0
        x.add_(st["weight"].float()[tgt] * (uniform(B, T, 1) * (2.0 * c["scale"])))
        st["x"] = pad(x.to(dt), float("nan"))
        tgt[:, : c["prompt"]] = IGNORE
        st["targets"] = _index(c, tgt)
        return st
    # a teacher's K best classes of each position, and the student's logits, raised where the teacher's are
    K = min(c["K"], V)
    first = torch.randint(0, V, (B, T, 1), generator=g, device="cuda")
    step = torch.randint(1, max(2, V // K + 1), (B, T, 1), generator=g, device="cuda")
    k = torch.arange(K, device="cuda")
    cls = (first + step * k) % V
    y = 14.0 - (1.0 + 2.0 * uniform(B, T, 1)) * torch.log1p(k.float()) - 0.5 * uniform(B, T, K)
    y = y.sort(-1, descending=True).values.to(_TYPES[c["teacher"]])
    x = normal(B, T, V).mul_(1.5)
    x.scatter_add_(2, cls, y.float() * (0.3 + 0.6 * uniform(B, T, 1)))
    st["logits"] = pad(x.to(dt), float("nan"))
    st["teacher"] = pad(y, float("inf"))
    st["teacher_lse"] = None
    if c["tail"]:
        # from a tenth of a percent to a fifth of the mass is on other classes
        mass = torch.exp(math.log(1e-3) + uniform(B, T) * (math.log(0.2) - math.log(1e-3)))
        st["teacher_lse"] = torch.logsumexp(y.float() / c["temperature"], -1) - torch.log1p(-mass)
    if c["fewer"]:
        kept = torch.randint(max(1, K // 4), K + 1, (B, T, 1), generator=g, device="cuda")
        cls = torch.where(k < kept, cls, -1)
    st["classes"] = _index(c, cls).contiguous()
    return st


# -------------------------------------------------------------- plain forms
def _counted(st, counted):
    return counted if st["keep"] is None else counted & st["keep"]


def _weights(st, counted):
    return counted.float() if st["weights"] is None else torch.where(counted, st["weights"], 0.0)


def _head(st):
    c = st["case"]
    counted = _counted(st, st["targets"] != IGNORE)
    n = (c["B"] * c["T"],)
    row = counted.reshape(n)
    tgt = torch.where(row, st["targets"].reshape(n).long(), 0)[:, None]
    w = _weights(st, counted).reshape(n)
    x = torch.where(row[:, None], st["x"].reshape(*n, c["d"]).float(), 0.0)
    W = st["weight"].float()
    z = x @ W.T
    z.mul_(c["scale"])
    top = z.amax(-1, keepdim=True)
    zt = z.gather(1, tgt)[:, 0]
    e = z.sub_(top).exp_()
    s = e.sum(-1)
    lse = top[:, 0] + torch.log(s)
    loss = (w * (lse - zt)).reshape(counted.shape)
    lse = torch.where(row, lse, 0.0).reshape(counted.shape)
    if not c["gradient"]:
        return loss, lse
    e.mul_((w / s)[:, None])
    e.scatter_add_(1, tgt, -w[:, None])
    dx = (e @ W) * c["scale"]
    dW = (e.T @ x) * c["scale"]
    return loss, lse, dx.to(st["x"].dtype).reshape(st["x"].shape), dW.to(_TYPES[c["grad"]])


def _distill(st):
    c = st["case"]
    t = c["temperature"]
    counted = torch.ones((c["B"], c["T"]), dtype=torch.bool, device="cuda")
    counted = _counted(st, counted)
    w = _weights(st, counted)
    there = (st["classes"] >= 0) & counted[..., None]
    cls = torch.where(there, st["classes"].long(), 0)
    y = torch.where(there, st["teacher"].float() / t, float("-inf"))
    x = torch.where(counted[..., None], st["logits"].float(), 0.0).div_(t)
    top = x.amax(-1, keepdim=True)
    xk = x.gather(-1, cls)
    e = x.sub_(top).exp_()
    s = e.sum(-1)
    lse = top[..., 0] + torch.log(s)
    # the teacher's probabilities and their logarithms
    if c["tail"]:
        log_q = y - torch.where(counted, st["teacher_lse"], 0.0)[..., None]
    else:
        best = y.amax(-1, keepdim=True)
        best = torch.where(torch.isfinite(best), best, 0.0)
        log_q = y - best - torch.log(torch.exp(y - best).sum(-1, keepdim=True))
    q = torch.where(there, torch.exp(log_q), 0.0)
    terms = torch.where(there, q * (log_q - (xk - lse[..., None])), 0.0)
    loss = terms.sum(-1)
    ek = torch.where(there, torch.exp(xk - top), 0.0)
    if c["tail"]:
        # summed without the listed classes: a difference of sums would lose a small remainder
        e.scatter_(-1, torch.where(there, cls, cls[..., :1]), 0.0)
        rest = e.sum(-1)
        q_rest = (1.0 - q.double().sum(-1)).clamp_(min=0.0).float()
        loss = loss + q_rest * (torch.log(q_rest) - torch.log(rest / s))
        ratio = q_rest * s / rest
    loss = torch.where(counted, w * loss, 0.0)
    lse = torch.where(counted, lse, 0.0)
    if not c["gradient"]:
        return loss, lse
    wt = w / t
    others = (1.0 - ratio if c["tail"] else 1.0) * wt / s
    e.mul_(torch.where(counted, others, 0.0)[..., None])
    if c["tail"]:
        e.scatter_add_(-1, cls, torch.where(there, ek * (wt / s)[..., None], 0.0))
    e.scatter_add_(-1, cls, -q * wt[..., None])
    return loss, lse, e.to(st["logits"].dtype)


def run(state):
    st, c = state, state["case"]
    if not own:
        return _head(st) if c["op"] == "head" else _distill(st)
    from paper_2609_37842_gb300 import eogp as E
    if c["op"] == "head":
        loss, lse, dx, dW = E.head_loss(st["x"], st["weight"], st["targets"], scale=c["scale"], weights=st["weights"],
                                        lengths=st["lengths"], ignore_index=IGNORE, want_dx=c["gradient"],
                                        want_dweight=c["gradient"], dtype=_TYPES[c["grad"]])
        return (loss, lse, dx, dW) if c["gradient"] else (loss, lse)
    loss, lse, dlogits = E.distill(st["logits"], st["classes"], st["teacher"], teacher_lse=st["teacher_lse"],
                                   temperature=c["temperature"], weights=st["weights"], lengths=st["lengths"],
                                   want_grad=c["gradient"])
    return (loss, lse, dlogits) if c["gradient"] else (loss, lse)


# --------------------------------------------------------------------- work
def work(case):
    c = case
    es, V = _SIZES[c["dtype"]], c["V"]
    M, n = c["B"] * c["T"], sum(_lengths(c))
    ix = 4 if c["index"] == "i32" else 8
    if c["op"] == "head":
        d = c["d"]
        m = sum(max(0, t - c["prompt"]) for t in _lengths(c))
        out = M * d * es + V * d * _SIZES[c["grad"]] if c["gradient"] else 0
        return {"bytes": (m + V) * d * es + n * ix + M * 8 + (m * 4 if c["weighted"] else 0) + out,
                "flops": m * V * (d * (6 if c["gradient"] else 2) + 4)}
    K = min(c["K"], V)
    lists = n * K * (ix + _SIZES[c["teacher"]]) + (n * 4 if c["tail"] else 0)
    return {"bytes": n * V * es + lists + M * 8 + (n * 4 if c["weighted"] else 0) +
            (M * V * es if c["gradient"] else 0), "flops": n * (V * (6 if c["gradient"] else 4) + 8 * K)}


# ------------------------------------------------------------------ 64 bits
def exact(case, seed):
    st, c = prepare(case, seed), case
    f64 = dict(dtype=torch.float64, device="cuda")
    B, T, V = c["B"], c["T"], c["V"]
    kept = torch.ones((B, T), dtype=torch.bool, device="cuda") if st["keep"] is None else st["keep"]
    loss, lse = torch.zeros((B, T), **f64), torch.zeros((B, T), **f64)
    step = max(1, int(2e8 / V))
    if c["op"] == "head":
        b, t = (kept & (st["targets"] != IGNORE)).nonzero(as_tuple=True)
        W = st["weight"].double()
        dx = torch.zeros((B, T, c["d"]), **f64)
        dW = torch.zeros((V, c["d"]), **f64)
        for i in range(0, b.numel(), step):
            at = (b[i:i + step], t[i:i + step])
            x = st["x"][at].double()
            z = (x @ W.T) * c["scale"]
            wt = torch.ones(x.shape[0], **f64) if st["weights"] is None else st["weights"][at].double()
            lp = torch.log_softmax(z, -1)
            mine = (torch.arange(x.shape[0], device="cuda"), st["targets"][at].long())
            lse[at] = z[mine] - lp[mine]
            loss[at] = -wt * lp[mine]
            if c["gradient"]:
                p = lp.exp_()
                p[mine] = torch.expm1(torch.log(p[mine]))
                p *= wt[:, None] * c["scale"]
                dx[at] = p @ W
                dW += p.T @ x
        return (loss, lse, dx, dW) if c["gradient"] else (loss, lse)
    b, t = kept.nonzero(as_tuple=True)
    grad = torch.zeros((B, T, V), **f64) if c["gradient"] else None
    for i in range(0, b.numel(), step):
        at = (b[i:i + step], t[i:i + step])
        x = (st["logits"][at].double() / c["temperature"]).requires_grad_(c["gradient"])
        cls = st["classes"][at].long()
        r, k = (cls >= 0).nonzero(as_tuple=True)
        listed_ = torch.zeros(x.shape, dtype=torch.bool, device="cuda")
        listed_[r, cls[r, k]] = True
        y = st["teacher"][at].double()[r, k] / c["temperature"]
        # log of the teacher's probability at the listed classes, in place
        log_q = torch.full(x.shape, float("-inf"), **f64)
        log_q[r, cls[r, k]] = y
        whole = st["teacher_lse"][at].double() if c["tail"] else torch.logsumexp(log_q, -1)
        log_q = torch.where(listed_, log_q - whole[:, None], 0.0)
        q = torch.where(listed_, torch.exp(log_q), 0.0)
        z = torch.logsumexp(x, -1)
        each = (q * (log_q - (x - z[:, None]))).sum(-1)
        if c["tail"]:
            q_rest = 1.0 - q.sum(-1)
            log_rest = torch.logsumexp(x.masked_fill(listed_, float("-inf")), -1) - z
            each = each + q_rest * (torch.log(q_rest) - log_rest)
        if st["weights"] is not None:
            each = each * st["weights"][at].double()
        loss[at], lse[at] = each.detach(), z.detach()
        if grad is not None:
            grad[at] = torch.autograd.grad(each.sum(), x)[0] / c["temperature"]
    return (loss, lse, grad) if grad is not None else (loss, lse)
