"""Example: attribute a small language model's answers to its training examples,
from tokens to a ranking.

    python -m paper_2609_37842_gb300.attribute_lm

One pass of the model with this library's model ends (token embedding,
normalisation, token loss, each with its gradient) and plain matrix products
between them gives the activations a_t and output gradients s_t of the linear
modules; these are compressed to one-bit codes, and queries are scored against the
stored examples. The model is random and untrained: each query repeats a stored
example, which has to rank first among all of them.

The model, tokens x of an example (padding beyond its length):
    h0 = table[x] + pos,  n1 = layernorm(h0),  u = n1 W1^T,  g = gelu(u),
    h1 = h0 + g W2^T,     n2 = rmsnorm(h1),    logits = n2 table^T,
with the loss of the next token at every position but an example's last.
"""
from __future__ import annotations

from dataclasses import dataclass

from . import eogp as E


@dataclass
class Model:
    table: "torch.Tensor"   # [V, d]
    pos: "torch.Tensor"     # [T, d]
    norm1: tuple            # weight, bias [d]
    W1: "torch.Tensor"      # [f, d]
    W2: "torch.Tensor"      # [d, f]
    norm2: "torch.Tensor"   # weight [d]


def make_model(V: int, T: int, d: int, f: int, dtype, generator, device="cuda") -> Model:
    import torch

    def normal(*shape, std):
        return (torch.randn(shape, generator=generator, device=device) * std).to(dtype)

    return Model(normal(V, d, std=0.5), normal(T, d, std=0.1), (1 + normal(d, std=0.1), normal(d, std=0.1)),
                 normal(f, d, std=d ** -0.5), normal(d, f, std=f ** -0.5), 1 + normal(d, std=0.1))


def next_tokens(tokens, lengths):
    """Targets [B, T]: the next token, ignored at an example's last position."""
    import torch
    targets = torch.full_like(tokens, -100)
    targets[:, :-1] = tokens[:, 1:]
    last = torch.arange(tokens.shape[1], device=tokens.device)[None] >= (lengths - 1)[:, None]
    return targets.masked_fill_(last, -100)


def backward_pass(model: Model, tokens, lengths):
    """One forward and backward pass. Returns loss [B, T], the modules' (a, s) pairs, and the gradients: of the
    table (over the batch), of the position table, and of the normalisations' weights for each example."""
    import torch
    V, (B, T) = model.table.shape[0], tokens.shape
    h0 = E.embed(tokens, model.table, pos=model.pos, lengths=lengths)
    n1, mean1, rstd1 = E.norm(h0, *model.norm1, lengths=lengths)
    u = n1 @ model.W1.T
    g = torch.nn.functional.gelu(u)
    h1 = h0 + g @ model.W2.T
    n2, _, rstd2 = E.norm(h1, model.norm2, kind=E.NORM_RMS, lengths=lengths)
    logits = n2 @ model.table.T
    loss, _, dlogits = E.cross_entropy(logits, next_tokens(tokens, lengths), lengths=lengths, dlogits=logits)

    dn2 = dlogits @ model.table
    dh1, dnorm2, _ = E.norm_grad(dn2, h1, None, rstd2, model.norm2, kind=E.NORM_RMS, lengths=lengths,
                                 per_example=True, want_dbias=False)
    uf = u.float()
    dgelu = 0.5 * (1 + torch.erf(uf * 0.5 ** 0.5)) + uf * torch.exp(-0.5 * uf * uf) * (2 * torch.pi) ** -0.5
    du = ((dh1 @ model.W2).float() * dgelu).to(u.dtype)
    dx, dw1, db1 = E.norm_grad(du @ model.W1, h0, mean1, rstd1, model.norm1[0], lengths=lengths, per_example=True)
    dh0 = dh1 + dx
    dtable = (dlogits.reshape(-1, V).T @ n2.reshape(-1, n2.shape[-1])).float()      # the head's share
    E.embed_grad(tokens, dh0, V, lengths=lengths, dtable=dtable, accumulate=True)   # the embedding's
    positions = torch.arange(T, device=tokens.device).expand(B, T)
    dpos = E.embed_grad(positions, dh0, T, lengths=lengths)
    return loss, {"W1": (n1, du), "W2": (g, dh1)}, {"table": dtable, "pos": dpos, "norm1": (dw1, db1),
                                                   "norm2": dnorm2}


def fit_module(a, s, lengths, m: int, k: int):
    """Plan, eigenbases and second-stage directions of one module from a batch of its a and s."""
    import torch
    B, T, _ = a.shape
    factors = []
    for x in (a, s):
        x2 = x.reshape(B * T, -1).double()
        lam, Q = torch.linalg.eigh(x2.T @ x2 / (B * T))
        factors.append((lam.clamp_min(0).cpu().numpy(), Q.T.to(x.dtype).contiguous()))
    (lam_a, Qa), (lam_s, Qs) = factors
    plan = E.Plan.from_factors(lam_s, lam_a, m, 0.1)
    VA, VS = plan.gather_rows(0, Qa), plan.gather_rows(1, Qs)
    first = E.layer_desc(plan, T, 1, VA, VS, lengths=lengths)
    Z = E.compress_layer(first, a, s, E.OUT_FIRST_STAGE)
    Pt, _ = E.fit_pca(Z, k, E.BF16 if a.dtype == torch.bfloat16 else E.F32)
    return plan, VA, VS, Pt


def codes_of(fits, pairs, lengths, k: int):
    """Codes [B, words] and scales [B, modules] of a batch."""
    import torch
    out = []
    for name, (a, s) in pairs.items():
        plan, VA, VS, Pt = fits[name]
        desc = E.layer_desc(plan, a.shape[1], k, VA, VS, Pt, lengths=lengths)
        out.append(E.compress_layer(desc, a.contiguous(), s.contiguous(), E.OUT_CODES))
    return torch.cat([c for c, _ in out], 1), torch.stack([sc for _, sc in out], 1)


def run(V: int = 1000, B: int = 192, T: int = 40, d: int = 128, f: int = 256, m: int = 512, k: int = 128,
        queries: int = 16, dtype=None, seed: int = 0):
    """Stores B examples, queries with `queries` of them. Returns the queried rows' ranks (0 = first)."""
    import torch
    dtype = dtype or torch.bfloat16
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    model = make_model(V, T, d, f, dtype, g)
    tokens = torch.randint(0, V, (B, T), generator=g, device="cuda")
    lengths = torch.randint(T // 4, T + 1, (B,), generator=g, device="cuda", dtype=torch.int32)
    _, pairs, _ = backward_pass(model, tokens, lengths)
    fits = {name: fit_module(a, s, lengths, m, k) for name, (a, s) in pairs.items()}
    codes, scales = codes_of(fits, pairs, lengths, k)

    asked = torch.randperm(B, generator=g, device="cuda")[:queries]
    _, qpairs, _ = backward_pass(model, tokens[asked], lengths[asked])
    qcodes, qscales = codes_of(fits, qpairs, lengths[asked], k)
    scores = E.score(codes, scales, [k] * len(pairs), E.SCORE_CODES, qcodes, qscales)
    E.sync_status()
    own = scores.gather(1, asked[:, None])
    return (scores > own).sum(1).tolist()


if __name__ == "__main__":
    ranks = run()
    print(f"{len(ranks)} queries, each repeating a stored example: {sum(r == 0 for r in ranks)} rank it first")
