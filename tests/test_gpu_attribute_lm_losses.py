"""The example model with the loss through the output matrix and with distillation: its
gradients against autograd in float64, and its rankings."""
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

from paper_2609_37842_gb300 import attribute_lm as L  # noqa: E402
from paper_2609_37842_gb300 import eogp as E  # noqa: E402


@pytest.fixture(scope="module", autouse=True)
def _lib():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    from paper_2609_37842_gb300 import build
    build.build()
    E.lib()
    old = torch.backends.cuda.matmul.allow_tf32
    torch.backends.cuda.matmul.allow_tf32 = False
    yield
    torch.backends.cuda.matmul.allow_tf32 = old
    torch.cuda.empty_cache()


def reference(model, tokens, lengths, loss_of):
    """loss_of(logits) in float64 and the gradients of its sum, each example's own for the normalisations."""
    B, d = tokens.shape[0], model.table.shape[1]
    p = {n: t.double().requires_grad_() for n, t in dict(table=model.table, pos=model.pos, W1=model.W1,
                                                        W2=model.W2).items()}
    own = [t.double().expand(B, d).clone().detach().requires_grad_()
           for t in (model.norm1[0], model.norm1[1], model.norm2)]
    h0 = p["table"][tokens] + p["pos"]
    n1 = torch.nn.functional.layer_norm(h0, (d,), eps=1e-5) * own[0][:, None] + own[1][:, None]
    u = n1 @ p["W1"].T
    h1 = h0 + torch.nn.functional.gelu(u) @ p["W2"].T
    n2 = h1 * torch.rsqrt((h1 * h1).mean(-1, keepdim=True) + 1e-5) * own[2][:, None]
    keep = torch.arange(tokens.shape[1], device=tokens.device)[None] < lengths[:, None]
    loss = loss_of(n2 @ p["table"].T) * keep
    u.retain_grad()
    h1.retain_grad()
    loss.sum().backward()
    k = keep[..., None]
    return [loss, p["table"].grad, p["pos"].grad, own[0].grad, own[1].grad, own[2].grad, u.grad * k, h1.grad * k]


def results(out):
    loss, pairs, grads = out
    return [loss, grads["table"], grads["pos"], *grads["norm1"], grads["norm2"], pairs["W1"][1], pairs["W2"][1]]


@pytest.mark.parametrize("loss_from", ["head", "distill"])
def test_gradients_equal_autograd(loss_from):
    """fp32 model against the same one in float64 with autograd: every rounding is at 2^-24 of values the size of
    their array's largest, over chains of some hundred operations, so 1e-4 of the largest entry is ample."""
    V, B, T, d, f = 97, 5, 13, 48, 40
    g = torch.Generator(device="cuda")
    g.manual_seed(1)
    model, other = (L.make_model(V, T, d, f, torch.float32, g) for _ in range(2))
    tokens = torch.randint(0, V, (B, T), generator=g, device="cuda")
    lengths = torch.tensor([13, 1, 7, 0, 12], dtype=torch.int32, device="cuda")
    teacher = L.top_logits(other, tokens, lengths, 9)
    got = results(L.backward_pass(model, tokens, lengths, loss_from, teacher))
    E.sync_status()

    def token_loss(z):
        return torch.nn.functional.cross_entropy(z.transpose(1, 2), L.next_tokens(tokens, lengths), reduction="none",
                                                 ignore_index=-100)

    def distance(z):
        classes, best, lse = teacher
        log_q = best.double() - lse.double()[..., None]
        log_p = torch.log_softmax(z, -1).gather(-1, classes)
        # the teacher's rounded logits may sum to a little more than 1: no rest, as the call defines it
        q_rest, p_rest = (1 - log_q.exp().sum(-1)).clamp_min(0), 1 - log_p.exp().sum(-1)
        return (log_q.exp() * (log_q - log_p)).sum(-1) + torch.xlogy(q_rest, q_rest) - q_rest * torch.log(p_rest)

    want = reference(model, tokens, lengths, token_loss if loss_from == "head" else distance)
    for a, b in zip(got, want):
        a, b = a.detach().double(), b.detach()
        assert (a - b).abs().max() <= 1e-4 * b.abs().max()


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_queries_find_their_own_example(dtype):
    ranks = L.run(dtype=dtype, loss_from="head")
    assert ranks == [0] * len(ranks)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_distilled_runs_are_reproducible(dtype):
    """Against one teacher the examples' gradients point much the same way, and a score s_q s_i <b_q, b_i> may be higher
    for a stored example of a larger scale s_i than for the query's own: that it ranks first is no property here."""
    a, b = (L.run(dtype=dtype, loss_from="distill") for _ in range(2))
    assert a == b and all(0 <= r < 192 for r in a)
