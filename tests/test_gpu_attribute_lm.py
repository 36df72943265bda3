"""The example model that runs the model ends together with the compression and
scoring: its gradients against autograd in float64, and its rankings."""
import numpy as np
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


def test_gradients_equal_autograd():
    """fp32 model against the same one in float64 with autograd: every rounding is at 2^-24 of values the size of
    their array's largest, over chains of some hundred operations, so 1e-4 of the largest entry is ample."""
    V, B, T, d, f = 97, 5, 13, 48, 40
    g = torch.Generator(device="cuda")
    g.manual_seed(1)
    model = L.make_model(V, T, d, f, torch.float32, g)
    tokens = torch.randint(0, V, (B, T), generator=g, device="cuda")
    lengths = torch.tensor([13, 1, 7, 0, 12], dtype=torch.int32, device="cuda")
    loss, pairs, grads = L.backward_pass(model, tokens, lengths)
    E.sync_status()

    p = {n: t.double().requires_grad_() for n, t in dict(table=model.table, pos=model.pos, w1=model.norm1[0],
                                                        b1=model.norm1[1], W1=model.W1, W2=model.W2,
                                                        w2=model.norm2).items()}
    keep = torch.arange(T, device="cuda")[None] < lengths[:, None]
    w1 = p["w1"].expand(B, d).clone().detach().requires_grad_()
    b1 = p["b1"].expand(B, d).clone().detach().requires_grad_()
    w2 = p["w2"].expand(B, d).clone().detach().requires_grad_()
    h0 = p["table"][tokens] + p["pos"]
    n1 = torch.nn.functional.layer_norm(h0, (d,), eps=1e-5) * w1[:, None] + b1[:, None]
    u = n1 @ p["W1"].T
    h1 = h0 + torch.nn.functional.gelu(u) @ p["W2"].T
    n2 = h1 * torch.rsqrt((h1 * h1).mean(-1, keepdim=True) + 1e-5) * w2[:, None]
    logits = n2 @ p["table"].T
    tgt = L.next_tokens(tokens, lengths)
    want = torch.nn.functional.cross_entropy(logits.transpose(1, 2), tgt, reduction="none", ignore_index=-100)
    want = want * keep
    u.retain_grad()
    h1.retain_grad()
    want.sum().backward()
    k = keep[..., None]
    for got, ref in ((loss, want), (grads["table"], p["table"].grad), (grads["pos"], p["pos"].grad),
                     (grads["norm1"][0], w1.grad), (grads["norm1"][1], b1.grad), (grads["norm2"], w2.grad),
                     (pairs["W1"][0], n1 * k), (pairs["W1"][1], u.grad * k), (pairs["W2"][1], h1.grad * k)):
        got, ref = got.detach().double(), ref.detach()
        assert (got - ref).abs().max() <= 1e-4 * ref.abs().max()
    G1 = torch.einsum("bto,bti->oi", pairs["W1"][1].double(), pairs["W1"][0].double())
    assert (G1 - p["W1"].grad).abs().max() <= 1e-4 * p["W1"].grad.abs().max()


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_queries_find_their_own_example(dtype):
    ranks = L.run(dtype=dtype)
    assert ranks == [0] * len(ranks)


def test_runs_are_reproducible():
    a, b = (L.run(seed=3, B=96, k=64, m=256) for _ in range(2))
    assert a == b == [0] * len(a)
    assert np.isfinite(a).all()
