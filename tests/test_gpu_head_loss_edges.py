"""GPU checks of the token loss through the output matrix where targets, probabilities or values are unevenly
distributed, against its formulas in float64 with the tolerances of test_gpu_head_loss.py."""
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

from paper_2609_37842_gb300 import eogp as E  # noqa: E402
from test_gpu_head_loss import BF, DEV, F32, _lib, _status, check, check_all, gen, make, reference, rounded  # noqa: E402,F401


@pytest.mark.parametrize("gdt", [BF, F32])
@pytest.mark.parametrize("T,d,V,many", [(1200, 64, 2000, 0.3), (2048, 64, 4100, 0.1), (3979, 256, 8192, 0.05),
                                        (511, 768, 1500, 0.2), (3000, 136, 5000, 0.9)])
def test_rare_classes_beside_a_frequent_one(T, d, V, many, gdt):
    """One class has many of the targets, the first ones among them; its 31 neighbours one each, spread over the rest.
    What rounding takes from the target's entry is added to the neighbours' rows whatever the frequent class has."""
    x, W, _, w, ln = make(T + d + V, 1, T, d, V, BF, weighted=True)
    g = gen(T)
    n = int(many * T)
    often, near = 512 + 7, torch.tensor([c for c in range(512, 544) if c != 512 + 7], device=DEV)
    tgt = torch.randint(0, V - 32, (T,), generator=g, device=DEV)
    tgt = torch.where(tgt >= 512, tgt + 32, tgt)
    others = torch.arange(40, T, device=DEV)[torch.randperm(T - 40, generator=g, device=DEV)]
    tgt[:40] = often
    tgt[others[:max(0, n - 40)]] = often
    tgt[others[-31:]] = near
    w[0, others[-31:]] = 1.0 + 2.0 ** -8 + 2.0 ** -10 * torch.arange(31, device=DEV)
    tgt = tgt[None]
    got = E.head_loss(x, W, tgt, weights=w, dtype=gdt)
    check_all(got, reference(x, W, tgt, w, ln, 1.0, BF, gdt), gdt)
    want, tol = rounded(reference(x, W, tgt, w, ln, 1.0, BF, gdt, whole_targets=True), None, gdt)
    check(got[3][near], want[near], tol[near], "rows of the neighbours")
    for a, b in zip(got, E.head_loss(x, W, tgt, weights=w, dtype=gdt)):
        assert torch.equal(a, b)


FORMS = [
    # few positions; logits kept; formed again; fp32; in several pieces, of each form of D
    (1, 40, 64, 300, BF, BF), (1, 40, 64, 300, BF, F32), (1, 200, 1100, 700, BF, BF), (1, 1500, 1100, 257, BF, F32),
    (2, 700, 200, 1500, BF, BF), (2, 700, 200, 1500, BF, F32), (1, 30, 70, 257, F32, F32), (2, 600, 136, 900, F32, F32),
    (2, 2600, 64, 400_000, BF, BF), (1, 1500, 40, 300_001, F32, F32),
]


@pytest.mark.parametrize("bad", [float("nan"), float("inf"), float("-inf")])
@pytest.mark.parametrize("B,T,d,V,dt,gdt", FORMS)
def test_not_finite_in_x(B, T, d, V, dt, gdt, bad):
    """One counted position's row: its own loss, lse and dx and all of dW have no finite value, and nothing else is
    touched, to the bit."""
    x, W, tgt, _, _ = make(B * T + V, B, T, d, V, dt, ignored=0.05)
    at = (B - 1, T - 7)
    tgt[at] = 3
    clean = E.head_loss(x, W, tgt, dtype=gdt)
    x[at][d // 2] = bad
    loss, lse, dx, dW = E.head_loss(x, W, tgt, dtype=gdt)
    assert bool(torch.isnan(loss[at])) and bool(torch.isnan(lse[at])) and bool(torch.isnan(dx[at]).all())
    assert bool(torch.isnan(dW).all())
    keep = torch.ones((B, T), dtype=torch.bool, device=DEV)
    keep[at] = False
    for a, b in zip((loss, lse, dx), clean):
        assert torch.equal(a[keep], b[keep])
    tgt[at] = -100
    x2 = torch.where(torch.isfinite(x), x, 0.0)
    for a, b in zip(E.head_loss(x, W, tgt, dtype=gdt), E.head_loss(x2, W, tgt, dtype=gdt)):
        assert torch.equal(a, b)


@pytest.mark.parametrize("B,T,d,V,dt,gdt", FORMS)
def test_nan_in_weight(B, T, d, V, dt, gdt):
    """It is in every position's logits: every counted position's results and all of dW are NaN; the others are 0."""
    x, W, tgt, _, _ = make(B * T + V + 1, B, T, d, V, dt, ignored=0.05)
    W[V - 5, d // 3] = float("nan")
    loss, lse, dx, dW = E.head_loss(x, W, tgt, dtype=gdt)
    c = tgt != -100
    for t in (loss, lse, dx):
        assert bool(torch.isnan(t[c]).all()) and not t[~c].any()
    assert bool(torch.isnan(dW).all())


@pytest.mark.parametrize("bad", [float("inf"), float("-inf")])
@pytest.mark.parametrize("B,T,d,V,dt,gdt", FORMS)
def test_infinity_in_weight(B, T, d, V, dt, gdt, bad):
    """A position whose x is positive there has a logit of `bad`: +inf gives NaN. That column of every dx, which it is
    multiplied with, is not finite."""
    x, W, tgt, _, _ = make(B * T + V + 2, B, T, d, V, dt, ignored=0.05)
    W[V - 5, d // 3] = bad
    loss, lse, dx, dW = E.head_loss(x, W, tgt, dtype=gdt)
    c = tgt != -100
    up = c & (x[..., d // 3].float() * bad > 0)
    for t in (loss, lse, dx):
        assert bool(torch.isnan(t[up]).all()) and not t[~c].any()
    assert not bool(torch.isfinite(dx[c][:, d // 3]).any())


@pytest.mark.parametrize("lean", [1.5, 3.0, 6.0])
@pytest.mark.parametrize("B,T,d,V,dt,gdt", [(1, 700, 256, 4000, BF, BF), (1, 700, 256, 4000, BF, F32),
                                            (2, 400, 1100, 1500, BF, BF), (1, 500, 72, 3000, F32, F32)])
def test_wrong_classes(B, T, d, V, dt, gdt, lean):
    """A class that is not the target has much of each position's mass, up to all of it; some of them shared."""
    x, W, _, w, _ = make(V + d, B, T, d, V, dt, weighted=True)
    g = gen(V)
    tgt, wrong = (torch.randint(0, V, (B, T), generator=g, device=DEV) for _ in range(2))
    wrong[:, ::3] = 5
    x = (torch.randn((B, T, d), generator=g, device=DEV) + lean * W.float()[wrong]).to(dt)
    got = E.head_loss(x, W, tgt, weights=w, dtype=gdt)
    check_all(got, reference(x, W, tgt, w, None, 1.0, dt, gdt), gdt)
