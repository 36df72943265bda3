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
