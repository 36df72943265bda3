"""GPU checks of distillation where list and remainder lie far apart, against the formulas in
float64 with the tolerances of test_gpu_distill.py."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

from paper_2609_37842_gb300 import eogp as E  # noqa: E402
from test_gpu_distill import BF, DEV, F32, _lib, _status, check_all, make, reference  # noqa: E402,F401


def lists(seed, rows, V, K, dt, tail, h):
    """Logits and lists whose teacher is as soft at every temperature, a tenth of its mass on other classes."""
    x, cls, y, _, _, _ = make(seed, 1, rows, V, K, dt)
    y = y * h
    ylse = torch.logsumexp(y.double() / h, -1).float() + 0.1 if tail else None
    free = torch.ones((1, rows, V), dtype=torch.bool, device=DEV).scatter_(2, cls, False)
    return x, cls, y, ylse, free


@pytest.mark.parametrize("h", [1.0, 0.01, 0.001])
@pytest.mark.parametrize("dt", [BF, F32])
@pytest.mark.parametrize("V", [300, 9000, 70_001])
@pytest.mark.parametrize("tail", [False, True])
def test_rest_far_below_the_list(tail, V, dt, h):
    """All classes that are not listed masked by finite values: the list's own sum keeps its digits."""
    h = float(np.float32(h))
    masks = [-1e3, -1e4, -65504.0, -1e6, -1e7, -1e8] + [-3e38] * (h == 1.0)  # where the loss is a float
    x, cls, y, ylse, free = lists(V, len(masks), V, 5, dt, tail, h)
    low = torch.tensor(masks, device=DEV)[None, :, None].expand_as(x).to(dt)
    x = torch.where(free, low, x)
    check_all(E.distill(x, cls, y, teacher_lse=ylse, temperature=h), reference(x, cls, y, ylse, h, None, None, dt))


@pytest.mark.parametrize("h", [1.0, 0.01, 0.001])
@pytest.mark.parametrize("dt", [BF, F32])
@pytest.mark.parametrize("V", [300, 9000, 70_001])
@pytest.mark.parametrize("tail", [False, True])
def test_list_far_above_the_rest(tail, V, dt, h):
    """Listed logits far above ordinary ones, equal or close to each other; above 1e8 only at h = 1, where the loss
    is a float."""
    h = float(np.float32(h))
    tops = [2e2, 2e3, 1e5, 1e8] + [3e38] * (h == 1.0)
    x, cls, y, ylse, free = lists(V + 1, 2 * len(tops), V, 4, dt, tail, h)
    top = torch.tensor(tops, device=DEV).repeat(2)[None, :, None].expand_as(x).to(dt)
    close = (torch.arange(2 * len(tops), device=DEV) >= len(tops))[None, :, None]
    # rows of one value, and rows of neighbours: the listed logits' own differences where the type has them
    x = torch.where(free, x, torch.where(close & (top < 1e38), (top.float() + x.float() * h).to(dt), top))
    check_all(E.distill(x, cls, y, teacher_lse=ylse, temperature=h), reference(x, cls, y, ylse, h, None, None, dt))


@pytest.mark.parametrize("h", [1.0, 0.01])
@pytest.mark.parametrize("dt", [BF, F32])
@pytest.mark.parametrize("V", [300, 9000, 70_001])
@pytest.mark.parametrize("tail", [False, True])
def test_all_far_from_zero(tail, V, dt, h):
    """Rows around large values of either sign, list and remainder close to each other."""
    h = float(np.float32(h))
    at = [-1e7, -1e5, -1e3, 1e3, 1e5, 1e7]
    x, cls, y, ylse, _ = lists(V + 2, len(at), V, 6, dt, tail, h)
    x = (x.float() * h + torch.tensor(at, device=DEV)[None, :, None]).to(dt)
    check_all(E.distill(x, cls, y, teacher_lse=ylse, temperature=h), reference(x, cls, y, ylse, h, None, None, dt))


@pytest.mark.parametrize("dt", [BF, F32])
@pytest.mark.parametrize("V", [64, 3000, 50_001, 70_001])
def test_empty_list_beside_a_log_sum(V, dt):
    """All of the teacher's mass and all of the student's on one class: no loss and no gradient, to the bit."""
    x, cls, y, ylse, _, _ = make(V, 2, 60, V, 3, dt, tail=True)
    cls.fill_(-1)
    loss, lse, dx = E.distill(x, cls, y, teacher_lse=ylse)
    assert not loss.any() and not dx.any()
    check_all((loss, lse, dx), reference(x, cls, y, ylse, 1.0, None, None, dt))
