"""GPU checks of distillation where list and remainder lie far apart, and where the teacher's mass is not 1, against
the formulas in float64 with the tolerances of test_gpu_distill.py."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

from paper_2609_37842_gb300 import eogp as E  # noqa: E402
from test_gpu_distill import BF, DEV, F32, U, _lib, _status, check_all, gen, make, out_u, reference  # noqa: E402,F401


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


def with_mass(x, cls, y, ylse, h, dt):
    """`reference` of one class each entry with a log-sum, its gradient of a teacher of mass Q = sum q + q_r, not 1:
    (w / h) (Q - 1) p more at every class. Its tolerance grows by the errors of that p (a logarithm 4 u (max - x) / h
    off, sums) and of Q (each q off by its logarithm's error and the sum's), and by the rounding."""
    r = reference(x, cls, y, ylse, h, None, None, dt)
    V, K = x.shape[-1], cls.shape[-1]
    z = x.double() / h
    z = z - z.amax(-1, keepdim=True)
    p = torch.softmax(z, -1)
    yy = y.double() / h
    q = torch.exp(yy - ylse.double()[..., None])
    listed = torch.zeros(x.shape, dtype=torch.bool, device=DEV).scatter_(2, cls.long(), True)
    q_r = torch.where(listed.all(-1), 0.0, (1 - q.sum(-1)).clamp_min(0))
    more = (q.sum(-1) + q_r - 1)[..., None]
    sums = (V / 32 + K / 32 + 160) * U
    e_q = (4 * U * (yy.abs().amax(-1) + ylse.double().abs()) + sums)[..., None] * q.sum(-1, keepdim=True) + 2 * U
    extra = more.abs() * p * (4 * U * z.abs() + 2 * sums) + p * e_q
    r["dx"] = r["dx"] + more * p / h
    r["tdx"] = r["tdx"] + (extra + (out_u(dt) + 4 * U) * (more.abs() * p + extra)) / h
    return r


def derivative(x, cls, y, ylse, h):
    """The loss's derivative by automatic differentiation in float64, the teacher's probabilities constants."""
    x = (x.double()).requires_grad_()
    z = x / h
    log_p = torch.log_softmax(z, -1)
    log_q = y.double() / h - ylse.double()[..., None]
    q = torch.exp(log_q)
    listed = torch.zeros(x.shape, dtype=torch.bool, device=DEV).scatter_(2, cls.long(), True)
    whole = listed.all(-1)
    q_r = torch.where(whole, 0.0, (1 - q.sum(-1)).clamp_min(0))
    log_pr = torch.logsumexp(z.masked_fill(listed & ~whole[..., None], float("-inf")), -1) - torch.logsumexp(z, -1)
    loss = (q * (log_q - log_p.gather(-1, cls.long()))).sum(-1) + torch.xlogy(q_r, q_r) - q_r * log_pr
    return torch.autograd.grad(loss.sum(), x)[0]


def check_mass(x, cls, y, ylse, h, dt):
    ref = with_mass(x, cls, y, ylse, h, dt)
    d = derivative(x, cls, y, ylse, h)
    assert (d - ref["dx"]).abs().max() <= 1e-9 * (1 + d.abs().max())
    check_all(E.distill(x, cls, y, teacher_lse=ylse, temperature=h), ref)


@pytest.mark.parametrize("dt", [BF, F32])
@pytest.mark.parametrize("by", [1e-3, 0.05, 0.7, 2.0])
@pytest.mark.parametrize("V", [100, 5000, 60_001, 70_001])
def test_mass_above_one(V, by, dt):
    """A log-sum too small for its list: the rest is 0, and p counts as often as the list's mass."""
    h = (1.0, 2.0, 0.7)[V % 3]
    x, cls, y, ylse, _, _ = make(V, 2, 9, V, 6, dt, tail=True, h=h)
    check_mass(x, cls, y, torch.logsumexp(y.double() / h, -1).float() - by, h, dt)


@pytest.mark.parametrize("V", [100, 5000, 60_001])
def test_mass_of_rounded_logits(V):
    """What a store of teachers' logits holds: the best ones in bf16, and the log-sum of all of them unrounded."""
    x, cls, _, _, _, _ = make(V, 1, 200, V, 8, BF, tail=True)
    g = gen(V)
    exact = 14.0 + 2.0 * torch.randn(cls.shape, generator=g, device=DEV)
    ylse = torch.logsumexp(exact.double(), -1).float() + 1e-3
    y = exact.to(BF)
    above = torch.logsumexp(y.double(), -1) > ylse.double()
    assert 0 < above.sum() < above.numel()
    check_mass(x, cls, y, ylse, 1.0, BF)


@pytest.mark.parametrize("V", [1, 7, 200])
@pytest.mark.parametrize("by", [-0.5, 0.0, 0.5])
def test_mass_of_all_classes(by, V):
    """Lists of every class: no rest, whatever their mass, below 1 or above."""
    x, cls, y, _, _, _ = make(V, 2, 15, V, V, F32)
    check_mass(x, cls, y, torch.logsumexp(y.double(), -1).float() + by, 1.0, F32)


@pytest.mark.parametrize("V", [300, 60_001, 70_001])
def test_mass_of_far_rows(V):
    """Rows that take the slow way: logits beyond 2^27, and others masked to -inf."""
    x, cls, y, _, free = lists(V, 4, V, 5, F32, True, 1.0)
    x[:, :2] += 1e9
    x[:, 2:] = torch.where(free[:, 2:], float("-inf"), x[:, 2:])
    ylse = torch.logsumexp(y.double(), -1).float() - 0.5
    ref = with_mass(x, cls, y, ylse, 1.0, F32)
    # Classes of p = 0 have a gradient of 0, to the bit; the formulas' shares of their empty sum are no numbers.
    none = x == float("-inf")
    ref["dx"], ref["tdx"] = torch.where(none, 0.0, ref["dx"]), torch.where(none, 0.0, ref["tdx"])
    check_all(E.distill(x, cls, y, teacher_lse=ylse), ref)


def test_mass_of_longest_rows():
    x, cls, y, _, _, _ = make(3, 1, 3, 1_000_003, 5, BF)
    check_mass(x, cls, y, torch.logsumexp(y.double(), -1).float() - 0.5, 1.0, BF)


@pytest.mark.parametrize("by", [0.3, 1.5])
def test_gradient_against_differences_above_one(by):
    """As test_gradient_against_differences of test_gpu_distill.py, with a log-sum that is too small: third
    derivatives grow with the list's mass."""
    h, s = 1.3, 2.0 ** -5
    x, cls, y, _, _, _ = make(10, 2, 12, 400, 20, F32, tail=True, h=h)
    ylse = torch.logsumexp(y.double() / h, -1).float() - by
    _, _, dx = E.distill(x, cls, y, teacher_lse=ylse, temperature=h)
    v = torch.randn(x.shape, generator=gen(11), device=DEV) * 0.2
    L = [E.distill(x + k * s * v, cls, y, teacher_lse=ylse, temperature=h)[0].double().sum().item() for k in (1, -1)]
    ref = reference(x, cls, y, ylse, h, None, None, F32)
    slope = (dx.double() * v.double()).sum().item()
    bend = float(np.exp(by)) * (((v.amax(-1) - v.amin(-1)).double() / h) ** 3).sum().item() * 2 * s * s / 6
    noise = 4 * ref["tloss"].sum().item() / (2 * s) + 2 * U * x.abs().sum().item() / x.shape[-1] / (2 * s)
    assert abs((L[0] - L[1]) / (2 * s) - slope) <= bend + noise + 1e-4 * abs(slope)


@pytest.mark.parametrize("K", [1, 20, 64, 256])
@pytest.mark.parametrize("V", [300, 9000, 70_001])
def test_small_rest(V, K):
    """q_r = 1 - sum q keeps its digits where little is left over. A listed class of p = 0 has the gradient -q, which
    gives each q as the kernel has it; with p = 0 at the others and their logits equal, their gradients add up to -q_r.
    So q_r is known from the q: the sum in 64 bits is off by K 2^-53; the difference, the share and the sum of the
    others' gradients round it by u a step (V / 32 + 160 u covers a sum over the classes)."""
    x, cls, y, _, free = lists(V + K, 12, V, K, F32, True, 1.0)
    mass = torch.logspace(-6, -1, 12, dtype=torch.float64, device=DEV)
    ylse = (torch.logsumexp(y.double(), -1) - torch.log1p(-mass)).float()
    _, _, dx = E.distill(torch.where(free, 0.0, -1e4), cls, y, teacher_lse=ylse)
    q = -dx.gather(-1, cls).double()
    want = 1 - q.sum(-1)
    assert bool((q > 0).all()) and bool((want > 0).sum() > 8)
    _, _, dx = E.distill(torch.where(free, -1e4, 0.0), cls, y, teacher_lse=ylse)
    got = -torch.where(free, dx, 0.0).double().sum(-1)
    off = (got - want.clamp_min(0)).abs()
    assert bool((off <= (V / 32 + 160) * U * want.clamp_min(0) + K * 2.0 ** -53).all())


@pytest.mark.parametrize("dt", [BF, F32])
@pytest.mark.parametrize("V", [300, 9000, 70_001])
@pytest.mark.parametrize("tail", [False, True])
def test_differences_beyond_floats(tail, V, dt):
    """Logits of 3e38 and -3e38 in one row, at temperatures that make ordinary numbers of them: their differences
    are no floats. On either side, listed and not, the student's and the teacher's."""
    for h in (1e37, 5e37):
        h = float(np.float32(h))
        x, cls, y, ylse, free = lists(V, 8, V, 4, dt, tail, h)
        big = 3e38
        x = x.float() * (h / 4)
        x[:, 0] = torch.where(free[:, 0], -big, big)
        x[:, 1] = torch.where(free[:, 1], big, -big)
        x[:, 2] = torch.where(torch.arange(V, device=DEV) % 2 == 0, -big, big)
        x[:, 3] = torch.where(torch.arange(V, device=DEV) == cls[:, 3, :1], big, -big)
        x[:, 4, V // 2:] = -big
        x[:, 4, : V // 2] = big
        x = x.to(dt)
        if not tail:
            y[:, 5, 0], y[:, 5, 1] = big, -big
            y[:, 0, 2] = -big
        ref = reference(x, cls, y, ylse, h, None, None, dt)
        # Gradients of 1 / h are below 2^-126, where steps no longer shrink: half of one, 2^-134 in bf16, for the result,
        # and 2^-150 each for the share's factor, its product (with at most 1) and w / h times a difference.
        ref["tdx"] = ref["tdx"] + (2.0 ** -134 if dt == BF else 2.0 ** -150) + 3 * 2.0 ** -150
        got = E.distill(x, cls, y, teacher_lse=ylse, temperature=h)
        # Of 4 h times a normal number some of the teacher's logits are +inf: their rows have no finite loss.
        fine = ~(y == float("inf")).any(-1)[0]
        assert not bool(torch.isfinite(got[0][0, ~fine]).any())
        check_all([t[:, fine] for t in got], {k: v[:, fine] for k, v in ref.items()})
