"""GPU checks of distillation from a teacher's top logits and of its gradient against the
formulas in float64.

Tolerances, with u = 2^-24 (fp32) and v = 2^-8 (bf16), the unit roundoffs; h is the temperature:
* x / h and y / h are formed with the rounded 1 / h, differences from a maximum first: a probability of the student's
  has a logarithm that is off by 4 u (max - x) / h, whatever the maximum is, and by the sum's error; the exponentials
  of the sums by 128 u (2 u from the function, u |x - max| / h each from the difference and its scaling; terms
  below e^-30 of the sum do not count); the sums over V or K terms are split over at least 32 threads: V / 32 + 16 u.
  Probabilities below what floats hold are 0 (`TINY`).
* the loss is a sum of at most K + 1 products, each off by the errors of its two factors; its sum adds (K / 32 + 16) u
  of the magnitudes.
* q_r = 1 - sum q is off by the sum's error: that of q times q, and u.
* a gradient is (w / h) (p - q) or (w / h) (p_r - q_r) times a class's share of p_r, and is rounded once.
"""
import numpy as np
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

from paper_2609_37842_gb300 import eogp as E  # noqa: E402

DEV = "cuda:0"
U, VB = 2.0 ** -24, 2.0 ** -8
BF, F32 = torch.bfloat16, torch.float32
TINY = 2.0 ** -125


@pytest.fixture(scope="module", autouse=True)
def _lib():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    from paper_2609_37842_gb300 import build
    build.build()
    E.lib()
    yield
    torch.cuda.empty_cache()


@pytest.fixture(autouse=True)
def _status():
    yield
    E.sync_status()


def gen(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    return g


def out_u(dt):
    return VB if dt == BF else U


def make(seed, B, T, V, K, dt, ydt=F32, index=torch.int64, tail=False, h=1.0, lengths=None, weighted=False,
         fewer=False):
    """Logits, lists of K distinct classes in random order, and the teacher's log-sum (None without tail)."""
    g = gen(seed)
    K = min(K, V)
    cls = torch.rand((B * T, V), generator=g, device=DEV).topk(K, -1).indices.view(B, T, K)
    y = (4 * torch.randn((B, T, K), generator=g, device=DEV)).to(ydt)
    x = 2 * torch.randn((B, T, V), generator=g, device=DEV)
    x.scatter_add_(2, cls, 0.7 * y.float())
    x = x.to(dt)
    lse = None
    if tail:
        mass = 0.3 * torch.rand((B, T), generator=g, device=DEV)
        lse = torch.logsumexp(y.float() / h, -1) - torch.log1p(-mass)
    if fewer:
        kept = torch.randint(0, K + 1, (B, T, 1), generator=g, device=DEV)
        cls = torch.where(torch.arange(K, device=DEV) < kept, cls, -7)
    w = None
    if weighted:
        w = torch.rand((B, T), generator=g, device=DEV) + 0.5
        w[torch.rand((B, T), generator=g, device=DEV) < 0.2] = 0.0
    ln = None
    if lengths is not None:
        ln = torch.tensor(lengths, dtype=torch.int32, device=DEV)
        pad = torch.arange(T, device=DEV)[None] >= ln[:, None]
        x[pad] = float("nan")
        y[pad] = float("inf")
    return x, cls.to(index), y, lse, w, ln


def reference(x, cls, y, ylse, h, w, ln, dt, counted=None):
    B, T, V = x.shape
    K = cls.shape[-1]
    if counted is None:
        counted = torch.ones((B, T), dtype=torch.bool, device=DEV)
    if w is not None:
        counted = counted & (w != 0)
    if ln is not None:
        counted = counted & (torch.arange(T, device=DEV)[None] < ln[:, None])
    there = cls >= 0
    if ylse is None:
        counted = counted & (there & (y.float() > float("-inf"))).any(-1)
    xs, c, yy, th = x[counted].double() / h, cls[counted].long().clamp_min(0), y[counted].double() / h, there[counted]
    best = xs.amax(-1, keepdim=True)
    best = torch.where(torch.isfinite(best), best, 0.0)
    xs = xs - best  # float64 would lose the sums beside a maximum of 1e38
    n = xs.shape[0]
    ws = torch.ones(n, dtype=torch.float64, device=DEV) if w is None else w[counted].double()
    yy = torch.where(th, yy, float("-inf"))
    whole = torch.logsumexp(yy, -1) if ylse is None else ylse[counted].double()
    log_q = yy - whole[:, None]
    q = torch.exp(log_q)
    lse = torch.logsumexp(xs, -1)
    log_p = xs.gather(1, c) - lse[:, None]
    mask = torch.zeros((n, V + 1), dtype=torch.bool, device=DEV)
    mask.scatter_(1, torch.where(th, c, V), True)
    mask = mask[:, :V]
    log_pr = torch.logsumexp(xs.masked_fill(mask, float("-inf")), -1) - lse
    q_r = torch.zeros_like(lse) if ylse is None else (1 - q.sum(-1)).clamp_min(0.0)
    q_r = torch.where(mask.all(-1), 0.0, q_r)
    xlogy = lambda a, b: torch.where(a > 0, a * b, torch.zeros_like(a * b))  # noqa: E731
    loss = ws * (xlogy(q, log_q - log_p).sum(-1) + xlogy(q_r, torch.log(q_r) - log_pr))
    # errors of logarithms of p and q, of q_r, and of the sums
    sums = (V / 32 + K / 32 + 160) * U
    rel = torch.where(torch.isinf(xs), 0.0, -4 * U * xs) + 2 * sums  # of each p
    e_k = rel.gather(1, c)  # of each listed one
    e_r = 2 * sums + torch.where(torch.isinf(log_pr), 0.0, 4 * U * log_pr.abs())  # of p_r
    live = torch.where(q > 0, yy.abs(), 0.0)
    e_q = 4 * U * (live.amax(-1) + whole.abs()) + sums
    e_qr = e_q * q.sum(-1) + 2 * U
    log_span = torch.where(q > 0, log_q.abs() + log_p.abs(), 0.0)
    tloss = ws * ((q * (e_k + e_q[:, None]) * (1 + log_span)).sum(-1) * 2 + (K / 32 + 16) * U * (q * log_span).sum(-1))
    if ylse is not None:
        span = torch.where(q_r > 0, torch.log(q_r).abs() + torch.where(q_r > 0, log_pr.abs(), 0.0) + 2, 0.0)
        tloss = tloss + ws * (e_qr * span + q_r * (2 * e_r + 2 * U * span)) + ws * torch.where(q_r > 0, e_qr, 0.0)
    lse = lse + best[:, 0]
    tlse = 2 * sums + 4 * U * (best[:, 0].abs() + lse.abs())
    share = torch.softmax(xs.masked_fill(mask, float("-inf")), -1)
    share = torch.where(mask, 0.0, share)
    d = share * (torch.exp(log_pr) - q_r)[:, None]
    p_r = torch.exp(log_pr)
    td = share * ((p_r * e_r + e_qr)[:, None] + (p_r + q_r)[:, None] * (rel + e_r[:, None])) + TINY
    p = torch.softmax(xs, -1)
    d, td = torch.where(mask, p, d), torch.where(mask, p * rel + TINY, td)
    add = torch.zeros((n, V + 1), dtype=torch.float64, device=DEV)
    tadd = add.clone()
    add.scatter_add_(1, torch.where(th, c, V), torch.where(th, q, 0.0))
    tadd.scatter_add_(1, torch.where(th, c, V), torch.where(th, q * (e_q[:, None] + 4 * U), 0.0))
    d, td = (d - add[:, :V]) * (ws / h)[:, None], (td + tadd[:, :V]) * (ws / h)[:, None]
    td = td + (out_u(dt) + 4 * U) * (d.abs() + td)
    full = {}
    for name, v, tol in (("loss", loss, tloss), ("lse", lse, tlse), ("dx", d, td)):
        for key, val in ((name, v), ("t" + name, tol)):
            out = torch.zeros((B, T, *v.shape[1:]), dtype=torch.float64, device=DEV)
            out[counted] = val
            full[key] = out
    return full


def check(got, want, tol, what):
    assert got.shape == want.shape, what
    got = got.double()
    fine = torch.isfinite(want)
    assert torch.equal(fine, torch.isfinite(got)), f"{what}: finite in other places"
    d = torch.where(fine, (got - torch.where(fine, want, 0.0)).abs(), 0.0)
    tol = torch.where(torch.isfinite(tol), tol, 0.0)
    worst = (d / tol.clamp_min(1e-300)).max().item() if got.numel() else 0.0
    print(f"{what}: worst error / tolerance {worst:.3g}")
    assert worst <= 1.0, f"{what}: {worst:.3g} of the tolerance"


def check_all(got, ref):
    loss, lse, dx = got
    check(loss, ref["loss"], ref["tloss"], "loss")
    check(lse, ref["lse"], ref["tlse"], "lse")
    if dx is not None:
        check(dx, ref["dx"], ref["tdx"], "dlogits")


SIZES = [
    # shortest rows and lists, rows of warps, of one block, of clusters, of odd lengths
    (1, 1, 1, 1), (1, 3, 2, 1), (2, 3, 5, 5), (1, 7, 31, 4), (2, 9, 257, 16), (3, 50, 1000, 64), (2, 33, 2048, 256),
    (1, 40, 4099, 100), (2, 17, 8192, 31), (5, 100, 3001, 20), (1, 5, 50_001, 128), (1, 37, 33_000, 8),
    (1, 3, 131_072, 256), (2, 2, 200_003, 33),
]


@pytest.mark.parametrize("dt", [BF, F32])
@pytest.mark.parametrize("tail", [False, True])
@pytest.mark.parametrize("B,T,V,K", SIZES)
def test_against_formulas(B, T, V, K, tail, dt):
    h = (1.0, 2.0, 0.7)[V % 3]
    ydt, index = ((F32, torch.int64), (BF, torch.int32))[(V + K) % 2]
    x, cls, y, ylse, w, ln = make(B * T + V + K, B, T, V, K, dt, ydt, index, tail, h, weighted=T % 2 == 0,
                                  fewer=K % 2 == 0)
    got = E.distill(x, cls, y, teacher_lse=ylse, temperature=h, weights=w)
    ref = reference(x, cls, y, ylse, h, w, ln, dt)
    check_all(got, ref)
    loss, lse, none = E.distill(x, cls, y, teacher_lse=ylse, temperature=h, weights=w, want_grad=False)
    assert none is None
    check_all((loss, lse, None), ref)


@pytest.mark.parametrize("dt", [BF, F32])
@pytest.mark.parametrize("V", [300, 6000, 70_001])
@pytest.mark.parametrize("lengths", [[9, 0, 4, 1], [0, 0, 0, 0], [99, -2, 9, 8]])
def test_lengths(lengths, V, dt):
    x, cls, y, ylse, w, ln = make(V, 4, 9, V, 12, dt, tail=True, lengths=lengths, weighted=True)
    got = E.distill(x, cls, y, teacher_lse=ylse, weights=w, lengths=ln)
    check_all(got, reference(x, cls, y, ylse, 1.0, w, ln, dt))


@pytest.mark.parametrize("V", [64, 5000, 70_000])
@pytest.mark.parametrize("tail", [False, True])
def test_empty_lists(V, tail):
    """No entries, or none above -inf: without the teacher's log-sum such positions are left out, whatever their
    logits; with it all its mass is on the other classes, and the gradient is 0."""
    x, cls, y, ylse, w, ln = make(V, 1, 6, V, 8, BF, tail=tail)
    cls[:, 1] = -1
    y[:, 2] = float("-inf")
    y[:, 3, 1:] = float("-inf")
    if not tail:
        x[:, 1] = float("nan")
    ref = reference(x, cls, y, ylse, 1.0, None, None, BF)
    got = E.distill(x, cls, y, teacher_lse=ylse)
    check_all(got, ref)
    assert not got[2][0, 1].any()


@pytest.mark.parametrize("tail", [False, True])
@pytest.mark.parametrize("V", [40, 4100, 60_001])
def test_repeated_classes(V, tail):
    """Each entry counts in the loss, and their sum in the gradient; the remainder leaves the class out once."""
    x, cls, y, ylse, w, ln = make(V, 2, 5, V, 10, F32, tail=tail)
    cls[..., 3] = cls[..., 0]
    cls[..., 9] = cls[..., 0]
    cls[0, :, :] = cls[0, :, :1]
    check_all(E.distill(x, cls, y, teacher_lse=ylse), reference(x, cls, y, ylse, 1.0, None, None, F32))


@pytest.mark.parametrize("tail", [False, True])
def test_all_classes_listed(tail):
    """Lists of every class: nothing remains, and a rounded sum of q below 1 is no mass."""
    x, cls, y, _, _, _ = make(3, 1, 30, 200, 200, F32)
    ylse = torch.logsumexp(y, -1) if tail else None
    check_all(E.distill(x, cls, y, teacher_lse=ylse), reference(x, cls, y, ylse, 1.0, None, None, F32))


@pytest.mark.parametrize("V", [100, 5000, 60_001])
def test_teacher_above_one(V):
    """A log-sum too small for its list: the rest is 0, and the listed classes keep their q."""
    x, cls, y, ylse, w, ln = make(V, 1, 8, V, 6, F32, tail=True)
    ylse = ylse - 2.0
    check_all(E.distill(x, cls, y, teacher_lse=ylse), reference(x, cls, y, ylse, 1.0, None, None, F32))


@pytest.mark.parametrize("dt", [BF, F32])
@pytest.mark.parametrize("V", [300, 9000, 70_001])
@pytest.mark.parametrize("tail", [False, True])
def test_masked_and_large_logits(V, tail, dt):
    """Masks of -inf and of the type's lowest value beside listed classes, logits far from 0, and a student that
    leaves the other classes less than a float holds."""
    x, cls, y, ylse, w, ln = make(V, 1, 8, V, 5, dt, tail=tail)
    free = torch.ones((1, 8, V), dtype=torch.bool, device=DEV).scatter_(2, cls, False)
    half = torch.arange(V, device=DEV) % 2 == 0
    x[:, 0] = torch.where(free[:, 0] & half, float("-inf"), x[:, 0])
    x[:, 1] = torch.where(free[:, 1] & half, torch.finfo(dt).min, x[:, 1])
    x[:, 2] += 3.0e4
    x[:, 3] = torch.where(free[:, 3], x[:, 3] - 200.0, x[:, 3])
    x[:, 4] = torch.where(free[:, 4], x[:, 4], x[:, 4] - 200.0)
    x[:, 5] = -1e9
    x[:, 6] = torch.finfo(dt).min
    check_all(E.distill(x, cls, y, teacher_lse=ylse), reference(x, cls, y, ylse, 1.0, None, None, dt))


@pytest.mark.parametrize("V", [300, 9000, 70_001])
@pytest.mark.parametrize("tail", [False, True])
def test_not_finite(V, tail):
    x, cls, y, ylse, w, ln = make(V, 1, 8, V, 5, F32, tail=tail)
    clean = E.distill(x, cls, y, teacher_lse=ylse)
    other = (cls[0, :, 0] + 1) % V
    x[0, 1, cls[0, 1, 2]] = float("nan")
    x[0, 2, other[2]] = float("nan")
    x[0, 3, other[3]] = float("inf")
    x[0, 4] = float("-inf")
    y[0, 5, 1] = float("nan")
    y[0, 6, 1] = float("inf")
    x[0, 7, cls[0, 7, 1]] = float("-inf")  # a class of the teacher's that the student excludes: infinitely far
    loss, lse, dx = E.distill(x, cls, y, teacher_lse=ylse)
    assert bool(torch.isnan(loss[0, 1:5]).all()) and bool(torch.isnan(lse[0, 1:5]).all())
    assert not bool(torch.isfinite(loss[0, 5:]).any()) and loss[0, 7] == float("inf")
    assert bool(torch.isnan(dx[0, 1:4]).any(-1).all())
    assert torch.equal(loss[0, 0], clean[0][0, 0]) and torch.equal(dx[0, 0], clean[2][0, 0])
    assert bool(torch.isfinite(dx[0, 7]).all())


def strided(t, how):
    B, T, n = t.shape
    fill = 0 if not t.dtype.is_floating_point else float("nan")
    if how == "offset":
        v = torch.full((B * T * n + 1,), fill, dtype=t.dtype, device=DEV)[1:].view(B, T, n)
    elif how == "wide":
        v = torch.full((B, T, n + 24), fill, dtype=t.dtype, device=DEV)[:, :, 8:8 + n]
    elif how == "odd":
        v = torch.full((B, T, n + 3), fill, dtype=t.dtype, device=DEV)[:, :, :n]
    elif how == "cut":
        v = torch.full((B, T + 2, n), fill, dtype=t.dtype, device=DEV)[:, :T]
    else:
        v = torch.full((T, B, n), fill, dtype=t.dtype, device=DEV).transpose(0, 1)
    v.copy_(t)
    return v


@pytest.mark.parametrize("dt", [BF, F32])
@pytest.mark.parametrize("V", [500, 12_000, 70_001])
@pytest.mark.parametrize("how", ["offset", "wide", "odd", "cut", "tokens first"])
def test_layouts(how, V, dt):
    x, cls, y, ylse, w, ln = make(V, 3, 5, V, 7, dt, tail=True, lengths=[5, 2, 4])
    ref = reference(x, cls, y, ylse, 1.0, None, ln, dt)
    dx = strided(torch.zeros_like(x), how)
    check_all(E.distill(strided(x, how), strided(cls, how), strided(y, how), teacher_lse=ylse, lengths=ln, dlogits=dx),
              ref)
    # inputs of one alignment, the gradient of another
    check_all(E.distill(x, cls, y, teacher_lse=ylse, lengths=ln, dlogits=dx), ref)


@pytest.mark.parametrize("dt", [BF, F32])
@pytest.mark.parametrize("V", [70, 500, 12_001, 70_000])
@pytest.mark.parametrize("tail", [False, True])
def test_gradient_over_logits(tail, V, dt):
    x, cls, y, ylse, w, ln = make(V, 2, 30, V, 20, dt, tail=tail, lengths=[30, 21])
    want = E.distill(x, cls, y, teacher_lse=ylse, lengths=ln)
    z = x.clone()
    for a, b in zip(E.distill(z, cls, y, teacher_lse=ylse, lengths=ln, dlogits=z), want):
        assert torch.equal(a, b)


def test_repeated_rows():
    x, cls, y, ylse, w, ln = make(5, 1, 1, 3000, 9, F32, tail=True)
    ex = [t.expand(3, 4, -1) for t in (x, cls, y)]
    lse4 = ylse.expand(3, 4).contiguous()
    a, b = E.distill(*ex, teacher_lse=lse4), E.distill(*(t.contiguous() for t in ex), teacher_lse=lse4)
    for p, q in zip(a, b):
        assert torch.equal(p, q)


@pytest.mark.parametrize("V", [300, 9000, 70_001])
def test_classes_out_of_range(V):
    x, cls, y, ylse, w, ln = make(V, 2, 5, V, 6, BF, tail=True)
    fine = (torch.arange(5, device=DEV) != 2).expand(2, 5)
    want = reference(x, cls, y, ylse, 1.0, None, None, BF, counted=fine)
    for bad in (V, V + 5, 1 << 40):
        c = cls.clone()
        c[:, 2, 3] = bad
        got = E.distill(x, c, y, teacher_lse=ylse)
        with pytest.raises(E.EOGPError) as e:
            E.sync_status()
        assert e.value.code == E.EDEVICE
        check_all(got, want)


@pytest.mark.parametrize("V,M", [(1000, 5000), (20_000, 1500), (100_096, 700)])
def test_many_rows(V, M):
    """More rows than blocks: they are taken in turn."""
    x, cls, y, ylse, w, ln = make(V, 1, M, V, 24, BF, tail=True, weighted=True)
    got = E.distill(x, cls, y, teacher_lse=ylse, weights=w)
    for i in range(0, M, 500):
        s = slice(i, i + 500)
        check_all([t[:, s] for t in got], reference(x[:, s], cls[:, s], y[:, s], ylse[:, s], 1.0, w[:, s], None, BF))
    for a, b in zip(got, E.distill(x, cls, y, teacher_lse=ylse, weights=w)):
        assert torch.equal(a, b)


def test_far_rows():
    """Offsets beyond 2^32 elements."""
    V = 1000
    x, cls, y, ylse, w, ln = make(7, 2, 3, V, 9, BF, tail=True)
    want = E.distill(x, cls, y, teacher_lse=ylse)
    base = torch.empty((1 << 32) + 8 * V, dtype=BF, device=DEV)
    far = base.as_strided((2, 3, V), ((1 << 32) + 8, V, 1))
    far.copy_(x)
    for a, b in zip(E.distill(far, cls, y, teacher_lse=ylse), want):
        assert torch.equal(a, b)
    E.distill(x, cls, y, teacher_lse=ylse, dlogits=far)
    assert torch.equal(far, want[2])


def test_other_stream_and_graph():
    x, cls, y, ylse, w, ln = make(8, 2, 40, 5000, 16, BF, tail=True, lengths=[40, 20])
    want = E.distill(x, cls, y, teacher_lse=ylse, lengths=ln)
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    got = E.distill(x, cls, y, teacher_lse=ylse, lengths=ln, stream=s)
    s.synchronize()
    for a, b in zip(got, want):
        assert torch.equal(a, b)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        out = E.distill(x, cls, y, teacher_lse=ylse, lengths=ln)
    x2, cls2, y2, ylse2, _, _ = make(9, 2, 40, 5000, 16, BF, tail=True)
    for a, b in ((x, x2), (cls, cls2), (y, y2), (ylse, ylse2)):
        a.copy_(b)
    ln.copy_(torch.tensor([3, 40], dtype=torch.int32))
    g.replay()
    torch.cuda.synchronize()
    for a, b in zip(out, E.distill(x, cls, y, teacher_lse=ylse, lengths=ln)):
        assert torch.equal(a, b)


@pytest.mark.parametrize("tail", [False, True])
def test_gradient_against_differences(tail):
    """A central difference of step s is off by s^2 / 6 of the third derivatives: at most (max - min)^3 of the
    direction over h, once for the log-sum and once for the remainder's; and by the two losses' tolerances over 2 s."""
    h, s = 1.3, 2.0 ** -5
    x, cls, y, ylse, w, ln = make(10, 2, 12, 400, 20, F32, tail=tail, h=h, weighted=True)
    _, _, dx = E.distill(x, cls, y, teacher_lse=ylse, temperature=h, weights=w)
    v = torch.randn(x.shape, generator=gen(11), device=DEV) * 0.2
    L = [E.distill(x + k * s * v, cls, y, teacher_lse=ylse, temperature=h, weights=w)[0].double().sum().item()
         for k in (1, -1)]
    ref = reference(x, cls, y, ylse, h, w, None, F32)
    slope = (dx.double() * v.double()).sum().item()
    bend = (w.double() * ((v.amax(-1) - v.amin(-1)).double() / h) ** 3).sum().item() * 2 * s * s / 6
    noise = 4 * ref["tloss"].sum().item() / (2 * s) + 2 * U * x.abs().sum().item() / x.shape[-1] / (2 * s)
    assert abs((L[0] - L[1]) / (2 * s) - slope) <= bend + noise + 1e-4 * abs(slope)


def test_equal_distributions():
    """A student equal to its teacher: loss and gradient are 0 up to rounding."""
    x, _, _, _, _, _ = make(12, 1, 20, 500, 1, F32)
    y, cls = x.topk(40, -1)
    ylse = torch.logsumexp(x.double(), -1).float()
    loss, lse, dx = E.distill(x, cls, y, teacher_lse=ylse)
    check_all((loss, lse, dx), reference(x, cls, y, ylse, 1.0, None, None, F32))
    assert loss.abs().max() < 1e-5 and dx.abs().max() < 1e-5


def test_refusals():
    x, cls, y, ylse, w, ln = make(13, 2, 4, 30, 3, BF, tail=True)
    for bad in (lambda: E.distill(x, cls[:, :3], y), lambda: E.distill(x, cls, y[..., :2]),
                lambda: E.distill(x, cls.float(), y), lambda: E.distill(x, cls, y.half()),
                lambda: E.distill(x.half(), cls, y), lambda: E.distill(x, cls, y, teacher_lse=ylse.double()),
                lambda: E.distill(x, cls, y, teacher_lse=ylse[:1]), lambda: E.distill(x, cls, y, dlogits=x.float()),
                lambda: E.distill(x, cls, y, weights=torch.ones((4, 2), device=DEV)),
                lambda: E.distill(x.transpose(1, 2), cls, y), lambda: E.distill(x, cls.cpu(), y)):
        with pytest.raises(ValueError):
            bad()
    for temperature in (0.0, -1.0, float("nan"), float("inf")):
        with pytest.raises(E.EOGPError) as e:
            E.distill(x, cls, y, temperature=temperature)
        assert e.value.code == E.EINVAL
    wide = torch.zeros((2, 4, E.DISTILL_MAX + 1), dtype=torch.int64, device=DEV)
    with pytest.raises(E.EOGPError):
        E.distill(x, wide, wide.float())
