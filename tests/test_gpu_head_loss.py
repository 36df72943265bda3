"""GPU checks of the token loss through the output matrix and of its gradient against its
formulas in float64.

Tolerances, with u = 2^-24 (fp32) and v = 2^-8 (bf16), the unit roundoffs:
* a logit is a sum of d products in fp32. In any order of rounded sums it is off by at
  most d u sum |x W|; a matrix instruction adds 16 products at a time to its sum, cuts
  each product and the sum off at the last place of the largest, so by 18 u of the
  magnitudes a step: 1.2 d u and 16 u for the rest cover both (`chain`).
* lse is off by the logits' errors averaged with softmax's weights, by the sum over V
  terms and by the exponentials: 128 u covers a term (2 u from the function, u |z - max| each from
  the difference and its scaling; terms below e^-30 of the sum do not count).
* D = w scale (p - e_target): p's relative error is that of its logit and of lse and u |z - lse| twice over, as for
  the exponentials, however small p is (down to where floats end, `TINY`); then D is
  rounded to bf16 (v |D|), or to two bf16 parts (v^2 |D|: each is off by half a step of what it
  rounds) where the weight's gradient is fp32, or is fp32.
* dx and dW are sums of V and of n products: the errors of D times the magnitudes, and
  `chain` again; then one rounding to the type, and one more where it is added to.
"""
import numpy as np
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

from paper_2609_37842_gb300 import eogp as E  # noqa: E402

DEV = "cuda:0"
U, VB = 2.0 ** -24, 2.0 ** -8
BF, F32 = torch.bfloat16, torch.float32
IGNORE = -100
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


def chain(n):
    return (1.2 * n + 16) * U


def out_u(dt):
    return VB if dt == BF else U


def make(seed, B, T, d, V, dt, lengths=None, weighted=False, ignored=0.0, index=torch.int64, scale=1.0):
    g = gen(seed)
    W = (torch.randn((V, d), generator=g, device=DEV) * (2.0 / (d ** 0.5 * scale))).to(dt)
    tgt = torch.randint(0, V, (B, T), generator=g, device=DEV)
    x = torch.randn((B, T, d), generator=g, device=DEV)
    x = (x + W.float()[tgt] * (2 * scale * torch.rand((B, T, 1), generator=g, device=DEV))).to(dt)
    if ignored:
        tgt[torch.rand((B, T), generator=g, device=DEV) < ignored] = IGNORE
    w = None
    if weighted:
        w = torch.rand((B, T), generator=g, device=DEV) + 0.5
        w[torch.rand((B, T), generator=g, device=DEV) < 0.2] = 0.0
    ln = None
    if lengths is not None:
        ln = torch.tensor(lengths, dtype=torch.int32, device=DEV)
        x[torch.arange(T, device=DEV)[None] >= ln[:, None]] = float("nan")
    return x, W, tgt.to(index), w, ln


def counted_of(x, tgt, w, ln):
    c = (tgt != IGNORE).clone()
    if w is not None:
        c &= w != 0
    if ln is not None:
        c &= torch.arange(tgt.shape[1], device=DEV)[None] < ln[:, None]
    return c


def reference(x, W, tgt, w, ln, scale, dt, gdt, counted=None, whole_targets=False):
    """Results and tolerances, positions left out at 0. whole_targets: without a rounding of D at the targets."""
    counted = counted_of(x, tgt, w, ln) if counted is None else counted
    B, T, d = x.shape
    V = W.shape[0]
    xs, t = x[counted].double(), tgt[counted].long()
    n = xs.shape[0]
    ws = torch.ones(n, dtype=torch.float64, device=DEV) if w is None else w[counted].double()
    W64 = W.double()
    z = scale * (xs @ W64.T)
    tz = chain(d) * abs(scale) * (xs.abs() @ W64.abs().T) + U * z.abs()
    lse = torch.logsumexp(z, -1)
    p = torch.softmax(z, -1)
    rows = torch.arange(n, device=DEV)
    tl = (p * tz).sum(-1) + (V / 32 + 128 + 16) * U + 4 * U * (lse.abs() + z.abs().amax(-1))
    zt = z[rows, t]
    loss = ws * (lse - zt)
    tloss = ws * (tl + tz[rows, t] + 4 * U * (lse.abs() + zt.abs())) + 2 * U * loss.abs()
    D = p.clone()
    D[rows, t] -= 1
    D *= (ws * scale)[:, None]
    exact_D = (ws * abs(scale))[:, None] * (p * (tz + tl[:, None] + (8 + 4 * (z - lse[:, None]).abs()) * U) + TINY)
    exact_D[rows, t] += 4 * U * ws * abs(scale)
    tD = exact_D + (VB if dt == BF else U) * (D.abs() + exact_D)
    part = VB if dt == BF and gdt == BF else VB * VB if dt == BF else U
    tDw = exact_D + part * (D.abs() + exact_D)
    if whole_targets:
        tD[rows, t] = exact_D[rows, t] + U * D[rows, t].abs()
        if gdt == BF:  # else two parts, both rounded: v^2 |D| as everywhere
            tDw[rows, t] = tD[rows, t]
    dx = D @ W64
    tdx = tD @ W64.abs() + chain(V) * (D.abs() @ W64.abs())
    tdx = tdx + out_u(dt) * (dx.abs() + tdx)
    dW = D.T @ xs
    tdW = tDw.T @ xs.abs() + chain(n) * (D.abs().T @ xs.abs())
    full = {}
    for name, v, tol in (("loss", loss, tloss), ("lse", lse, tl), ("dx", dx, tdx)):
        for key, val in ((name, v), ("t" + name, tol)):
            out = torch.zeros((B, T, *v.shape[1:]), dtype=torch.float64, device=DEV)
            out[counted] = val
            full[key] = out
    full.update(dW=dW, tdW=tdW)
    return full


def rounded(ref, old, gdt):
    """dW and its tolerance once it has been added to `old` and rounded."""
    want = ref["dW"] if old is None else ref["dW"] + old.double()
    extra = 0.0 if old is None else U * (want.abs() + ref["dW"].abs())
    return want, ref["tdW"] + extra + out_u(gdt) * (want.abs() + ref["tdW"])


def check(got, want, tol, what):
    assert got.shape == want.shape, what
    got = got.double()
    assert bool(torch.isfinite(got).all()), f"{what}: not finite"
    worst = ((got - want).abs() / tol.clamp_min(1e-300)).max().item() if got.numel() else 0.0
    print(f"{what}: worst error / tolerance {worst:.3g}")
    assert worst <= 1.0, f"{what}: {worst:.3g} of the tolerance"


def check_all(got, ref, gdt, old=None):
    loss, lse, dx, dW = got
    check(loss, ref["loss"], ref["tloss"], "loss")
    check(lse, ref["lse"], ref["tlse"], "lse")
    if dx is not None:
        check(dx, ref["dx"], ref["tdx"], "dx")
    if dW is not None:
        want, tol = rounded(ref, old, gdt)
        check(dW, want, tol, "dweight")


SIZES = [
    (1, 1, 64, 1000), (1, 1, 1, 1), (1, 1, 3, 2), (2, 5, 64, 257), (3, 37, 70, 1001), (1, 130, 768, 4099),
    (2, 300, 200, 515), (1, 511, 136, 1030), (5, 129, 264, 256), (1, 64, 2050, 300), (1, 257, 65, 255),
    (7, 191, 128, 2048), (1, 33, 4100, 129), (1, 1, 520, 20_011),
]


@pytest.mark.parametrize("dt,gdt", [(BF, BF), (BF, F32), (F32, F32)])
@pytest.mark.parametrize("B,T,d,V", SIZES)
def test_against_formulas(B, T, d, V, dt, gdt):
    x, W, tgt, w, ln = make(B * T + d + V, B, T, d, V, dt, weighted=V % 2 == 1, ignored=0.1 * (T > 8))
    got = E.head_loss(x, W, tgt, weights=w, dtype=gdt)
    check_all(got, reference(x, W, tgt, w, ln, 1.0, dt, gdt), gdt)
    assert got[2].dtype == dt and got[3].dtype == gdt


@pytest.mark.parametrize("dt", [BF, F32])
@pytest.mark.parametrize("B,T,d,V", SIZES)
def test_loss_alone(B, T, d, V, dt):
    """Without gradients, and with one of them, the values are within the same bounds."""
    x, W, tgt, w, ln = make(B * T + d + V + 1, B, T, d, V, dt, index=torch.int32)
    ref = reference(x, W, tgt, w, ln, 1.0, dt, dt)
    loss, lse, dx, dW = E.head_loss(x, W, tgt, want_dx=False, want_dweight=False)
    assert dx is None and dW is None
    check_all((loss, lse, None, None), ref, dt)
    loss, lse, dx, dW = E.head_loss(x, W, tgt, want_dweight=False)
    assert dW is None
    check_all((loss, lse, dx, None), ref, dt)
    loss, lse, dx, dW = E.head_loss(x, W, tgt, want_dx=False)
    assert dx is None
    check_all((loss, lse, None, dW), ref, dt)


@pytest.mark.parametrize("dt,gdt", [(BF, BF), (BF, F32), (F32, F32)])
@pytest.mark.parametrize("lengths", [[40, 0, 17, 1, 39], [0, 0, 0, 0, 0], [40, 40, 40, 40, 40], [0, 0, 0, 0, 1],
                                     [99, -3, 5, 40, 41]])
def test_lengths_and_weights(lengths, dt, gdt):
    """Padding holds NaN; lengths beyond T keep all of it, negative ones nothing."""
    B, T, d, V = 5, 40, 96, 700
    x, W, tgt, w, ln = make(sum(lengths), B, T, d, V, dt, lengths=lengths, weighted=True, ignored=0.2, scale=0.3)
    old = torch.randn((V, d), generator=gen(5), device=DEV).to(gdt)
    ref = reference(x, W, tgt, w, ln, 0.3, dt, gdt)
    check_all(E.head_loss(x, W, tgt, scale=0.3, weights=w, lengths=ln, dtype=gdt), ref, gdt)
    acc = old.clone()
    check_all(E.head_loss(x, W, tgt, scale=0.3, weights=w, lengths=ln, dweight=acc, accumulate=True), ref, gdt, old)
    if not counted_of(x, tgt, w, ln).any():
        assert torch.equal(acc, old)


def test_no_positions():
    W = torch.randn((50, 16), device=DEV)
    for shape in ((0, 4), (3, 0)):
        x, tgt = torch.zeros((*shape, 16), device=DEV), torch.zeros(shape, dtype=torch.int64, device=DEV)
        loss, lse, dx, dW = E.head_loss(x, W, tgt)
        assert loss.shape == lse.shape == shape and dx.shape == x.shape and not dW.any()
        old = torch.ones_like(W)
        E.head_loss(x, W, tgt, dweight=old, accumulate=True)
        assert bool((old == 1).all())


@pytest.mark.parametrize("ignore", [-100, 3])
def test_everything_ignored(ignore):
    x, W, tgt, _, _ = make(2, 2, 70, 64, 300, BF)
    tgt.fill_(ignore)
    x.fill_(float("nan"))
    loss, lse, dx, dW = E.head_loss(x, W, tgt, ignore_index=ignore)
    assert not loss.any() and not lse.any() and not dx.any() and not dW.any()


def strided(t, how):
    B, T, n = t.shape
    if how == "offset":
        v = torch.full((B * T * n + 1,), float("nan"), dtype=t.dtype, device=DEV)[1:].view(B, T, n)
    elif how == "wide":
        v = torch.full((B, T, n + 24), float("nan"), dtype=t.dtype, device=DEV)[:, :, 8:8 + n]
    elif how == "odd":
        v = torch.full((B, T, n + 3), float("nan"), dtype=t.dtype, device=DEV)[:, :, :n]
    elif how == "cut":
        v = torch.full((B, T + 2, n), float("nan"), dtype=t.dtype, device=DEV)[:, :T]
    else:
        v = torch.full((T, B, n), float("nan"), dtype=t.dtype, device=DEV).transpose(0, 1)
    v.copy_(t)
    return v


@pytest.mark.parametrize("dt", [BF, F32])
@pytest.mark.parametrize("how", ["offset", "wide", "odd", "cut", "tokens first"])
def test_layouts(how, dt):
    """x and dx, the matrix and its gradient laid out in other ways: the same bits as dense ones."""
    B, T, d, V = 3, 50, 72, 333
    x, W, tgt, w, ln = make(9, B, T, d, V, dt, lengths=[50, 7, 31])
    want = E.head_loss(x, W, tgt, lengths=ln)
    dx = strided(torch.zeros_like(x), how)
    Ws = strided(W[None], "cut" if how == "tokens first" else how)[0]
    dW = strided(torch.zeros((1, V, d), device=DEV, dtype=dt), "wide" if how == "tokens first" else how)[0]
    got = E.head_loss(strided(x, how), Ws, tgt, lengths=ln, dx=dx, dweight=dW)
    for a, b in zip(got, want):
        assert torch.equal(a, b)
    if how == "wide":
        assert bool(torch.isnan(dx.as_strided((B, T, d + 24), (T * (d + 24), d + 24, 1), 0)[..., :8]).all())


def test_repeated_rows():
    """Strides of 0: every position has the same row."""
    x, W, tgt, _, _ = make(4, 1, 1, 64, 300, F32)
    tgt = torch.arange(12, device=DEV).view(3, 4)
    one = x.expand(3, 4, 64)
    for a, b in zip(E.head_loss(one, W, tgt), E.head_loss(one.contiguous(), W, tgt)):
        assert torch.equal(a, b)


@pytest.mark.parametrize("dt", [BF, F32])
def test_dx_over_x(dt):
    x, W, tgt, w, ln = make(11, 2, 300, 136, 999, dt, lengths=[300, 201], ignored=0.2)
    want = E.head_loss(x, W, tgt, lengths=ln)
    y = x.clone()
    got = E.head_loss(y, W, tgt, lengths=ln, dx=y)
    for a, b in zip(got, want):
        assert torch.equal(a, b)


def test_targets_out_of_range():
    x, W, tgt, _, _ = make(12, 2, 9, 64, 100, BF)
    want = reference(x, W, tgt, None, None, 1.0, BF, BF, counted=~((torch.arange(9, device=DEV) == 4).expand(2, 9)))
    for bad in (100, -1, 1 << 40, -(1 << 40)):
        t = tgt.clone()
        t[:, 4] = bad
        got = E.head_loss(x, W, t)
        with pytest.raises(E.EOGPError) as e:
            E.sync_status()
        assert e.value.code == E.EDEVICE
        check_all(got, want, BF)


@pytest.mark.parametrize("dt", [BF, F32])
def test_large_logits(dt):
    """Logits of thousands: certain predictions, right and wrong ones."""
    x, W, tgt, _, _ = make(13, 1, 150, 64, 520, dt, scale=1.0)
    ref = reference(x, W, tgt, None, None, 300.0, dt, dt)
    check_all(E.head_loss(x, W, tgt, scale=300.0), ref, dt)


def test_not_finite():
    """A NaN or infinity in one position's x reaches that position alone among losses and dx."""
    for bad in (float("nan"), float("inf")):
        x, W, tgt, _, _ = make(14, 1, 40, 64, 300, BF)
        clean = E.head_loss(x, W, tgt)
        x[0, 5, 3] = bad
        loss, lse, dx, dW = E.head_loss(x, W, tgt)
        assert torch.isnan(loss[0, 5]) and torch.isnan(lse[0, 5])
        keep = torch.arange(40, device=DEV) != 5
        assert torch.equal(loss[0, keep], clean[0][0, keep]) and torch.equal(dx[0, keep], clean[2][0, keep])
        assert bool(torch.isnan(dW).any())


@pytest.mark.parametrize("gdt", [BF, F32])
def test_pieces(gdt):
    """More logits than a piece holds: 4 GB of them, 5,368 rows of 200,000 classes."""
    B, T, d, V = 3, 2100, 64, 200_000
    x, W, tgt, w, ln = make(15, B, T, d, V, BF, lengths=[2100, 2090, 1800], ignored=0.01)
    loss, lse, dx, dW = E.head_loss(x, W, tgt, lengths=ln, dtype=gdt)
    counted = counted_of(x, tgt, None, ln)
    old = torch.randn((V, d), generator=gen(5), device=DEV).to(gdt)
    acc = old.clone()
    E.head_loss(x, W, tgt, lengths=ln, dweight=acc, accumulate=True, want_dx=False)
    # in blocks of positions, their tolerances of dW added up
    at = counted.nonzero()
    dW64 = tol = 0.0
    for i in range(0, at.shape[0], 1000):
        m = torch.zeros_like(counted)
        b = at[i:i + 1000]
        m[b[:, 0], b[:, 1]] = True
        r = reference(x, W, tgt, None, None, 1.0, BF, gdt, counted=m)
        for got, name in ((loss, "loss"), (lse, "lse"), (dx, "dx")):
            check(got[m], r[name][m], r["t" + name][m], name)
        dW64, tol = dW64 + r["dW"], tol + r["tdW"] + chain(counted.sum().item()) * r["dW"].abs()
    for got, before in ((dW, None), (acc, old)):
        want, t = rounded(dict(dW=dW64, tdW=tol), before, gdt)
        check(got, want, t, "dweight")


@pytest.mark.parametrize("dt", [BF, F32])
def test_runs_are_the_same(dt):
    x, W, tgt, w, ln = make(16, 2, 700, 200, 1500, dt, lengths=[700, 333], weighted=True)
    a = E.head_loss(x, W, tgt, weights=w, lengths=ln)
    for _ in range(3):
        for p, q in zip(a, E.head_loss(x, W, tgt, weights=w, lengths=ln)):
            assert torch.equal(p, q)


def test_other_stream_and_graph():
    """On a stream of the caller's; captured and replayed on new values and lengths, two graphs on one workspace."""
    x, W, tgt, w, ln = make(17, 2, 150, 128, 1000, BF, lengths=[150, 80])
    want = E.head_loss(x, W, tgt, lengths=ln)
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    got = E.head_loss(x, W, tgt, lengths=ln, stream=s)
    s.synchronize()
    for a, b in zip(got, want):
        assert torch.equal(a, b)
    ws = E.workspace(1 << 26, DEV)
    dx, dW = torch.empty_like(x), torch.empty_like(W)
    graphs, outs = [], []
    for scale in (1.0, 0.5):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            outs.append(E.head_loss(x, W, tgt, lengths=ln, dx=dx, dweight=dW, ws=ws, scale=scale))
        graphs.append(g)
    x2, _, tgt2, _, _ = make(18, 2, 150, 128, 1000, BF)
    x.copy_(x2)
    tgt.copy_(tgt2)
    ln.copy_(torch.tensor([33, 149], dtype=torch.int32))
    for i in (0, 1, 0):
        graphs[i].replay()
        torch.cuda.synchronize()
        want = E.head_loss(x, W, tgt, lengths=ln, scale=(1.0, 0.5)[i])
        for a, b in zip(outs[i], want):
            assert torch.equal(a, b)


def test_gradient_against_differences():
    """Directional differences of the summed loss in fp32. With a = the logits' change along the direction, the
    third derivative of a row's loss is at most (max a - min a)^3, so a central difference of step h is off by
    h^2 / 6 of their sum, and by the two losses' tolerances over 2 h."""
    B, T, d, V, h = 2, 20, 48, 90, 2.0 ** -5
    x, W, tgt, w, ln = make(19, B, T, d, V, F32, weighted=True)
    _, _, dx, dW = E.head_loss(x, W, tgt, weights=w)
    g = gen(20)
    ref = reference(x, W, tgt, w, None, 1.0, F32, F32)
    noise = 4 * ref["tloss"].sum().item() / (2 * h)
    for which in ("x", "W"):
        v = torch.randn((x if which == "x" else W).shape, generator=g, device=DEV) * 0.1
        if which == "x":
            L = [E.head_loss(x + k * h * v, W, tgt, weights=w)[0].double().sum().item() for k in (1, -1)]
            a, slope = v.double() @ W.double().T, (dx.double() * v.double()).sum().item()
        else:
            L = [E.head_loss(x, W + k * h * v, tgt, weights=w)[0].double().sum().item() for k in (1, -1)]
            a, slope = x.double() @ v.double().T, (dW.double() * v.double()).sum().item()
        bend = (w.double() * (a.amax(-1) - a.amin(-1)) ** 3).sum().item() * h * h / 6
        moved = U * 2 * (x.abs().double() @ W.abs().double().T).amax(-1).sum().item() * 1.5 / (2 * h)
        assert abs((L[0] - L[1]) / (2 * h) - slope) <= bend + noise + moved + 1e-4 * abs(slope)


def test_as_the_token_loss_of_its_logits():
    """The same losses as eogp_cross_entropy on the logits, in a run with the operators around it."""
    x, W, tgt, w, ln = make(21, 3, 60, 128, 640, F32, lengths=[60, 20, 0], weighted=True)
    xz = torch.where(torch.isnan(x), 0.0, x)
    n, mean, rstd = E.norm(xz, torch.ones(128, device=DEV), kind=E.NORM_RMS, lengths=ln)
    loss, lse, dx, dW = E.head_loss(n, W, tgt, weights=w, lengths=ln)
    z = (n.double() @ W.double().T).float()
    want, wlse, dz = E.cross_entropy(z, tgt, weights=w, lengths=ln)
    ref = reference(n, W, tgt, w, ln, 1.0, F32, F32)
    check(loss, want.double(), 2 * ref["tloss"] + 4 * U, "loss")
    check(dx, dz.double() @ W.double(), 2 * ref["tdx"], "dx")
    back, _, _ = E.norm_grad(dx, xz, None, rstd, kind=E.NORM_RMS, lengths=ln, want_dbias=False, want_dweight=False)
    assert bool(torch.isfinite(back).all())


def test_refusals():
    x, W, tgt, _, _ = make(22, 2, 4, 16, 30, BF)
    for bad in (lambda: E.head_loss(x, W.float(), tgt), lambda: E.head_loss(x, W[:, :8], tgt),
                lambda: E.head_loss(x, W.T, tgt), lambda: E.head_loss(x, W, tgt[:, :3]),
                lambda: E.head_loss(x, W, tgt.float()), lambda: E.head_loss(x, W, tgt, accumulate=True),
                lambda: E.head_loss(x, W, tgt, dx=x.float()), lambda: E.head_loss(x, W, tgt, dweight=W[:5]),
                lambda: E.head_loss(x, W, tgt, weights=torch.ones((2, 5), device=DEV)),
                lambda: E.head_loss(x, W, tgt, lengths=torch.ones(3, dtype=torch.int32, device=DEV)),
                lambda: E.head_loss(x, W, tgt.cpu())):
        with pytest.raises(ValueError):
            bad()
    with pytest.raises(E.EOGPError) as e:
        E.head_loss(x.float(), W.float(), tgt, dtype=BF)
    assert e.value.code == E.EUNSUPPORTED
    with pytest.raises(E.EOGPError) as e:
        E.head_loss(x, W, tgt, ws=E.workspace(512, DEV))
    assert e.value.code == E.EWORKSPACE


@pytest.mark.parametrize("B,T,d,V,dt,gdt", [
    (2, 2600, 64, 400_000, BF, BF),   # D kept alone, in one part
    (1, 2100, 1032, 600_000, BF, BF),  # wide rows: D in the logits' place
    (1, 1500, 40, 300_001, F32, F32),
])
def test_pieces_of_each_form(B, T, d, V, dt, gdt):
    """More than a piece holds in each of the forms that D is kept in; dW's sum over the pieces, and on top of old ones."""
    x, W, tgt, w, ln = make(23, B, T, d, V, dt, ignored=0.01)
    loss, lse, dx, dW = E.head_loss(x, W, tgt, dtype=gdt)
    old = torch.randn((V, d), generator=gen(5), device=DEV).to(gdt)
    acc = old.clone()
    E.head_loss(x, W, tgt, dweight=acc, accumulate=True, want_dx=False)
    counted = counted_of(x, tgt, None, None)
    at = counted.nonzero()
    dW64 = tol = 0.0
    for i in range(0, at.shape[0], 550):
        m = torch.zeros_like(counted)
        b = at[i:i + 550]
        m[b[:, 0], b[:, 1]] = True
        r = reference(x, W, tgt, None, None, 1.0, dt, gdt, counted=m)
        for got, name in ((loss, "loss"), (lse, "lse"), (dx, "dx")):
            check(got[m], r[name][m], r["t" + name][m], name)
        dW64, tol = dW64 + r["dW"], tol + r["tdW"] + chain(counted.sum().item()) * r["dW"].abs()
    for got, before in ((dW, None), (acc, old)):
        want, t = rounded(dict(dW=dW64, tdW=tol), before, gdt)
        check(got, want, t, "dweight")


@pytest.mark.parametrize("gdt", [BF, F32])
@pytest.mark.parametrize("B,T,d,V", [(1, 2048, 64, 257), (3, 1000, 72, 1001), (2, 1030, 513, 700), (1, 2500, 768, 4099),
                                     (4, 700, 1024, 321), (2, 1300, 1032, 511), (1, 2304, 8, 63)])
def test_many_positions(B, T, d, V, gdt):
    """Enough positions that the logits may be formed twice instead of kept, at widths on both sides of that choice."""
    x, W, tgt, w, ln = make(B * T + d, B, T, d, V, BF, lengths=[T] + [T // 3] * (B - 1), weighted=True, ignored=0.1)
    got = E.head_loss(x, W, tgt, scale=0.7, weights=w, lengths=ln, dtype=gdt)
    check_all(got, reference(x, W, tgt, w, ln, 0.7, BF, gdt), gdt)
    for a, b in zip(got, E.head_loss(x, W, tgt, scale=0.7, weights=w, lengths=ln, dtype=gdt)):
        assert torch.equal(a, b)
    few = tgt.clone()
    few.view(-1)[5:] = IGNORE  # hardly any of them counted
    got = E.head_loss(x, W, few, dtype=gdt, lengths=ln)
    check_all(got, reference(x, W, few, None, ln, 1.0, BF, gdt), gdt)


@pytest.mark.parametrize("gdt", [BF, F32])
@pytest.mark.parametrize("B,T,d,V", [(1, 1, 64, 500), (1, 60, 72, 4099), (2, 300, 770, 2000), (1, 511, 768, 30_001),
                                     (1, 2300, 136, 9000), (3, 900, 1032, 8191)])
def test_targets_are_not_rounded(B, T, d, V, gdt):
    """D's largest entry in a row, at the target, enters dx and a dW of bf16 as in fp32: rounded to bf16 and the rest
    added; a dW of fp32 in two parts (a few positions a class here, fewer than a dW of bf16 has turns for)."""
    x, W, tgt, w, ln = make(B * T + d + 3, B, T, d, V, BF, weighted=True, ignored=0.1 * (T > 8))
    tgt = torch.where(tgt == IGNORE, tgt, torch.randperm(V, generator=gen(1), device=DEV).repeat(2)[:B * T].view(B, T))
    ref = reference(x, W, tgt, w, ln, 1.0, BF, gdt, whole_targets=True)
    check_all(E.head_loss(x, W, tgt, weights=w, dtype=gdt), ref, gdt)


def test_one_class_for_all():
    """Every position has the same target: more positions of a class than have their own turn."""
    x, W, tgt, _, _ = make(24, 2, 1000, 64, 1000, BF)
    tgt.fill_(777)
    got = E.head_loss(x, W, tgt)
    check_all(got, reference(x, W, tgt, None, None, 1.0, BF, BF), BF)
    for a, b in zip(got, E.head_loss(x, W, tgt)):
        assert torch.equal(a, b)


def test_two_streams_at_once():
    """Calls on two streams, one after the other on the host, each with a workspace of its own."""
    sets = [make(30 + k, 2, 400, 256, 3000, (BF, F32)[k], lengths=[400, 100 + k]) for k in range(2)]
    want = [E.head_loss(x, W, tgt, lengths=ln) for x, W, tgt, _, ln in sets]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in sets]
    for _ in range(5):
        got = [E.head_loss(x, W, tgt, lengths=ln, stream=s) for (x, W, tgt, _, ln), s in zip(sets, streams)]
        torch.cuda.synchronize()
        for g, w in zip(got, want):
            for a, b in zip(g, w):
                assert torch.equal(a, b)
