"""GPU checks of the model-end operators over many rows, where blocks take several
rows in turn, rings of buffers wrap and sums are joined from many blocks. The
formulas are evaluated in float64 on the device.

Sums over rows are checked exactly: with whole numbers of a few bits, statistics that
are whole numbers and powers of two, every product and every partial sum in any order
is below 2^24 and so is exact in fp32, and a row that is lost, doubled or put in a
wrong place shows. Tolerances of the other results, with u = 2^-24 and v = 2^-8 the
unit roundoffs of fp32 and bf16: a rounding to the result's type (v or u of it), a sum
of n terms split over at least 32 threads (n / 32 + 16) u of the terms' magnitudes,
and 128 u for an exponential whose argument is above -30.
"""
import numpy as np
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

from paper_2609_37842_gb300 import eogp as E  # noqa: E402

DEV = "cuda:0"
U, VB = 2.0 ** -24, 2.0 ** -8
BF, F32 = torch.bfloat16, torch.float32


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


def whole(g, shape, dt, most):
    """Whole numbers from -most to most."""
    return torch.randint(-most, most + 1, shape, generator=g, device=DEV).to(dt)


def ragged(g, B, T):
    ln = torch.randint(0, T + 1, (B,), generator=g, device=DEV, dtype=torch.int32)
    ln[:3] = torch.tensor([0, T, 1], dtype=torch.int32)
    return ln


def kept(B, T, ln):
    k = torch.ones((B, T), dtype=torch.bool, device=DEV)
    return k if ln is None else torch.arange(T, device=DEV)[None] < ln[:, None]


def check(got, want, tol, what):
    got = got.double()
    assert got.shape == want.shape and torch.isfinite(got).all(), what
    over = (got - want).abs() - tol
    assert torch.all(over <= 0), f"{what}: {over.max().item():.3g} over the tolerance"


# --------------------------------------------------------------- embedding
@pytest.mark.parametrize("dt", [F32, BF])
@pytest.mark.parametrize("B,T,V,d,tokens,with_lengths", [
    (1, 5000, 100, 64, "even", False), (9, 1000, 511, 40, "even", True), (2, 4500, 512, 24, "even", False),
    (70, 300, 50_257, 128, "zipf", True), (1, 40_000, 262_143, 16, "zipf", False),
    (1, 30_000, 262_144, 16, "even", False), (5, 2500, 1_000_000, 8, "even", True),
    (1, 60_000, 3000, 72, "one", False), (40, 1500, 3000, 77, "one", True), (3, 20_000, 40, 130, "zipf", False),
    (1, 4097, 2, 770, "even", False), (1, 9000, 700, 1, "zipf", False), (64, 1024, 32_000, 200, "halves", False)])
def test_embed_grad(dt, B, T, V, d, tokens, with_lengths):
    g = gen(B + T + V + d)
    if tokens == "zipf":
        tok = (torch.rand((B, T), generator=g, device=DEV) * np.log(V + 1)).exp().long().clamp(1, V) - 1
    else:
        tok = torch.randint(0, V, (B, T), generator=g, device=DEV)
        if tokens == "one":          # most positions hold one token
            tok[torch.rand((B, T), generator=g, device=DEV) < 0.9] = V // 2
        elif tokens == "halves":     # two tokens hold the front and the back
            tok[:B // 2], tok[B // 2:, T // 2:] = V - 1, 0
    ln = ragged(g, B, T) if with_lengths else None
    keep = kept(B, T, ln)
    dout = whole(g, (B, T, d), dt, 15)       # 15 x 65536 < 2^24
    dout[~keep] = float("nan")
    want = torch.zeros((V, d), dtype=torch.float64, device=DEV)
    want.index_add_(0, tok[keep], dout[keep].double())
    for idt in (torch.int32, torch.int64):
        got = E.embed_grad(tok.to(idt), dout, V, scale=0.5, lengths=ln, dtype=F32)
        assert torch.equal(got.double(), want * 0.5)
    base = whole(g, (V, d), F32, 9)
    acc = base.clone()
    E.embed_grad(tok, dout, V, lengths=ln, dtable=acc, accumulate=True)
    assert torch.equal(acc.double(), base.double() + want)
    assert torch.equal(E.embed_grad(tok, dout, V, lengths=ln, dtype=BF), want.float().to(BF))


@pytest.mark.parametrize("dt", [F32, BF])
@pytest.mark.parametrize("d", [8, 64, 100, 256, 384, 520, 770, 1536, 2560])
def test_embed(dt, d):
    g = gen(d)
    B, T, V = 31, 700, 5000
    tok, ln = torch.randint(0, V, (B, T), generator=g, device=DEV), ragged(g, B, T)
    table, pos = whole(g, (V, d), dt, 60), whole(g, (T, d), dt, 60)   # sums of at most 8 bits: exact in bf16
    keep = kept(B, T, ln)[..., None]
    want = torch.where(keep, table[tok] * 2 + pos[None], torch.zeros((), dtype=dt, device=DEV))
    assert torch.equal(E.embed(tok, table, scale=2.0, pos=pos, lengths=ln), want)
    assert torch.equal(E.embed(tok.int(), table), table[tok])


# ----------------------------------------------------------- normalisation
WIDTHS = [(40_000, 8), (40_000, 64), (40_000, 72), (30_000, 100), (30_000, 128), (30_000, 250), (30_000, 256),
          (20_000, 384), (20_000, 512), (20_000, 520), (20_000, 770), (20_000, 1536), (12_000, 2560), (9000, 4100),
          (6000, 5120), (5000, 8192), (3000, 12_000), (1200, 16_384), (1000, 20_001)]


@pytest.mark.parametrize("kind", [E.NORM_LAYER, E.NORM_RMS])
@pytest.mark.parametrize("dt,pt", [(F32, F32), (BF, BF), (BF, F32), (F32, BF)])
@pytest.mark.parametrize("rows,d", WIDTHS)
def test_norm(kind, dt, pt, rows, d):
    g = gen(rows + d)
    B, T = 10, rows // 10
    ln, rms = ragged(g, B, T), kind == E.NORM_RMS
    keep = kept(B, T, ln)
    x = torch.randn((B, T, d), generator=g, device=DEV).add_(0.5).to(dt)
    x[~keep] = float("nan")
    w = torch.randn((d,), generator=g, device=DEV).add_(1).to(pt)
    b = None if rms else torch.randn((d,), generator=g, device=DEV).to(pt)
    y, mean, rstd = E.norm(x, w, b, kind=kind, eps=1e-5, lengths=ln)
    X = torch.where(keep[..., None], x.double(), 0.0)
    mu = torch.zeros((B, T, 1), dtype=torch.float64, device=DEV) if rms else X.mean(-1, keepdim=True)
    r = ((X - mu).square().mean(-1, keepdim=True) + 1e-5).rsqrt()
    xh = (X - mu) * r
    bb = 0.0 if b is None else b.double()
    want = (xh * w.double() + bb) * keep[..., None]
    c = (d / 32 + 24) * U
    tol = (c * (xh.abs() + r * (X.abs().mean(-1, keepdim=True) + X.abs())) * w.double().abs()
           + 4 * U * ((xh * w.double()).abs() + (0.0 if b is None else bb.abs())))
    check(y, want, tol * keep[..., None] + (VB if dt == BF else U) * want.abs(), "y")
    check(rstd, (r * keep[..., None])[..., 0], c * (r[..., 0] + r[..., 0] ** 2 * X.abs().mean(-1)), "rstd")
    if not rms:
        check(mean, mu[..., 0] * keep, c * X.abs().mean(-1) + U * mu[..., 0].abs(), "mean")


@pytest.mark.parametrize("kind", [E.NORM_LAYER, E.NORM_RMS])
@pytest.mark.parametrize("dt,pt", [(F32, F32), (BF, BF), (BF, F32), (F32, BF)])
@pytest.mark.parametrize("rows,d", WIDTHS)
def test_norm_grad(kind, dt, pt, rows, d):
    g = gen(rows + d)
    rms = kind == E.NORM_RMS
    for B, with_lengths in ((1, False), (10, True)):
        T = rows // B
        ln = ragged(g, B, T) if with_lengths else None
        keep = kept(B, T, ln)
        x, dy = whole(g, (B, T, d), dt, 7), whole(g, (B, T, d), dt, 4)
        x[~keep], dy[~keep] = float("nan"), float("inf")
        w = whole(g, (d,), pt, 3)
        # (x - mean) rstd: multiples of 1/2 of at most 10; its products with dy sum to less than 2^23
        mean = whole(g, (B, T), F32, 3)
        rstd = torch.randint(0, 2, (B, T), generator=g, device=DEV).float() * 0.5 + 0.5
        k = keep[..., None]
        X, DY = torch.where(k, x.double(), 0.0), torch.where(k, dy.double(), 0.0)
        M, R = mean.double()[..., None], rstd.double()[..., None]
        if rms:
            M = torch.zeros_like(M)
        xh = (X - M) * R * k
        for ww in (w, None):
            G = DY if ww is None else DY * w.double()
            m1 = torch.zeros_like(M) if rms else G.mean(-1, keepdim=True)
            m2 = (G * xh).mean(-1, keepdim=True)
            dx_w = (G - m1 - xh * m2) * R * k
            # xh and g are exact, and so are their sums but for the division by d; xh m2 may be taken in two parts
            tol = (8 * U * R * (G.abs() + m1.abs() + (X.abs() + M.abs()) * R * m2.abs())
                   + (VB if dt == BF else U) * dx_w.abs())
            for per in (False, True):
                dx, dw, db = E.norm_grad(dy, x, None if rms else mean, rstd, ww, kind=kind, lengths=ln,
                                         per_example=per)
                over = (1,) if per else (0, 1)
                assert torch.equal(dw.double(), (DY * xh).sum(over)), "dweight"
                assert torch.equal(db.double(), DY.sum(over)), "dbias"
                check(dx, dx_w, tol, "dx")


@pytest.mark.parametrize("per", [False, True])
@pytest.mark.parametrize("d,dt", [(64, BF), (768, BF), (770, F32), (4096, BF), (2048, F32)])
@pytest.mark.parametrize("T,lengths", [(64, [0, 0, 0]), (100, [0] * 40), (64, [0] * 20 + [1] + [0] * 20),
                                       (3000, [0, 0, 3000, 0]), (5000, [1]), (5000, [4999]), (300, [300, 0] * 30),
                                       (90, [90] * 50 + [0] * 50), (200, [0] * 50 + [200] * 50 + [1])])
def test_norm_grad_uneven_lengths(T, lengths, d, dt, per):
    """Rows are shared out by the work of the lengths: none at all, a few, all in one place; with and without dx."""
    g = gen(T + d)
    B = len(lengths)
    ln = torch.tensor(lengths, dtype=torch.int32, device=DEV)
    keep = kept(B, T, ln)[..., None]
    x, dy = whole(g, (B, T, d), dt, 7), whole(g, (B, T, d), dt, 4)
    x.masked_fill_(~keep, float("nan"))
    dy.masked_fill_(~keep, float("nan"))
    rstd = torch.ones((B, T), device=DEV)
    X, DY = torch.where(keep, x.double(), 0.0), torch.where(keep, dy.double(), 0.0)
    over = (1,) if per else (0, 1)
    args = dict(kind=E.NORM_RMS, lengths=ln, per_example=per)
    for want_dx in (True, False):
        dx, dw, db = E.norm_grad(dy, x, None, rstd, None, want_dx=want_dx, **args)
        assert torch.equal(dw.double(), (DY * X).sum(over)) and torch.equal(db.double(), DY.sum(over))
        if want_dx:
            full = dx
            assert not torch.where(keep, 0.0, dx.double()).any() and torch.isfinite(dx).all()
    only = E.norm_grad(dy, x, None, rstd, None, want_dweight=False, want_dbias=False, **args)[0]
    assert torch.equal(only, full)


# -------------------------------------------------------------------- loss
@pytest.mark.parametrize("dt", [F32, BF])
@pytest.mark.parametrize("rows,V", [(40_000, 40), (40_000, 1000), (40_000, 1025), (30_000, 2100), (20_000, 4099),
                                    (16_000, 8192), (9000, 20_000), (6000, 32_003), (5000, 50_257), (3600, 60_000),
                                    (3000, 100_001), (1500, 131_072), (700, 260_000)])
def test_cross_entropy(dt, rows, V):
    g = gen(rows + V)
    B, T = 10, rows // 10
    ln = ragged(g, B, T)
    x = torch.randn((B, T, V), generator=g, device=DEV).mul_(3).to(dt)
    tgt = torch.randint(0, V, (B, T), generator=g, device=DEV)
    w = torch.rand((B, T), generator=g, device=DEV) + 0.1
    pick = torch.randint(0, 16, (B, T), generator=g, device=DEV)
    tgt[pick == 0] = -100
    w[pick == 1] = 0
    low = torch.finfo(dt).min
    half = torch.arange(V, device=DEV) >= V // 2
    x.masked_fill_((pick == 2)[..., None] & half, -float("inf"))
    x.masked_fill_((pick == 3)[..., None] & half, low)
    tgt = torch.where((pick == 2) | (pick == 3), tgt % (V // 2), tgt)
    x.masked_fill_((pick == 4)[..., None], low)                         # one value everywhere
    x.masked_fill_((pick == 5)[..., None], -float("inf"))               # nothing is left
    counted = kept(B, T, ln) & (tgt != -100) & (w != 0)
    x[~counted & (pick < 8)] = float("nan")
    got = E.cross_entropy(x, tgt, weights=w, lengths=ln)
    alone = E.cross_entropy(x, tgt, weights=w, lengths=ln, want_grad=False)
    empty = counted & (pick == 5)
    assert torch.isnan(got[0][empty]).all() and torch.isnan(got[1][empty]).all() and torch.isnan(alone[0][empty]).all()
    c = (V / 32 + 156) * U
    for b in range(B):
        n = int(counted[b].sum()) and int(counted[b].nonzero().max()) + 1
        assert not any(o[b, n:].any() for o in got) and not alone[0][b, n:].any() and not alone[1][b, n:].any()
        for t0 in range(0, n, 500):
            at = slice(t0, min(n, t0 + 500))
            yes = counted[b, at] & ~empty[b, at]
            X = torch.where(yes[:, None], x[b, at].double(), 0.0)
            t = torch.where(yes, tgt[b, at], 0)
            ww = torch.where(yes, w[b, at].double(), 0.0)
            m = X.amax(-1, keepdim=True)
            e = (X - m).exp()
            s = e.sum(-1, keepdim=True)
            ls, dt_ = s.log()[:, 0], m[:, 0] - X.gather(-1, t[:, None])[:, 0]
            loss, lse = ww * (dt_ + ls), (m[:, 0] + ls) * yes
            hot = torch.zeros_like(X).scatter_(-1, t[:, None], 1.0)
            p = e / s
            grad = ww[:, None] * (p - hot)
            left = ~empty[b, at]
            for o in (got, alone):
                check(o[0][b, at][left], loss[left], (ww * (c + 4 * U * (dt_.abs() + ls.abs())))[left], "loss")
                check(o[1][b, at][left], lse[left], ((c + 4 * U * (m[:, 0].abs() + ls.abs())) * yes)[left], "lse")
            tol = ww[:, None] * (c * p + 4 * U * hot) + 1e-37 + (VB if dt == BF else U) * grad.abs()
            check(got[2][b, at][left], grad[left], tol[left], "dlogits")
            assert torch.isnan(got[2][b, at][~left]).all()
