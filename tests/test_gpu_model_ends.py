"""GPU checks of the model-end operators (token embedding, normalisation, token
loss, each with its gradient) against float64 NumPy restatements of their formulas.

Tolerances come from rounding analysis, with u = 2^-24 (fp32) and v = 2^-8 (bf16),
the unit roundoffs:
* a result is rounded once to its type: v |want| for bf16, a few u for fp32;
* a sum of n fp32 terms in any order is off by at most (n - 1) u times the sum of
  the magnitudes; the sums over channels or classes are split over at least 32
  threads and joined in a tree, so a chain is at most n / 32 + 16 terms long;
* exp(x - max) is off by 2 u from the function, and by u |x - max| each from the
  difference and from its scaling; terms below e^-30 of the sum do not count, so
  128 u covers a term;
* first-order propagation of the statistics' errors to what is formed from them.
"""
import numpy as np
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

from paper_2609_37842_gb300 import eogp as E  # noqa: E402

DEV = "cuda:0"
U, VB = 2.0 ** -24, 2.0 ** -8
BF, F32 = torch.bfloat16, torch.float32
TYPES = [F32, BF]


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


def chain(n):
    return n / 32 + 16


def out_u(dt):
    return VB if dt == BF else U


def rnd(rng, shape, dt, scale=1.0):
    return torch.from_numpy((rng.standard_normal(shape) * scale).astype(np.float32)).to(DEV).to(dt)


def f64(t):
    return t.detach().double().cpu().numpy()


def keep_of(B, T, lengths):
    return np.arange(T)[None] < (np.full(B, T) if lengths is None else np.asarray(lengths))[:, None]


def ilen(lengths):
    return None if lengths is None else torch.tensor(lengths, dtype=torch.int32, device=DEV)


def check(got, want, tol, what):
    got = f64(got) if isinstance(got, torch.Tensor) else got
    assert got.shape == want.shape
    fine = np.isfinite(want)
    assert np.array_equal(fine, np.isfinite(got)), f"{what}: finite in other places"
    d = np.abs(np.where(fine, got, 0) - np.where(fine, want, 0))
    tol = np.broadcast_to(np.where(np.isfinite(tol), tol, 0), d.shape)
    worst = np.max(d / np.maximum(tol, 1e-300), initial=0.0)
    print(f"{what}: worst error / tolerance {worst:.3g}")
    assert np.all(d <= tol), f"{what}: {worst:.3g} of the tolerance"


def strided(t, how, fill=float("nan")):
    """The values of t [B, T, n] in memory laid out another way."""
    B, T, n = t.shape
    if how == "dense":
        return t.clone()
    if how == "offset":      # base one element past a 16-byte boundary
        flat = torch.full((B * T * n + 1,), fill, dtype=t.dtype, device=t.device)
        v = flat[1:].view(B, T, n)
    elif how == "wide":      # rows inside wider rows, 8 elements in
        v = torch.full((B, T, n + 24), fill, dtype=t.dtype, device=t.device)[:, :, 8:8 + n]
    elif how == "odd":       # row stride of another alignment
        v = torch.full((B, T, n + 3), fill, dtype=t.dtype, device=t.device)[:, :, :n]
    elif how == "cut":       # the first T of T + 2 tokens of each example
        v = torch.full((B, T + 2, n), fill, dtype=t.dtype, device=t.device)[:, :T]
    elif how == "tokens first":
        v = torch.full((T, B, n), fill, dtype=t.dtype, device=t.device).transpose(0, 1)
    v.copy_(t)
    return v


LAYOUTS = ["dense", "offset", "wide", "odd", "cut", "tokens first"]


# --------------------------------------------------------------- embedding
def zipf(rng, V, shape):
    return np.clip(np.exp(rng.uniform(0, np.log(V + 1), shape)).astype(np.int64) - 1, 0, V - 1)


def embed_ref(tok, table, scale, pos, keep):
    out = table[np.where(keep, tok, 0)] * scale
    mag = np.abs(out)
    if pos is not None:
        out = out + pos[None, :tok.shape[1]]
        mag = mag + np.abs(pos[None, :tok.shape[1]])
    return out * keep[..., None], mag


@pytest.mark.parametrize("dt", TYPES)
@pytest.mark.parametrize("B,T,V,d,lengths,pos", [
    (1, 1, 5, 1, None, False), (1, 1, 1000, 768, None, True), (3, 7, 50, 770, [7, 0, 3], True),
    (2, 65, 1000, 129, [64, 1], False), (4, 33, 700, 4096, None, True), (5, 1, 9, 8, [1, 0, 1, 1, 0], False),
    (2, 3, 4, 20008, [2, 3], True), (300, 2, 12, 64, None, False)])
def test_embed(dt, B, T, V, d, lengths, pos):
    rng = np.random.default_rng(B * 100 + T + d)
    tok = zipf(rng, V, (B, T))
    keep = keep_of(B, T, lengths)
    table, p = rnd(rng, (V, d), dt), rnd(rng, (T + 2, d), dt) if pos else None
    scale = 1.7
    want, mag = embed_ref(tok, f64(table), np.float64(np.float32(scale)), None if p is None else f64(p), keep)
    for idt in (torch.int32, torch.int64):
        tk = torch.from_numpy(np.where(keep, tok, -7)).to(DEV).to(idt)   # padding may hold any number
        got = E.embed(tk, table, scale=scale, pos=p, lengths=ilen(lengths))
        check(got, want, out_u(dt) * np.abs(want) + 3 * U * mag, "out")
    if B == 1:
        assert torch.equal(E.embed(tk[0], table, scale=scale, pos=p), got[0])


@pytest.mark.parametrize("dt", TYPES)
@pytest.mark.parametrize("how", LAYOUTS[1:])
@pytest.mark.parametrize("d", [64, 77])
def test_embed_layouts(dt, how, d):
    rng = np.random.default_rng(d)
    B, T, V = 3, 9, 40
    tok = torch.from_numpy(zipf(rng, V, (B, T + 4))).to(DEV)[:, 2:2 + T]       # strided token rows
    table = strided(rnd(rng, (1, V, d), dt), "odd" if how == "odd" else "dense")[0]
    pos = rnd(rng, (T, d), dt)
    ln = ilen([9, 4, 0])
    want = E.embed(tok.contiguous(), table.contiguous(), pos=pos, lengths=ln)
    out = strided(torch.zeros((B, T, d), dtype=dt, device=DEV), how)
    E.embed(tok, table, pos=pos, lengths=ln, out=out)
    assert torch.equal(out, want)


def test_embed_single_token_at_a_position():
    """Serving: the token at position p alone equals row p of the whole sequence."""
    rng = np.random.default_rng(5)
    table, pos = rnd(rng, (100, 256), BF), rnd(rng, (32, 256), BF)
    tok = torch.from_numpy(zipf(rng, 100, (2, 32))).to(DEV)
    whole = E.embed(tok, table, scale=3.0, pos=pos)
    for p in (0, 13, 31):
        assert torch.equal(E.embed(tok[:, p:p + 1], table, scale=3.0, pos=pos[p:]), whole[:, p:p + 1])


def test_embed_token_out_of_range():
    table = torch.ones((4, 16), device=DEV)
    tok = torch.tensor([[0, 4, 3, -1]], device=DEV)
    out = E.embed(tok, table)
    with pytest.raises(E.EOGPError) as ei:
        E.sync_status()
    assert ei.value.code == E.EDEVICE
    assert out[0, :, 0].tolist() == [1.0, 0.0, 1.0, 0.0]
    g = E.embed_grad(tok, torch.ones((1, 4, 16), device=DEV), 4)
    with pytest.raises(E.EOGPError) as ei:
        E.sync_status()
    assert ei.value.code == E.EDEVICE
    assert g[:, 0].tolist() == [1.0, 0.0, 0.0, 1.0]


def embed_grad_ref(tok, dout, V, scale, keep):
    d = dout.shape[-1]
    g, mag, n = np.zeros((V, d)), np.zeros((V, d)), np.zeros((V, 1))
    rows = np.where(keep[..., None], dout, 0.0)
    for b, t in zip(*np.nonzero(keep)):
        g[tok[b, t]] += rows[b, t]
        mag[tok[b, t]] += np.abs(rows[b, t])
        n[tok[b, t]] += 1
    return g * scale, mag * abs(scale), n


@pytest.mark.parametrize("dt,gt", [(F32, F32), (BF, F32), (BF, BF), (F32, BF)])
@pytest.mark.parametrize("B,T,V,d,lengths,tokens", [
    (1, 1, 1, 1, None, "zipf"), (1, 1, 300, 768, None, "zipf"), (1, 509, 301, 77, None, "zipf"),
    (3, 200, 1000, 130, [200, 0, 77], "zipf"), (4, 1025, 5000, 64, None, "zipf"), (2, 900, 1, 40, None, "zipf"),
    (2, 700, 70_000, 16, [1, 700], "zipf"), (3, 64, 50, 8, [0, 0, 0], "zipf"), (1, 3000, 20, 264, None, "same"),
    (1, 2049, 600_000, 9, None, "spread"), (700, 5, 513, 32, None, "zipf"), (2, 40, 64, 5001, [39, 40], "zipf")])
def test_embed_grad(dt, gt, B, T, V, d, lengths, tokens):
    rng = np.random.default_rng(B * 7 + T + V + d)
    tok = zipf(rng, V, (B, T)) if tokens == "zipf" else rng.integers(0, V, (B, T))
    if tokens == "same":
        tok[:, 5:-3] = 7
    keep = keep_of(B, T, lengths)
    dout = rnd(rng, (B, T, d), dt)
    dout[torch.from_numpy(~keep).to(DEV)] = float("nan")
    scale = np.float64(np.float32(0.3))
    want, mag, n = embed_grad_ref(tok, np.nan_to_num(f64(dout)), V, scale, keep)
    tol = out_u(gt) * np.abs(want) + (n + 2) * U * mag
    ref = None
    for idt in (torch.int32, torch.int64):
        tk = torch.from_numpy(np.where(keep, tok, V + 3)).to(DEV).to(idt)
        got = E.embed_grad(tk, dout, V, scale=0.3, lengths=ilen(lengths), dtype=gt)
        check(got, want, tol, "dtable")
        assert ref is None or torch.equal(ref, got)   # bitwise reproducible
        ref = got
    # accumulated into a table: rows of absent tokens keep their bits
    base = rnd(rng, (V, d), gt)
    acc = base.clone()
    E.embed_grad(tk, dout, V, scale=0.3, lengths=ilen(lengths), dtable=acc, accumulate=True)
    check(acc, f64(base) + want, out_u(gt) * np.abs(f64(base) + want) + (n + 3) * U * (mag + np.abs(f64(base))),
          "accumulated")
    absent = torch.from_numpy(n[:, 0] == 0).to(DEV)
    assert torch.equal(acc[absent], base[absent])


@pytest.mark.parametrize("how", LAYOUTS[1:])
@pytest.mark.parametrize("d", [64, 77])
@pytest.mark.parametrize("dt", TYPES)
def test_embed_grad_layouts(dt, how, d):
    rng = np.random.default_rng(3 * d)
    B, T, V = 3, 50, 37
    tok = torch.from_numpy(zipf(rng, V, (B, T + 5))).to(DEV)[:, 5:]
    dout = rnd(rng, (B, T, d), dt)
    ln = ilen([50, 20, 0])
    want = E.embed_grad(tok.contiguous(), dout, V, lengths=ln)
    wide = strided(torch.full((1, V, d), 5.0, device=DEV), "odd" if how == "odd" else "wide")[0]
    got = E.embed_grad(tok, strided(dout, how), V, lengths=ln, dtable=wide)
    assert got is wide and torch.equal(got, want)


def test_embed_grad_broadcast_rows_and_empty_batch():
    """A gradient row shared by every position (stride 0), and a batch without tokens."""
    rng = np.random.default_rng(11)
    tok = torch.from_numpy(zipf(rng, 20, (4, 30))).to(DEV)
    row = rnd(rng, (1, 1, 96), F32)
    got = E.embed_grad(tok, row.expand(4, 30, 96), 20)
    count = torch.bincount(tok.reshape(-1), minlength=20).double()[:, None]
    check(got, f64(count.cpu()) * f64(row[0]), 130 * U * f64(count.cpu()) * np.abs(f64(row[0])), "dtable")
    got = E.embed_grad(tok[:0], row.expand(4, 30, 96)[:0], 20)
    assert got.shape == (20, 96) and not got.any()
    keep = torch.ones((20, 96), device=DEV)
    E.embed_grad(tok[:, :0], row.expand(4, 30, 96)[:, :0], 20, dtable=keep, accumulate=True)
    assert torch.all(keep == 1.0)


def test_position_gradient():
    """The position table's gradient: the numbers 0..T-1 as tokens."""
    rng = np.random.default_rng(12)
    B, T, d = 5, 37, 72
    dout = rnd(rng, (B, T, d), BF)
    ids = torch.arange(T, device=DEV).expand(B, T)
    got = E.embed_grad(ids, dout, T + 3)
    want = np.concatenate([f64(dout).sum(0), np.zeros((3, d))])
    mag = np.concatenate([np.abs(f64(dout)).sum(0), np.zeros((3, d))])
    check(got, want, (B + 2) * U * mag, "dpos")


# ----------------------------------------------------------- normalisation
def norm_ref(x, w, b, rms, eps, keep):
    d = x.shape[-1]
    x = np.where(keep[..., None], x, 0.0)
    mu = np.zeros(x.shape[:-1]) if rms else x.mean(-1)
    xc = x - mu[..., None]
    r = 1.0 / np.sqrt((xc * xc).mean(-1) + eps)
    xh = xc * r[..., None]
    y = xh * w + b
    # error of xh: mean off by c u mean|x|, rstd by c u relative (c: chain of the sums)
    c = chain(d) + 8
    exh = c * U * (np.abs(xh) + r[..., None] * (np.abs(x).mean(-1, keepdims=True) + np.abs(x)))
    k = keep[..., None]
    return y * k, mu * keep, r * keep, (exh * np.abs(w) + 4 * U * (np.abs(xh * w) + np.abs(b))) * k, c, np.abs(x)


NORM_SIZES = [(1, 1, 1, None), (1, 1, 4096, None), (1, 1, 8, None), (2, 3, 33, [3, 1]), (3, 5, 768, [5, 0, 2]),
              (2, 7, 770, None), (1, 9, 1024, None), (4, 3, 2048, [3, 3, 1, 0]), (2, 2, 5120, None), (1, 3, 8192, None),
              (1, 2, 16_384, None), (2, 2, 16_390, [1, 2]), (1, 2, 50_001, None), (130, 3, 64, None), (1, 300, 96, None)]


@pytest.mark.parametrize("kind", [E.NORM_LAYER, E.NORM_RMS])
@pytest.mark.parametrize("dt,pt", [(F32, F32), (BF, BF), (BF, F32), (F32, BF)])
@pytest.mark.parametrize("B,T,d,lengths", NORM_SIZES)
def test_norm(kind, dt, pt, B, T, d, lengths):
    rng = np.random.default_rng(d + B + T)
    keep = keep_of(B, T, lengths)
    x = rnd(rng, (B, T, d), dt) + 0.5
    x[torch.from_numpy(~keep).to(DEV)] = float("nan")
    w, b = rnd(rng, (d,), pt) + 1, rnd(rng, (d,), pt)
    eps = np.float64(np.float32(1e-5))
    for ww, bb in ((w, b), (w, None), (None, b), (None, None)):
        y, mean, rstd = E.norm(x, ww, bb, kind=kind, eps=1e-5, lengths=ilen(lengths))
        W = np.ones(d) if ww is None else f64(ww)
        Bv = np.zeros(d) if bb is None else f64(bb)
        want, mu, r, tol, c, ax = norm_ref(f64(x), W, Bv, kind == E.NORM_RMS, eps, keep)
        # where the variance is below eps, x - mean is what remains of the mean's rounding
        check(y, want, out_u(dt) * np.abs(want) + tol, "y")
        check(rstd, r, c * U * r * 3, "rstd")
        if kind == E.NORM_LAYER:
            check(mean, mu, c * U * ax.mean(-1), "mean")
        else:
            assert mean is None


@pytest.mark.parametrize("kind", [E.NORM_LAYER, E.NORM_RMS])
def test_norm_hard_rows(kind):
    """Constant rows (variance 0), a large offset, tiny and large values, zeros."""
    d = 1536
    rng = np.random.default_rng(2)
    rows = [np.full(d, 3.0), np.zeros(d), 1000.0 + rng.standard_normal(d), 1e-12 * rng.standard_normal(d),
            1e15 * rng.standard_normal(d)]
    x = torch.tensor(np.stack(rows)[None], dtype=F32, device=DEV)
    y, mean, rstd = E.norm(x, kind=kind, eps=1e-5)
    keep = keep_of(1, len(rows), None)
    want, mu, r, tol, c, ax = norm_ref(f64(x), np.ones(d), np.zeros(d), kind == E.NORM_RMS,
                                       np.float64(np.float32(1e-5)), keep)
    check(y, want, tol + U * np.abs(want), "y")
    check(rstd, r, 3 * c * U * r, "rstd")


@pytest.mark.parametrize("how", LAYOUTS[1:])
@pytest.mark.parametrize("d", [64, 77, 2048])
@pytest.mark.parametrize("dt", TYPES)
def test_norm_layouts(dt, how, d):
    """Any layout of inputs and outputs gives the dense layout's values to rounding; in place gives its own bits."""
    rng = np.random.default_rng(d)
    B, T = 3, 6
    x, dy = rnd(rng, (B, T, d), dt), rnd(rng, (B, T, d), dt)
    w, b = rnd(rng, (d + 1,), dt)[1:], rnd(rng, (d + 1,), dt)[1:]     # params off a 16-byte boundary too
    ln = ilen([6, 0, 5])
    y0, mean0, rstd0 = E.norm(x, w, b, lengths=ln)
    g0 = E.norm_grad(dy, x, mean0, rstd0, w, lengths=ln, per_example=True)
    xs, ys = strided(x, how), strided(torch.zeros_like(x), how)
    y, mean, rstd = E.norm(xs, w, b, lengths=ln, out=ys)
    near = dict(rtol=4 * out_u(dt), atol=1e-5)
    torch.testing.assert_close(y, y0, **near)
    torch.testing.assert_close(rstd, rstd0, rtol=1e-5, atol=0)
    dx = strided(torch.zeros_like(x), how)
    wide = torch.full((2, B, d + 5), 9.0, device=DEV)
    E.norm_grad(strided(dy, how), xs, mean0, rstd0, w, lengths=ln, per_example=True, dx=dx,
                dweight=wide[0][:, :d], dbias=wide[1][:, :d])
    torch.testing.assert_close(dx, g0[0], **near)
    torch.testing.assert_close(wide[0][:, :d], g0[1], rtol=1e-5, atol=1e-5)
    torch.testing.assert_close(wide[1][:, :d], g0[2], rtol=1e-5, atol=1e-5)
    assert torch.all(wide[:, :, d:] == 9.0)
    E.norm(xs, w, b, lengths=ln, out=xs)                    # y over x
    assert torch.equal(xs, y)


def norm_grad_ref(dy, x, mu, r, w, rms, keep, per_example):
    k = keep[..., None]
    dy, x = np.where(k, dy, 0.0), np.where(k, x, 0.0)
    mu = np.zeros_like(r) if rms else mu
    xh = (x - mu[..., None]) * r[..., None] * k
    g = dy * w
    m1 = np.zeros_like(r)[..., None] if rms else g.mean(-1, keepdims=True)
    m2 = (g * xh).mean(-1, keepdims=True)
    dx = (g - m1 - xh * m2) * r[..., None] * k
    d = x.shape[-1]
    # xh is off by 2 u (|x| + |mean|) rstd; the means by the chain of their sums
    exh = 2 * U * (np.abs(x) + np.abs(mu)[..., None]) * r[..., None]
    a2 = (np.abs(g) * (np.abs(xh) + exh / U)).mean(-1, keepdims=True)
    edx = r[..., None] * ((chain(d) + 8) * U * (np.abs(g) + np.abs(g).mean(-1, keepdims=True) + np.abs(xh) * a2)
                          + exh * np.abs(m2))
    over = (1,) if per_example else (0, 1)
    n = np.maximum(keep.sum(over), 1).reshape(-1, 1) if per_example else max(1, keep.sum())
    edw = (np.abs(dy) * exh).sum(over) + (n + 4) * U * np.abs(dy * xh).sum(over)
    edb = (n + 4) * U * np.abs(dy).sum(over)
    return dx, (dy * xh).sum(over), dy.sum(over), edx * k, edw, edb


@pytest.mark.parametrize("kind", [E.NORM_LAYER, E.NORM_RMS])
@pytest.mark.parametrize("dt,pt", [(F32, F32), (BF, BF), (BF, F32)])
@pytest.mark.parametrize("per_example", [False, True])
@pytest.mark.parametrize("B,T,d,lengths", NORM_SIZES + [(2, 400, 72, [400, 399]), (1, 1500, 130, None),
                                                       (3, 4, 40, [0, 0, 0])])
def test_norm_grad(kind, dt, pt, per_example, B, T, d, lengths):
    rng = np.random.default_rng(d * 3 + B + T)
    keep = keep_of(B, T, lengths)
    x, dy = rnd(rng, (B, T, d), dt) + 0.5, rnd(rng, (B, T, d), dt)
    pad = torch.from_numpy(~keep).to(DEV)
    x[pad], dy[pad] = float("nan"), float("inf")
    w = rnd(rng, (d,), pt) + 1
    xz = np.where(keep[..., None], f64(x), 1.0)
    rms = kind == E.NORM_RMS
    mu = np.zeros((B, T)) if rms else xz.mean(-1)
    r = 1.0 / np.sqrt(((xz - mu[..., None]) ** 2).mean(-1) + 1e-5)
    mean = None if rms else torch.from_numpy(mu.astype(np.float32)).to(DEV)
    rstd = torch.from_numpy(r.astype(np.float32)).to(DEV)
    mu, r = (mu if rms else f64(mean)), f64(rstd)
    for ww in (w, None):
        W = np.ones(d) if ww is None else f64(ww)
        dx_w, dw_w, db_w, edx, edw, edb = norm_grad_ref(np.nan_to_num(f64(dy), posinf=0), np.nan_to_num(f64(x)), mu, r,
                                                       W, rms, keep, per_example)
        args = dict(kind=kind, lengths=ilen(lengths), per_example=per_example)
        dx, dw, db = E.norm_grad(dy, x, mean, rstd, ww, **args)
        check(dx, dx_w, out_u(dt) * np.abs(dx_w) + edx, "dx")
        check(dw, dw_w, edw, "dweight")
        check(db, db_w, edb, "dbias")
        # reproducible, and the same when only some results are wanted
        again = E.norm_grad(dy, x, mean, rstd, ww, **args)
        assert all(torch.equal(p, q) for p, q in zip((dx, dw, db), again))
        only = E.norm_grad(dy, x, mean, rstd, ww, want_dweight=False, want_dbias=False, **args)
        assert torch.equal(only[0], dx) and only[1] is None and only[2] is None
        only = E.norm_grad(dy, x, mean, rstd, ww, want_dx=False, want_dbias=False, **args)
        torch.testing.assert_close(only[1], dw, rtol=1e-4, atol=1e-3)
        assert only[0] is None and only[2] is None
    # accumulation, and dx over dy
    dw2, db2 = dw.clone(), db.clone()
    E.norm_grad(dy, x, mean, rstd, None, want_dx=False, dweight=dw2, dbias=db2, accumulate=True, **args)
    check(dw2, 2 * dw_w, 2 * edw + 2 * U * np.abs(dw_w), "dweight twice")
    check(db2, 2 * db_w, 2 * edb + 2 * U * np.abs(db_w), "dbias twice")
    over = dy.clone()
    got = E.norm_grad(over, x, mean, rstd, None, dx=over, **args)
    assert torch.equal(over, dx) and torch.equal(got[1], dw)


@pytest.mark.parametrize("kind", [E.NORM_LAYER, E.NORM_RMS])
def test_norm_gradient_against_differences(kind):
    """Directional differences of the forward pass, f(p) = <c, norm(p)>, in fp32 inputs and float64 sums.
    Central differences of step h are off by h^2 f''' / 6, about 1e-4 of the slope here at h = 1e-2, and by the
    outputs' rounding, 3 u |f's terms| / h, about 2e-4 of it."""
    rng = np.random.default_rng(8)
    B, T, d, h = 2, 5, 256, 1e-2
    x, w, b, c = (rng.standard_normal(s).astype(np.float32) for s in ((B, T, d), (d,), (d,), (B, T, d)))

    def f(xv, wv, bv):
        y, _, _ = E.norm(*(torch.from_numpy(v.astype(np.float32)).to(DEV) for v in (xv, wv, bv)), kind=kind)
        return float((f64(y) * c).sum())

    td = [torch.from_numpy(v).to(DEV) for v in (x, w, b, c)]
    _, mean, rstd = E.norm(td[0], td[1], td[2], kind=kind)
    dx, dw, db = E.norm_grad(td[3], td[0], mean, rstd, td[1], kind=kind)
    for i, g in enumerate((dx, dw, db)):
        u = rng.standard_normal(g.shape)
        u = u / np.linalg.norm(u) * 3
        at = [x.astype(np.float64), w.astype(np.float64), b.astype(np.float64)]
        up, dn = list(at), list(at)
        up[i], dn[i] = at[i] + h * u, at[i] - h * u
        got, want = float((f64(g) * u).sum()), (f(*up) - f(*dn)) / (2 * h)
        scale = np.linalg.norm(f64(g)) * 3 / np.sqrt(g.numel()) + abs(want)
        assert abs(got - want) <= 5e-3 * scale + 5e-3, (i, got, want)


# -------------------------------------------------------------------- loss
def loss_ref(x, tgt, w, counted):
    """loss, lse, gradient and their tolerances without the output type's rounding."""
    V = x.shape[-1]
    with np.errstate(all="ignore"):
        xz = np.where(counted[..., None], x, 0.0)
        m = xz.max(-1, keepdims=True)
        e = np.exp(xz - m)
        s = e.sum(-1, keepdims=True)
        p = e / s
        ls = np.log(s)[..., 0]
        xt = np.take_along_axis(xz, np.where(counted, tgt, 0)[..., None], -1)[..., 0]
        k = (chain(V) + 140) * U
        loss = w * ((m[..., 0] - xt) + ls)
        eloss = np.abs(w) * (k + 4 * U * (np.abs(m[..., 0] - xt) + np.abs(ls)))
        lse = m[..., 0] + ls
        elses = k + 4 * U * (np.abs(m[..., 0]) + np.abs(ls))
        onehot = np.zeros_like(p)
        np.put_along_axis(onehot, np.where(counted, tgt, 0)[..., None], 1.0, -1)
        g = w[..., None] * (p - onehot)
        eg = np.abs(w[..., None]) * (k * p + 4 * U * onehot) + 1e-37
    z = lambda a: np.where(counted if a.ndim == 2 else counted[..., None], a, 0.0)  # noqa: E731
    return [z(a) for a in (loss, lse, g, eloss, elses, eg)]


LOSS_SIZES = [(1, 1, 1, None), (1, 1, 7, None), (1, 1, 50_001, None), (2, 5, 1000, [5, 2]), (3, 4, 4099, [0, 4, 1]),
              (1, 37, 32_000, None), (2, 3, 50_001, [3, 1]), (1, 2, 131_073, None), (1, 2, 300_001, None),
              (1, 1, 1_000_003, None), (40, 9, 515, None), (1, 700, 129, None), (2, 170, 8192, [170, 100])]


@pytest.mark.parametrize("dt", TYPES)
@pytest.mark.parametrize("B,T,V,lengths", LOSS_SIZES)
def test_cross_entropy(dt, B, T, V, lengths):
    rng = np.random.default_rng(V + B + T)
    keep = keep_of(B, T, lengths)
    x = rnd(rng, (B, T, V), dt, 3.0)
    tgt = rng.integers(0, V, (B, T))
    tgt[rng.random((B, T)) < 0.2] = -100
    if B * T == 1:
        tgt[:] = V - 1
    w = rng.uniform(0.1, 2.0, (B, T)).astype(np.float32)
    w[rng.random((B, T)) < 0.1] = 0.0
    if B * T == 1:
        w[:] = 1.5
    for weights, idt in ((w, torch.int64), (None, torch.int32)):
        wv = np.ones((B, T)) if weights is None else w.astype(np.float64)
        counted = keep & (tgt != -100) & (wv != 0)
        xx = x.clone()
        xx[torch.from_numpy(~counted).to(DEV)] = float("nan")      # left-out rows may hold anything
        loss_w, lse_w, g_w, el, es, eg = loss_ref(np.nan_to_num(f64(xx)), tgt, wv, counted)
        args = dict(weights=None if weights is None else torch.from_numpy(w).to(DEV), lengths=ilen(lengths))
        tk = torch.from_numpy(tgt).to(DEV).to(idt)
        loss, lse, g = E.cross_entropy(xx, tk, **args)
        check(loss, loss_w, el, "loss")
        check(lse, lse_w, es, "lse")
        check(g, g_w, out_u(dt) * np.abs(g_w) + eg, "dlogits")
        alone = E.cross_entropy(xx, tk, want_grad=False, **args)
        assert alone[2] is None
        check(alone[0], loss_w, el, "loss alone")
        again = E.cross_entropy(xx, tk, **args)
        assert all(torch.equal(p, q) for p, q in zip((loss, lse, g), again))
        E.cross_entropy(xx, tk, dlogits=xx, **args)                # the gradient over its logits
        assert torch.equal(xx, g)


@pytest.mark.parametrize("dt", TYPES)
@pytest.mark.parametrize("V", [64, 1003, 50_001, 140_000])
def test_cross_entropy_masks_and_extremes(dt, V):
    """Vocabulary masks of -inf and of the type's lowest value, single survivors, equal logits, huge logits, a
    masked target, rows that nothing is left of, and NaN / +inf in a row."""
    low = torch.finfo(dt).min
    big = torch.finfo(dt).max
    rng = np.random.default_rng(V)
    x = rng.standard_normal((1, 12, V)).astype(np.float32) * 2
    tgt = np.full((1, 12), 3)
    x[0, 0, V // 2:] = -np.inf
    x[0, 1, V // 2:] = low
    x[0, 2, :] = -np.inf
    x[0, 2, 3] = 0.25                      # the target alone is left: loss 0, gradient 0
    x[0, 3, :] = low                       # all at the lowest value: uniform
    x[0, 4, :] = big                       # all at the largest value: uniform
    x[0, 5, 3] = -np.inf                   # the target is masked: loss inf, finite gradient
    x[0, 6, :] = -np.inf                   # nothing is left: NaN
    x[0, 7, V - 1] = np.nan
    x[0, 8, 0] = np.inf
    x[0, 9, :] = 5.0
    x[0, 10, :] = low
    x[0, 10, V - 1] = big                  # differences beyond fp32's range
    x[0, 11] = x[0, 11] * 30
    xt = torch.from_numpy(x).to(DEV).to(dt)
    loss, lse, g = E.cross_entropy(xt, torch.from_numpy(tgt).to(DEV))
    x64 = f64(xt)
    counted = np.ones((1, 12), bool)
    loss_w, lse_w, g_w, el, es, eg = loss_ref(x64, tgt, np.ones((1, 12)), counted)
    assert loss_w[0, 5] == np.inf and loss[0, 5] == np.inf
    with np.errstate(over="ignore"):       # a loss beyond fp32's range is inf
        loss_w = loss_w.astype(np.float32).astype(np.float64)
    fine = [0, 1, 2, 3, 4, 5, 9, 10, 11]
    check(loss[:, fine], loss_w[:, fine], el[:, fine], "loss")
    check(lse[:, fine], lse_w[:, fine], es[:, fine], "lse")
    check(g[:, fine], g_w[:, fine], out_u(dt) * np.abs(g_w[:, fine]) + eg[:, fine], "dlogits")
    assert loss[0, 2] == 0 and not g[0, 2].any()
    for bad in (6, 7, 8):
        assert torch.isnan(loss[0, bad]) and torch.isnan(g[0, bad]).all()
        assert torch.isnan(lse[0, bad])
    # the same rows left out: nothing of theirs shows
    w = torch.ones((1, 12), device=DEV)
    w[0, 6:9] = 0
    loss2, lse2, g2 = E.cross_entropy(xt, torch.from_numpy(tgt).to(DEV), weights=w)
    assert not loss2[0, 6:9].any() and not lse2[0, 6:9].any() and not g2[0, 6:9].any()
    assert torch.equal(g2[0, fine], g[0, fine])


@pytest.mark.parametrize("how", LAYOUTS[1:])
@pytest.mark.parametrize("V", [512, 1001, 70_001])
@pytest.mark.parametrize("dt", TYPES)
def test_cross_entropy_layouts(dt, how, V):
    rng = np.random.default_rng(V)
    B, T = 3, 5
    x = rnd(rng, (B, T, V), dt, 2.0)
    tok = torch.from_numpy(rng.integers(0, V, (B, T + 1))).to(DEV)
    tgt = tok[:, 1:]                       # next tokens: a strided view
    ln = ilen([5, 0, 3])
    want = E.cross_entropy(x, tgt.contiguous(), lengths=ln)
    for hx, hg in ((how, how), (how, "dense"), ("dense", how)):
        g = strided(torch.zeros_like(x), hg)
        got = E.cross_entropy(strided(x, hx), tgt, lengths=ln, dlogits=g)
        torch.testing.assert_close(got[0], want[0], rtol=1e-5, atol=1e-5)
        torch.testing.assert_close(got[2], want[2], rtol=4 * out_u(dt), atol=1e-6)
    xs = strided(x, how)
    E.cross_entropy(xs, tgt, lengths=ln, dlogits=xs)
    torch.testing.assert_close(xs, want[2], rtol=4 * out_u(dt), atol=1e-6)


def test_cross_entropy_target_out_of_range():
    x = torch.zeros((1, 4, 10), device=DEV)
    tgt = torch.tensor([[2, 10, -1, 9]], device=DEV)
    loss, lse, g = E.cross_entropy(x, tgt)
    with pytest.raises(E.EOGPError) as ei:
        E.sync_status()
    assert ei.value.code == E.EDEVICE
    assert not loss[0, 1:3].any() and not g[0, 1:3].any() and torch.all(loss[0, [0, 3]] > 2.3)


def test_cross_entropy_against_differences():
    """Directional differences of the summed loss. A step of 1e-2 is off by about h^2 / 6 of the third derivative
    (below 1e-4 here), the losses' fp32 rounding by 20 u T / h, about 2e-3 at most."""
    rng = np.random.default_rng(4)
    B, T, V, h = 2, 3, 1003, 1e-2
    x = rng.standard_normal((B, T, V)).astype(np.float32)
    tgt = torch.from_numpy(rng.integers(0, V, (B, T))).to(DEV)
    w = torch.rand((B, T), device=DEV) + 0.5

    def f(v):
        return float(f64(E.cross_entropy(torch.from_numpy(v.astype(np.float32)).to(DEV), tgt, weights=w,
                                         want_grad=False)[0]).sum())

    g = f64(E.cross_entropy(torch.from_numpy(x).to(DEV), tgt, weights=w)[2])
    for k in range(4):
        u = rng.standard_normal(x.shape) + (20 * g if k else 0)
        got, want = float((g * u).sum()), (f(x + h * u) - f(x - h * u)) / (2 * h)
        assert abs(got - want) <= 5e-3 * (1 + abs(want)), (got, want)


# ----------------------------------------------------------- all operators
def test_offsets_beyond_32_bits():
    """Rows whose offset passes 2^31 (and 2^32) elements, reached by an example stride rather than by their number."""
    if torch.cuda.mem_get_info()[0] < 40 << 30:
        pytest.skip("needs 40 GB of device memory")
    rng = np.random.default_rng(6)
    far = (1 << 32) + 64                    # elements between the two examples: 8 GiB of bf16
    d = 512
    buf = torch.empty(far + 4 * d, dtype=BF, device=DEV)
    view = buf.as_strided((2, 2, d), (far, d, 1))
    x = rnd(rng, (2, 2, d), BF)
    view.copy_(x)
    tgt = torch.tensor([[1, 2], [3, 4]], device=DEV)
    y, mean, rstd = E.norm(x)
    assert torch.equal(E.norm(view)[0], y)
    want = E.norm_grad(x, x, mean, rstd, per_example=True)
    got = E.norm_grad(view, view, mean, rstd, per_example=True)
    assert all(torch.equal(p, q) for p, q in zip(got, want))
    assert torch.equal(E.cross_entropy(view, tgt)[2], E.cross_entropy(x, tgt)[2])
    assert torch.equal(E.embed_grad(tgt, view, 5), E.embed_grad(tgt, x, 5))
    table = buf.as_strided((2, d), (far, 1))
    assert torch.equal(E.embed(torch.tensor([1, 0], device=DEV), table), x[[1, 0], 0])
    E.norm(x, out=view)
    assert torch.equal(view, y)


def test_large_logits_matrix():
    """More than 2^31 logits in one call, checked on its last rows."""
    if torch.cuda.mem_get_info()[0] < 40 << 30:
        pytest.skip("needs 40 GB of device memory")
    T, V = 21_500, 100_003
    g = torch.Generator(device=DEV)
    g.manual_seed(3)
    x = torch.empty((1, T, V), dtype=BF, device=DEV).normal_(generator=g)
    tgt = torch.randint(0, V, (1, T), generator=g, device=DEV)
    last = E.cross_entropy(x[:, -3:].clone(), tgt[:, -3:].clone())
    loss, lse, grad = E.cross_entropy(x, tgt, dlogits=x)
    torch.testing.assert_close(loss[:, -3:], last[0], rtol=1e-5, atol=1e-5)
    torch.testing.assert_close(grad[:, -3:], last[2], rtol=4 * VB, atol=1e-6)


def test_other_stream():
    """Calls on a stream that is not current work there, in order, with memory of that stream."""
    rng = np.random.default_rng(9)
    x, w = rnd(rng, (4, 600, 1024), BF), rnd(rng, (1024,), BF)
    tok = torch.from_numpy(zipf(rng, 500, (4, 600))).to(DEV)
    table = rnd(rng, (500, 1024), BF)
    logits, tgt = rnd(rng, (4, 20, 5000), BF), torch.randint(0, 5000, (4, 20), device=DEV)

    def all_of(stream):
        y, mean, rstd = E.norm(x, w, stream=stream)
        outs = [y, *E.norm_grad(y, x, mean, rstd, w, stream=stream), E.embed(tok, table, stream=stream),
                E.embed_grad(tok, x, 500, stream=stream), *E.cross_entropy(logits, tgt, stream=stream)]
        return outs

    want = all_of(None)
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    for _ in range(3):
        got = all_of(s)
        junk = [torch.full_like(t, 7) for t in got]     # the current stream goes on allocating and writing
        s.synchronize()
        assert all(torch.equal(p, q) for p, q in zip(got, want))
        del junk
    by_number = E.embed(tok, table, stream=s.cuda_stream)
    s.synchronize()
    assert torch.equal(by_number, want[4])


def test_captured_in_a_graph():
    """The calls allocate nothing of their own and can be captured, then replayed on new inputs."""
    rng = np.random.default_rng(10)
    B, T, d, V = 2, 65, 256, 300
    tok = torch.from_numpy(zipf(rng, V, (B, T))).to(DEV)
    table, w = rnd(rng, (V, d), BF), rnd(rng, (d,), BF)

    def step():
        x = E.embed(tok, table)
        y, mean, rstd = E.norm(x, w, kind=E.NORM_RMS)
        loss, _, dl = E.cross_entropy(y, tok % d)
        dx, dw, _ = E.norm_grad(dl, x, mean, rstd, w, kind=E.NORM_RMS, want_dbias=False)
        return loss, dw, E.embed_grad(tok, dx, V)

    step()
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        got = step()
    tok.copy_(torch.from_numpy(zipf(rng, V, (B, T))).to(DEV))
    g.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(p, q) for p, q in zip(got, step()))
