"""GPU checks of the model-end operators where values, sizes or aliasing are at their
edges, against float64 restatements of the formulas (tolerances: test_gpu_model_ends)."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

from paper_2609_37842_gb300 import eogp as E  # noqa: E402
from test_gpu_model_ends import (BF, DEV, F32, TYPES, U, _lib, _status, chain, check, f64, loss_ref,  # noqa: E402,F401
                                 out_u, rnd)


# -------------------------------------------------------------------- loss
# Rows that a warp, a block, a cluster and the two-pass kernel work on, in both types.
LOSS_WIDTHS = [64, 1003, 8192, 50_001, 140_000, 1_000_003]


def check_loss(x, tgt, **args):
    """Loss, lse and gradient of rows x [T, V] of one type against loss_ref, and the call without gradient."""
    T = x.shape[0]
    tk = torch.from_numpy(tgt).to(DEV)
    loss, lse, g = E.cross_entropy(x, tk, **args)
    want = loss_ref(f64(x)[None], tgt[None], np.ones((1, T)), np.ones((1, T), bool))
    loss_w, lse_w, g_w, el, es, eg = (a[0] for a in want)
    check(loss, loss_w, el, "loss")
    check(lse, lse_w, es, "lse")
    check(g, g_w, out_u(x.dtype) * np.abs(g_w) + eg, "dlogits")
    alone = E.cross_entropy(x, tk, want_grad=False, **args)
    check(alone[0], loss_w, el, "loss alone")
    check(alone[1], lse_w, es, "lse alone")


@pytest.mark.parametrize("dt", TYPES)
@pytest.mark.parametrize("V", LOSS_WIDTHS)
def test_cross_entropy_far_rows(dt, V):
    """Rows of equal and of mixed logits far from 0: finite logits give finite losses, whatever they are."""
    far = [s * m for m in (1e6, 2.0 ** 20, 2.0 ** 20 + 1, 3e7, 1e8, 2.0 ** 27, 2.0 ** 27 + 16, 3e8, 1e9, 1e10, 1.1e10, 1e12, 1e20, 0.9e29, 3e29)
           for s in (1, -1)]
    rng = np.random.default_rng(V)
    for q in far:
        x = np.full((2, V), q, np.float64)
        # in steps of the type's spacing there, some of which are less than 1
        x[1] += rng.integers(-4, 5, V) * abs(q) * 2 * out_u(dt)
        check_loss(torch.from_numpy(x.astype(np.float32)).to(DEV).to(dt), np.array([3, V - 1]))


@pytest.mark.parametrize("dt", TYPES)
@pytest.mark.parametrize("V", LOSS_WIDTHS)
def test_cross_entropy_far_masks(dt, V):
    """Masks of finite values in front of, behind and between ordinary logits, single survivors, and logits that
    rise from far below: a thread, a warp or a block may meet the masked ones first, or nothing else."""
    rng = np.random.default_rng(V + 1)
    for mask in (-3e4, -1e8, -1e9, -1e10, -1.1e10, -1e12, -1e20, -0.9e29, -1e30):
        x = rng.standard_normal((6, V)) * 2
        x[0, :V // 2] = mask
        x[1, V // 2:] = mask
        x[2, rng.random(V) < 0.9] = mask
        x[2, V - 1] = 0.3
        x[3, :] = mask
        x[3, V - 2] = 0.3              # the target alone is left
        x[4, :-1] = mask               # a far row but for one logit of ordinary size
        x[5] = np.linspace(mask, 0, V)
        tgt = np.array([V - 2, 1, V - 1, V - 2, V - 1, V - 1])
        check_loss(torch.from_numpy(x.astype(np.float32)).to(DEV).to(dt), tgt)
    for far in (3e6, 3e8):             # through every bound on the way
        x = np.stack([np.linspace(-far, 0, V), np.linspace(-far, -0.47 * far, V), np.linspace(0, far, V)])
        check_loss(torch.from_numpy(x.astype(np.float32)).to(DEV).to(dt), np.array([V - 1, V - 1, V - 2]))


@pytest.mark.parametrize("dt", TYPES)
@pytest.mark.parametrize("V", [1, 7, 64, 97, 515, 1000, 1024, 2000, 2048, 5000, 50_001, 140_000])
def test_cross_entropy_over_its_logits(dt, V):
    """Loss and lse, not the gradient alone, have the same bits where the gradient is written over the logits, with
    targets in every place of a row: the target's logit is read before anything is written over it."""
    T = min(8192, max(64, (1 << 25) // V))
    gen = torch.Generator(device=DEV)
    gen.manual_seed(V)
    x = torch.empty((T, V), dtype=dt, device=DEV).normal_(generator=gen).mul_(3)
    tgt = torch.arange(T, device=DEV) * 7 % V
    want = E.cross_entropy(x, tgt)
    for _ in range(3):
        xx = x.clone()
        got = E.cross_entropy(xx, tgt, dlogits=xx)
        assert got[2] is xx
        assert all(torch.equal(p, q) for p, q in zip(got, want))


# ----------------------------------------------------------- normalisation
@pytest.mark.parametrize("kind", [E.NORM_LAYER, E.NORM_RMS])
@pytest.mark.parametrize("d", [33, 64, 256, 768, 770, 2048, 4095, 20_000])
def test_norm_grad_of_rows_with_an_offset(kind, d):
    """dx where the rows' mean is many times their spread and dy follows the rows: its error is that of centred rows.

    mean and rstd are inputs, so the formula holds for them as given. With e = x - mean (off by u |e|), xh = e rstd
    and g = dy w: mean(g) and mean(g xh) are off by (c + 4) u of the mean magnitudes, c the chain of the sums, and
    the terms g, mean(g) and xh mean(g xh), in whatever grouping, by a few u each."""
    rng = np.random.default_rng(d)
    rows = np.array([0.0, 3.0, 30.0, 300.0, 3000.0])
    T = len(rows)
    x = (rng.standard_normal((1, T, d)) + rows[None, :, None]).astype(np.float32)
    x64 = x.astype(np.float64)
    mu64 = x64.mean(-1) if kind == E.NORM_LAYER else np.zeros((1, T))
    mu = mu64.astype(np.float32)
    rs = (1 / np.sqrt(((x64 - mu64[..., None]) ** 2).mean(-1) + 1e-5)).astype(np.float32)
    xh = (x64 - mu[..., None].astype(np.float64)) * rs[..., None].astype(np.float64)
    w = (1 + 0.1 * rng.standard_normal(d)).astype(np.float32)
    dy = (xh + 0.3 * rng.standard_normal((1, T, d))).astype(np.float32)
    g = dy.astype(np.float64) * w
    r = rs[..., None].astype(np.float64)
    m1 = g.mean(-1, keepdims=True) if kind == E.NORM_LAYER else np.zeros((1, T, 1))
    m2 = (g * xh).mean(-1, keepdims=True)
    want = r * (g - m1 - xh * m2)
    c = chain(d) + (d / 256 if d > 16_384 else 0)      # the widest rows: one block, an element a thread
    e1 = np.abs(g).mean(-1, keepdims=True) if kind == E.NORM_LAYER else 0.0
    tol = r * U * ((c + 8) * (e1 + np.abs(xh) * np.abs(g * xh).mean(-1, keepdims=True)) +
                   8 * (np.abs(g) + np.abs(m1) + np.abs(xh * m2)))
    t = lambda a: torch.from_numpy(a).to(DEV)  # noqa: E731
    dx, _, _ = E.norm_grad(t(dy), t(x), t(mu) if kind == E.NORM_LAYER else None, t(rs), t(w), kind=kind)
    check(dx, want, tol, "dx")


@pytest.mark.parametrize("kind", [E.NORM_LAYER, E.NORM_RMS])
@pytest.mark.parametrize("dt", TYPES)
@pytest.mark.parametrize("d", [8, 24, 40, 72, 100, 136, 200, 264, 392, 520, 770, 776, 1003, 1544, 4104, 16_392, 20_000])
def test_norm_grad_over_its_inputs(kind, dt, d):
    """dx over dy and over x, in rows that leave lanes and threads of their last vector over: the bits of the others."""
    T = min(4096, max(8, (1 << 22) // d))
    gen = torch.Generator(device=DEV)
    gen.manual_seed(d)
    x, dy = (torch.empty((3, T, d), dtype=dt, device=DEV).normal_(generator=gen) for _ in range(2))
    ln = torch.tensor([T, 1, T // 2], dtype=torch.int32, device=DEV)
    w = torch.rand((d,), generator=gen, device=DEV).to(dt)
    for lengths in (None, ln):
        _, mean, rstd = E.norm(x, w, kind=kind, lengths=lengths)
        want = E.norm_grad(dy, x, mean, rstd, w, kind=kind, lengths=lengths)
        for over in ("dy", "x"):
            a, b = dy.clone(), x.clone()
            got = E.norm_grad(a, b, mean, rstd, w, kind=kind, lengths=lengths, dx=a if over == "dy" else b)
            assert all(torch.equal(p, q) for p, q in zip(got, want)), over


def test_norm_grad_of_very_wide_rows():
    """More channels than 65,535 blocks of threads: the weights' gradients and dx, in place of dy."""
    if torch.cuda.mem_get_info()[0] < 8 << 30:
        pytest.skip("needs 8 GB of device memory")
    T, d = 2, 65_536 * 256 + 257
    gen = torch.Generator(device=DEV)
    gen.manual_seed(5)
    x, dy = (torch.randn((1, T, d), generator=gen, device=DEV) for _ in range(2))
    mean, rstd = x.mean(-1), 1 / x.std(-1)
    xh = (x.double() - mean.double()[..., None]) * rstd.double()[..., None]
    g = dy.double()
    dw_w, db_w = (g * xh).sum((0, 1)), g.sum((0, 1))
    dw_m, db_m = (g * xh).abs().sum((0, 1)), g.abs().sum((0, 1))
    m1, m2 = g.mean(-1, keepdim=True), (g * xh).mean(-1, keepdim=True)
    dx_w = rstd.double()[..., None] * (g - m1 - xh * m2)
    # The means over channels: chains of d / 256 terms, whose errors of random sign add up to far less than the
    # bound d / 256 u; it is 4e-3 of the mean magnitudes, which are below 1.
    c = d / 256 + 32
    dx_m = rstd.double()[..., None] * U * ((c + 8) * (1 + xh.abs()) + 8 * g.abs())
    dx, dw, db = E.norm_grad(dy, x, mean, rstd, dx=dy)
    assert dx is dy
    assert bool(((dw.double() - dw_w).abs() <= 8 * U * dw_m).all())
    assert bool(((db.double() - db_w).abs() <= 4 * U * db_m).all())
    assert bool(((dx.double() - dx_w).abs() <= dx_m).all())


# ----------------------------------------------------------- all operators
def test_host_threads_with_calls_of_different_sizes():
    """Calls of several host threads, each on a stream of its own, that launch one kernel with different amounts of
    shared memory: none is refused, and all give what they give alone."""
    import threading
    gen = torch.Generator(device=DEV)
    gen.manual_seed(1)
    R, L = 200, E.lib()
    jobs = []      # (call, its arguments but for the stream, outputs): nothing but the C calls in the threads' loops
    for V in (12_500, 17_000, 22_000, 27_000):     # 50 to 108 KB a row of fp32
        x = torch.randn((R, V), generator=gen, device=DEV)
        tgt = torch.randint(0, V, (R,), generator=gen, device=DEV)
        loss, g = torch.empty(R, device=DEV), torch.empty_like(x)
        jobs.append((L.eogp_cross_entropy,
                     (x.data_ptr(), E.F32, 0, V, tgt.data_ptr(), E.I64, 0, None, -100, None, 1, R, V, loss.data_ptr(),
                      None, g.data_ptr(), 0, V), (loss, g), (x, tgt)))
    for d in (260, 300, 340, 384):                 # 51 to 53 KB a block, of one kernel
        x, dy = (torch.randn((R, d), generator=gen, device=DEV) for _ in range(2))
        _, mean, rstd = E.norm(x)
        dx = torch.empty_like(x)
        jobs.append((L.eogp_norm_grad,
                     (E.NORM_LAYER, dy.data_ptr(), 0, d, x.data_ptr(), E.F32, 0, d, mean.data_ptr(), rstd.data_ptr(),
                      None, E.F32, None, 1, R, d, dx.data_ptr(), 0, d, None, None, 0, 0, 0, None, 0), (dx,),
                     (x, dy, mean, rstd)))
    torch.cuda.synchronize()
    for call, args, outs, _ in jobs:
        assert call(*args, None) == E.OK
    torch.cuda.synchronize()
    want = [[t.clone() for t in outs] for _, _, outs, _ in jobs]
    torch.cuda.synchronize()
    refused = []

    def work(call, args):
        stream = torch.cuda.Stream()
        for _ in range(4000):
            if call(*args, stream.cuda_stream) != E.OK:
                refused.append(E.lib().eogp_last_error())
                break
        stream.synchronize()

    threads = [threading.Thread(target=work, args=j[:2]) for j in jobs]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    torch.cuda.synchronize()
    assert not refused, refused
    for j, expect in zip(jobs, want):
        assert all(torch.equal(p, q) for p, q in zip(j[2], expect))
