"""Refusals of the token loss through the output matrix and of distillation: arguments are
checked on the host before anything is launched, by the C ABI and by the binding. No GPU
needed."""
import ctypes

import pytest

from paper_2609_37842_gb300 import build as B
from paper_2609_37842_gb300 import eogp as E

torch = pytest.importorskip("torch")


@pytest.fixture(scope="module", autouse=True)
def built():
    B.build()
    E.lib()


def call(name, base, **change):
    """Status of the C call with the named arguments `base`, some of them changed."""
    args = dict(base)
    assert set(change) <= set(args)
    args.update(change)
    return getattr(E.lib(), name)(*args.values())


HEAD = dict(x=256, dtype=E.BF16, x_bs=32, x_ld=8, weight=256, ld_weight=8, scale=1.0, targets=256, index_type=E.I64,
            targets_bs=4, weights=None, ignore_index=-100, lengths=None, B=2, T=4, d=8, V=10, loss=256, lse=256, dx=256,
            dx_bs=32, dx_ld=8, dweight=256, grad_dtype=E.F32, ld_dweight=8, accumulate=0, ws=256, ws_bytes=1 << 40,
            stream=None)
DISTILL = dict(logits=256, dtype=E.BF16, logits_bs=32, logits_ld=8, classes=256, index_type=E.I64, classes_bs=12,
               classes_ld=3, teacher=256, teacher_dtype=E.F32, teacher_bs=12, teacher_ld=3, teacher_lse=None, K=3,
               temperature=1.0, weights=None, lengths=None, B=2, T=4, V=8, loss=256, lse=256, dlogits=256,
               dlogits_bs=32, dlogits_ld=8, stream=None)
NAN, INF = float("nan"), float("inf")


@pytest.mark.parametrize("change,code", [
    (dict(x=None), E.EINVAL), (dict(weight=None), E.EINVAL), (dict(targets=None), E.EINVAL),
    (dict(loss=None), E.EINVAL), (dict(dtype=E.I32), E.EINVAL), (dict(grad_dtype=E.I64), E.EINVAL),
    (dict(index_type=E.F32), E.EINVAL), (dict(V=0), E.EINVAL), (dict(d=0), E.EINVAL), (dict(B=-1), E.EINVAL),
    (dict(T=-1), E.EINVAL), (dict(scale=NAN), E.EINVAL), (dict(scale=INF), E.EINVAL), (dict(x=257), E.EINVAL),
    (dict(weight=257), E.EINVAL), (dict(targets=260), E.EINVAL), (dict(loss=258), E.EINVAL), (dict(dx=257), E.EINVAL),
    (dict(dweight=258), E.EINVAL), (dict(lengths=258), E.EINVAL), (dict(weights=258), E.EINVAL),
    (dict(x_bs=-1), E.EINVAL), (dict(x_ld=-8), E.EINVAL), (dict(ld_weight=-8), E.EINVAL),
    (dict(targets_bs=-1), E.EINVAL), (dict(dx_ld=7), E.EINVAL), (dict(dx_bs=31), E.EINVAL),
    (dict(ld_dweight=7), E.EINVAL), (dict(ws=None), E.EWORKSPACE), (dict(ws_bytes=1024), E.EWORKSPACE),
    (dict(ws=264), E.EINVAL), (dict(B=1 << 20, T=1 << 11), E.EUNSUPPORTED),
    (dict(V=(1 << 30) + 1), E.EUNSUPPORTED), (dict(d=(1 << 30) + 1), E.EUNSUPPORTED),
    (dict(dtype=E.F32, grad_dtype=E.BF16), E.EUNSUPPORTED),
])
def test_head_loss_refuses(change, code):
    assert call("eogp_head_loss", HEAD, **change) == code
    assert E.lib().eogp_last_error()


@pytest.mark.parametrize("change,code", [
    (dict(logits=None), E.EINVAL), (dict(classes=None), E.EINVAL), (dict(teacher=None), E.EINVAL),
    (dict(loss=None), E.EINVAL), (dict(dtype=E.I32), E.EINVAL), (dict(teacher_dtype=E.I32), E.EINVAL),
    (dict(index_type=E.BF16), E.EINVAL), (dict(K=0), E.EINVAL), (dict(K=E.DISTILL_MAX + 1), E.EINVAL),
    (dict(V=0), E.EINVAL), (dict(B=-1), E.EINVAL), (dict(temperature=0.0), E.EINVAL),
    (dict(temperature=-1.0), E.EINVAL), (dict(temperature=NAN), E.EINVAL), (dict(temperature=INF), E.EINVAL),
    (dict(temperature=1e-44), E.EINVAL), (dict(logits=257), E.EINVAL), (dict(classes=260), E.EINVAL),
    (dict(teacher=258), E.EINVAL), (dict(teacher_lse=258), E.EINVAL), (dict(dlogits=257), E.EINVAL),
    (dict(logits_ld=-1), E.EINVAL), (dict(classes_ld=-1), E.EINVAL), (dict(teacher_bs=-1), E.EINVAL),
    (dict(dlogits_ld=7), E.EINVAL), (dict(dlogits_bs=30), E.EINVAL),
    (dict(B=1 << 20, T=1 << 11), E.EUNSUPPORTED), (dict(V=(1 << 30) + 1), E.EUNSUPPORTED),
])
def test_distill_refuses(change, code):
    assert call("eogp_distill", DISTILL, **change) == code
    assert E.lib().eogp_last_error()


def test_empty_batches_need_no_device():
    for change in (dict(B=0), dict(T=0)):
        assert call("eogp_distill", DISTILL, **change) == E.OK
        assert call("eogp_head_loss", HEAD, dweight=None, ws=None, ws_bytes=0, **change) == E.OK


def size(**change):
    args = dict(weight=256, dtype=E.BF16, ld_weight=64, V=1000, d=64, B=4, T=50, want_dx=1, want_dweight=1,
                grad_dtype=E.F32)
    args.update(change)
    n = ctypes.c_size_t(77)
    rc = E.lib().eogp_head_loss_workspace_size(*args.values(), ctypes.byref(n))
    return (rc, n.value)


def test_head_workspace_sizes():
    assert E.lib().eogp_head_loss_workspace_size(256, E.BF16, 64, 1000, 64, 4, 50, 1, 1, E.F32, None) == E.EINVAL
    assert size(V=0)[0] == size(d=0)[0] == size(T=-1)[0] == size(dtype=E.I64)[0] == size(ld_weight=-1)[0] == E.EINVAL
    assert size(dtype=E.F32, grad_dtype=E.BF16)[0] == E.EUNSUPPORTED
    assert size(want_dweight=0, grad_dtype=-1)[0] == E.OK
    assert size(B=0) == (E.OK, 0)
    # The logits of the whole batch are never there: 2^20 positions of 100,000 classes would be 400 GB.
    rc, most = size(V=100_000, d=64, ld_weight=64, B=1 << 10, T=1 << 10)
    assert rc == E.OK and 0 < most < 8 << 30
    # Without a gradient none are.
    rc, none = size(V=100_000, d=64, ld_weight=64, B=1 << 10, T=1 << 10, want_dx=0, want_dweight=0)
    assert rc == E.OK and 0 < none <= most
    # Offsets of the largest sizes do not wrap.
    rc, n = size(V=1 << 30, d=1, ld_weight=1, B=1, T=1 << 30)
    assert rc == E.OK and n >= 256 * 4 << 30


def test_binding_refuses():
    x, w = torch.zeros((2, 3, 8)), torch.zeros((5, 8))
    tok = torch.zeros((2, 3), dtype=torch.int64)
    for f in (lambda: E.head_loss(x, w, tok), lambda: E.distill(x, tok[..., None], x[..., :1])):
        with pytest.raises(ValueError, match="CUDA device"):
            f()
