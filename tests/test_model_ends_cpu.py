"""Refusals of the model-end operators (token embedding, normalisation, token
loss): arguments are checked on the host before anything is launched, by the C
ABI and by the binding. No GPU needed."""
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


EMBED = dict(tokens=256, index_type=E.I64, tokens_bs=4, table=256, dtype=E.BF16, V=10, d=8, ld_table=8, scale=1.0,
             pos=None, ld_pos=0, lengths=None, B=2, T=4, out=256, out_bs=32, out_ld=8, stream=None)
EMBED_GRAD = dict(tokens=256, index_type=E.I32, tokens_bs=4, dout=256, dtype=E.F32, dout_bs=32, dout_ld=8,
                  lengths=None, B=2, T=4, V=10, d=8, scale=1.0, dtable=256, grad_dtype=E.F32, ld_dtable=8,
                  accumulate=0, ws=256, ws_bytes=1 << 30, stream=None)
NORM = dict(kind=E.NORM_LAYER, x=256, dtype=E.BF16, x_bs=32, x_ld=8, weight=256, bias=256, param_dtype=E.BF16,
            eps=1e-5, lengths=None, B=2, T=4, d=8, y=256, y_bs=32, y_ld=8, mean=256, rstd=256, stream=None)
NORM_GRAD = dict(kind=E.NORM_LAYER, dy=256, dy_bs=32, dy_ld=8, x=256, dtype=E.F32, x_bs=32, x_ld=8, mean=256, rstd=256,
                 weight=256, param_dtype=E.F32, lengths=None, B=2, T=4, d=8, dx=256, dx_bs=32, dx_ld=8, dweight=256,
                 dbias=256, ld_dparam=8, per_example=1, accumulate=0, ws=256, ws_bytes=1 << 30, stream=None)
LOSS = dict(logits=256, dtype=E.BF16, logits_bs=32, logits_ld=8, targets=256, index_type=E.I64, targets_bs=4,
            weights=None, ignore_index=-100, lengths=None, B=2, T=4, V=8, loss=256, lse=256, dlogits=256,
            dlogits_bs=32, dlogits_ld=8, stream=None)


@pytest.mark.parametrize("name,base,change,code", [
    ("eogp_embed", EMBED, dict(tokens=None), E.EINVAL), ("eogp_embed", EMBED, dict(table=None), E.EINVAL),
    ("eogp_embed", EMBED, dict(out=None), E.EINVAL), ("eogp_embed", EMBED, dict(index_type=E.BF16), E.EINVAL),
    ("eogp_embed", EMBED, dict(dtype=E.I32), E.EINVAL), ("eogp_embed", EMBED, dict(V=0), E.EINVAL),
    ("eogp_embed", EMBED, dict(d=0), E.EINVAL), ("eogp_embed", EMBED, dict(B=-1), E.EINVAL),
    ("eogp_embed", EMBED, dict(out_ld=7), E.EINVAL), ("eogp_embed", EMBED, dict(out_bs=31), E.EINVAL),
    ("eogp_embed", EMBED, dict(table=257), E.EINVAL), ("eogp_embed", EMBED, dict(tokens=260), E.EINVAL),
    ("eogp_embed", EMBED, dict(tokens_bs=-1), E.EINVAL), ("eogp_embed", EMBED, dict(ld_table=-8), E.EINVAL),
    ("eogp_embed", EMBED, dict(B=1 << 20, T=1 << 11), E.EUNSUPPORTED),
    ("eogp_embed_grad", EMBED_GRAD, dict(dout=None), E.EINVAL),
    ("eogp_embed_grad", EMBED_GRAD, dict(dtable=None), E.EINVAL),
    ("eogp_embed_grad", EMBED_GRAD, dict(ld_dtable=7), E.EINVAL),
    ("eogp_embed_grad", EMBED_GRAD, dict(ws=None), E.EWORKSPACE),
    ("eogp_embed_grad", EMBED_GRAD, dict(ws_bytes=16), E.EWORKSPACE),
    ("eogp_embed_grad", EMBED_GRAD, dict(ws=264), E.EINVAL),
    ("eogp_embed_grad", EMBED_GRAD, dict(grad_dtype=7), E.EINVAL),
    ("eogp_embed_grad", EMBED_GRAD, dict(dout_ld=-1), E.EINVAL),
    ("eogp_norm", NORM, dict(kind=2), E.EINVAL), ("eogp_norm", NORM, dict(x=None), E.EINVAL),
    ("eogp_norm", NORM, dict(y=None), E.EINVAL), ("eogp_norm", NORM, dict(eps=-1e-5), E.EINVAL),
    ("eogp_norm", NORM, dict(eps=float("nan")), E.EINVAL), ("eogp_norm", NORM, dict(y_ld=4), E.EINVAL),
    ("eogp_norm", NORM, dict(y_bs=8), E.EINVAL), ("eogp_norm", NORM, dict(param_dtype=5), E.EINVAL),
    ("eogp_norm", NORM, dict(mean=258), E.EINVAL), ("eogp_norm", NORM, dict(d=0), E.EINVAL),
    ("eogp_norm_grad", NORM_GRAD, dict(dy=None), E.EINVAL), ("eogp_norm_grad", NORM_GRAD, dict(rstd=None), E.EINVAL),
    ("eogp_norm_grad", NORM_GRAD, dict(mean=None), E.EINVAL),
    ("eogp_norm_grad", NORM_GRAD, dict(ld_dparam=7), E.EINVAL),
    ("eogp_norm_grad", NORM_GRAD, dict(ws=None), E.EWORKSPACE),
    ("eogp_norm_grad", NORM_GRAD, dict(dx_ld=7), E.EINVAL), ("eogp_norm_grad", NORM_GRAD, dict(T=-2), E.EINVAL),
    ("eogp_cross_entropy", LOSS, dict(logits=None), E.EINVAL), ("eogp_cross_entropy", LOSS, dict(loss=None), E.EINVAL),
    ("eogp_cross_entropy", LOSS, dict(targets=None), E.EINVAL), ("eogp_cross_entropy", LOSS, dict(V=0), E.EINVAL),
    ("eogp_cross_entropy", LOSS, dict(dlogits_ld=7), E.EINVAL),
    ("eogp_cross_entropy", LOSS, dict(dlogits_bs=30), E.EINVAL),
    ("eogp_cross_entropy", LOSS, dict(logits_bs=-1), E.EINVAL),
    ("eogp_cross_entropy", LOSS, dict(logits=257), E.EINVAL), ("eogp_cross_entropy", LOSS, dict(dtype=3), E.EINVAL),
])
def test_c_calls_refuse(name, base, change, code):
    assert call(name, base, **change) == code
    assert E.lib().eogp_last_error()


def test_empty_batches_need_no_device():
    """Nothing to read and nothing that a sum over tokens would set: done without a launch."""
    for name, base in (("eogp_embed", EMBED), ("eogp_norm", NORM), ("eogp_cross_entropy", LOSS)):
        assert call(name, base, B=0) == E.OK
        assert call(name, base, T=0) == E.OK


def test_workspace_sizes():
    n = ctypes.c_size_t()
    L = E.lib()
    assert L.eogp_embed_grad_workspace_size(100, 64, 0, 5, ctypes.byref(n)) == E.OK and n.value == 0
    assert L.eogp_embed_grad_workspace_size(100, 64, 4, 5, ctypes.byref(n)) == E.OK and n.value > 0
    assert L.eogp_embed_grad_workspace_size(0, 64, 4, 5, ctypes.byref(n)) == E.EINVAL
    assert L.eogp_embed_grad_workspace_size(100, 64, 4, 5, None) == E.EINVAL
    assert L.eogp_norm_grad_workspace_size(4, 5, 64, 1, ctypes.byref(n)) == E.OK
    assert L.eogp_norm_grad_workspace_size(4, 5, 0, 1, ctypes.byref(n)) == E.EINVAL
    assert L.eogp_norm_grad_workspace_size(4, -5, 64, 1, ctypes.byref(n)) == E.EINVAL


def test_binding_refuses_host_tensors():
    x = torch.zeros((2, 3, 8))
    tok = torch.zeros((2, 3), dtype=torch.int64)
    for f in (lambda: E.norm(x), lambda: E.embed(tok, torch.zeros((4, 8))), lambda: E.embed_grad(tok, x, 4),
              lambda: E.cross_entropy(x, tok), lambda: E.norm_grad(x, x, x[..., 0], x[..., 0])):
        with pytest.raises(ValueError, match="CUDA device"):
            f()
