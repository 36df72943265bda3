"""Refusals and sizes of the token loss through the output matrix and of distillation at the ends of their
ranges: arguments are checked on the host before anything is launched. No GPU needed."""
import pytest

pytest.importorskip("torch")

from paper_2609_37842_gb300 import eogp as E  # noqa: E402
from test_more_losses_cpu import DISTILL, HEAD, built, call, size  # noqa: E402,F401


@pytest.mark.parametrize("temperature", [3.0e-39, 4.0e-39, 5.8e-39, 8.8e-39])
def test_temperatures_whose_exponents_are_no_floats(temperature):
    """log2(e) / h or twice that, which differences are scaled by, is beyond a float there: answers would be NaN."""
    assert call("eogp_distill", DISTILL, temperature=temperature) == E.EINVAL


@pytest.mark.parametrize("dtype,grad,T,d,V", [(E.BF16, E.BF16, 511, 768, 50_001), (E.F32, E.F32, 509, 770, 32_001),
                                              (E.BF16, E.F32, 511, 768, 50_001), (E.BF16, E.BF16, 64, 4096, 100_000)])
def test_workspace_of_one_example(dtype, grad, T, d, V):
    """What one example's workspace holds: its logits in fp32, D where it lies beside them (fp32: three bf16 parts),
    a copy of an fp32 matrix in such parts, and slabs of dx for sums split 32 times at most; not slabs of dW, whose
    sum over so few positions is not split."""
    rows, cols = -(-T // 256) * 256, -(-V // 64) * 64
    most = rows * cols * (4 if dtype == E.BF16 else 4 + 6) + 32 * T * (d + 8) * 4
    if dtype == E.F32:
        most += V * (d + 64) * 6
    most += rows * (d + 64) * 6 + rows * cols // 8  # rows of x; sums of half tiles, positions
    rc, n = size(dtype=dtype, grad_dtype=grad, T=T, B=1, d=d, V=V, ld_weight=d)
    assert rc == E.OK and n <= most


def test_widest_rows():
    """Rows of an fp32 x are three bf16 rows side by side, whose columns are counted by ints; the sizes of those that
    are taken do not wrap."""
    for V, d in ((1, 1 << 30), (50, 800_000_000), (1000, 715_827_841)):
        assert size(dtype=E.F32, B=1, T=1, V=V, d=d, ld_weight=d)[0] == E.EUNSUPPORTED
        assert call("eogp_head_loss", HEAD, dtype=E.F32, V=V, d=d, ld_weight=d, dx_ld=d, dx_bs=4 * d, ld_dweight=d,
                    ws_bytes=1 << 62) == E.EUNSUPPORTED
    rc, n = size(dtype=E.F32, B=1, T=1, V=2, d=715_827_840, ld_weight=715_827_840)
    assert rc == E.OK and n >= 258 * 715_827_840 * 6
    rc, n = size(dtype=E.BF16, B=1, T=1, V=2, d=1 << 30, ld_weight=1 << 30)
    assert rc == E.OK and n >= 256 << 31


def test_example_refuses_unknown_losses():
    from paper_2609_37842_gb300 import attribute_lm as L
    for loss_from, message in (("logit", "loss_from must be"), ("distill", "needs a teacher")):
        with pytest.raises(ValueError, match=message):
            L.backward_pass(None, None, None, loss_from)
