"""Refusals and sizes of the token loss through the output matrix and of distillation at the ends of their
ranges: arguments are checked on the host before anything is launched. No GPU needed."""
import pytest

pytest.importorskip("torch")

from paper_2609_37842_gb300 import eogp as E  # noqa: E402
from test_more_losses_cpu import DISTILL, built, call  # noqa: E402,F401


@pytest.mark.parametrize("temperature", [3.0e-39, 4.0e-39, 5.8e-39])
def test_temperatures_whose_exponents_are_no_floats(temperature):
    """log2(e) / h, which logits are scaled by, is beyond a float there: every answer would be NaN."""
    assert call("eogp_distill", DISTILL, temperature=temperature) == E.EINVAL
