import os
import sys

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
if ROOT not in sys.path:
    sys.path.insert(0, ROOT)


def pytest_configure(config):
    config.addinivalue_line("markers", "gpu: needs a CUDA GPU (GB300, sm_103a)")
    config.addinivalue_line("markers", "slow: long-running CPU test")


# Tests whose expected value is wrong, and why. They run, and have to fail.
_MASS = ("takes p - q for the gradient where the list's q and the rest add up to Q, not 1; the derivative of that loss is "
         "Q p - q (test_gpu_distill_edges.py: test_mass_above_one, test_mass_of_all_classes)")
WRONG_VALUE = {f"test_gpu_distill.py::{name}": _MASS for name in (
    "test_teacher_above_one[100]", "test_teacher_above_one[5000]", "test_teacher_above_one[60001]",
    # every class listed, of a teacher whose log-sum leaves some of its mass
    "test_against_formulas[1-1-1-1-True-dt0]", "test_against_formulas[1-1-1-1-True-dt1]",
    "test_against_formulas[2-3-5-5-True-dt0]", "test_against_formulas[2-3-5-5-True-dt1]")}


def pytest_collection_modifyitems(items):
    for item in items:
        reason = WRONG_VALUE.get(f"{item.path.name}::{item.name}")
        if reason:
            item.add_marker(pytest.mark.xfail(reason=reason, strict=True))


@pytest.fixture
def eogp_options():
    """Setter for the library's process-wide dispatch options
    (eogp_set_option); both are put back to their defaults afterwards."""
    from paper_2609_37842_gb300 import eogp as E

    def setter(score_operand=None, topk_path=None):
        if score_operand is not None:
            E.set_option(E.OPT_SCORE_OPERAND, score_operand)
        if topk_path is not None:
            E.set_option(E.OPT_TOPK_PATH, topk_path)

    yield setter
    E.set_option(E.OPT_SCORE_OPERAND, 0)
    E.set_option(E.OPT_TOPK_PATH, 0)
