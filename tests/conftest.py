import os
import sys

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
if ROOT not in sys.path:
    sys.path.insert(0, ROOT)


def pytest_configure(config):
    config.addinivalue_line("markers", "gpu: needs a real MI355X (run with -m gpu)")


# Tests that hold a wrong value: they run, and have to fail (strict).
WRONG_VALUES = {
    "test_gpu_operators.py::test_log_probs_special_rows[":
        "rows 4 and 7 are V equal logits, so p = 1/V; the test expects p = exp(x - lse) = 1 from an lse that fp32 rounds to x "
        "(the expected gradient of a log probability then sums to 1 - V over the row instead of to 0).  The right values, with all "
        "else that it checks: test_log_probs_special_rows_both_directions",
}


def pytest_collection_modifyitems(config, items):
    """GPU tests are skipped when no device is visible (the CPU suite runs with -m 'not gpu')."""
    for item in items:
        for name, reason in WRONG_VALUES.items():
            if name in item.nodeid:
                item.add_marker(pytest.mark.xfail(reason=reason, strict=True))
    try:
        import torch
        has_gpu = torch.cuda.is_available()
    except Exception:  # pragma: no cover
        has_gpu = False
    if has_gpu:
        return
    skip = pytest.mark.skip(reason="no GPU visible")
    for item in items:
        if "gpu" in item.keywords:
            item.add_marker(skip)
