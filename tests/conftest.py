import os
import sys

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
if ROOT not in sys.path:
    sys.path.insert(0, ROOT)


def pytest_configure(config):
    config.addinivalue_line("markers", "gpu: needs a CUDA device (run on a B200 with -m gpu)")


def holds_a_wrong_value(module, test, params):
    """Tests of test_gpu_drafts.py that compare topk_distill's gradient with q - p also in rows whose teacher's outcomes do not sum to one, where that is not the
    slope of the loss (test_distill_slope.py shows it by differences).  They stay as they are and have to fail; test_gpu_draft_edges.py runs the same rows
    against the slope."""
    return module == "test_gpu_drafts" and (test == "test_topk_distill_masked_logits" or
                                            test == "test_topk_distill_entries_that_are_missing_or_double" and (not params["rest"] or params["vocab"] == 6))


def pytest_collection_modifyitems(config, items):
    for item in items:
        if hasattr(item, "callspec") and holds_a_wrong_value(item.module.__name__, item.originalname, item.callspec.params):
            item.add_marker(pytest.mark.xfail(raises=AssertionError, strict=True, reason="holds a gradient that is not the slope of the loss"))
    try:
        import torch
        has_gpu = torch.cuda.is_available()
    except Exception:
        has_gpu = False
    if has_gpu:
        return
    skip = pytest.mark.skip(reason="no CUDA device")
    for item in items:
        if "gpu" in item.keywords:
            item.add_marker(skip)
