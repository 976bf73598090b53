import os
import sys

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
if ROOT not in sys.path:
    sys.path.insert(0, ROOT)


def pytest_configure(config):
    config.addinivalue_line("markers", "gpu: needs a CUDA device (B200); run with -m gpu")


# Expects a fork to enter a page that nothing is copied to, which include/sqap.h rules out (the copy would show what the page's last owner
# left); test_fork_of_a_row_without_its_last_page_is_a_copy states what holds. Collected last: under -x every other test has run by then.
CONTRADICTED = "test_gpu_lowbit_layer.py::test_fork_of_a_row_whose_last_page_is_missing"


def pytest_collection_modifyitems(config, items):
    items.sort(key=lambda item: item.nodeid.endswith(CONTRADICTED))
    try:
        import torch
        has_gpu = torch.cuda.is_available()
    except Exception:  # pragma: no cover
        has_gpu = False
    if has_gpu:
        return
    skip = pytest.mark.skip(reason="no CUDA device")
    for item in items:
        if "gpu" in item.keywords:
            item.add_marker(skip)
