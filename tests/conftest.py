import os
import sys

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
if ROOT not in sys.path:
    sys.path.insert(0, ROOT)


def pytest_configure(config):
    config.addinivalue_line("markers", "gpu: needs a real MI355X (run with -m gpu)")


def _gpu_available() -> bool:
    try:
        import torch
        return torch.cuda.is_available()
    except Exception:
        return False


# Tests of refusals with a call in them that is not refused: without a GPU it ends where the device is asked for, with one it would
# read made-up addresses.
NO_GPU_ONLY = ("test_paged_q4.py::test_row_calls_and_copy_refusals",)


def pytest_collection_modifyitems(config, items):
    if _gpu_available():
        skip = pytest.mark.skip(reason="hands made-up addresses to a call that is not refused")
        for item in items:
            if item.nodeid.endswith(NO_GPU_ONLY):
                item.add_marker(skip)
        return
    skip = pytest.mark.skip(reason="no GPU in this process")
    for item in items:
        if "gpu" in item.keywords:
            item.add_marker(skip)
