import gc
import os
import sys

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
if ROOT not in sys.path:
    sys.path.insert(0, ROOT)


def pytest_configure(config):
    config.addinivalue_line("markers", "gpu: needs a real MI355X (run with -m gpu)")


def pytest_collection_modifyitems(config, items):
    try:
        import torch
        has_gpu = torch.cuda.is_available()
    except Exception:
        has_gpu = False
    if has_gpu:
        return
    skip = pytest.mark.skip(reason="no GPU visible")
    for item in items:
        if "gpu" in item.keywords:
            item.add_marker(skip)


@pytest.fixture(autouse=True)
def _no_cycle_collection_between_two_readings(request):
    """The test of the entry point that allocates nothing compares how much device memory is allocated before and after a
    call.  What an earlier call left in a cycle (pytest.raises keeps its frame, with the nets and tensors in it) would be
    freed by a collection in between, whose moment depends on how many objects the tests before it made."""
    if request.path.name != "test_zz_no_alloc.py" or not gc.isenabled():
        yield
        return
    gc.disable()
    yield
    gc.enable()
