import contextlib
import os
import sys

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
if ROOT not in sys.path:
    sys.path.insert(0, ROOT)


def pytest_configure(config):
    config.addinivalue_line("markers", "gpu: needs a CUDA device (runs on a B200)")


def pytest_collection_modifyitems(config, items):
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


def run_once_before(function, params):
    """The first of two runs of a test that compares the device's free memory: the driver loads a kernel's code (the
    library's, torch's) at its first launch and takes 2 MiB when a chunk of code is full, which such a comparison cannot tell
    from an allocation.  After this run all code the test needs is loaded, whichever tests ran before.  What it asserts
    counts in the second run."""
    if "mem_get_info" in function.__code__.co_names:
        with contextlib.suppress(AssertionError):
            function(**params)


@pytest.fixture(autouse=True)
def _code_is_loaded(request):
    if "gpu" in request.node.keywords:
        run_once_before(request.function, request.node.callspec.params if hasattr(request.node, "callspec") else {})
