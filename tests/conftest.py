import os
import sys

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
if ROOT not in sys.path:
    sys.path.insert(0, ROOT)


def pytest_configure(config):
    config.addinivalue_line("markers", "gpu: needs an MI355X (gfx950) GPU and the built HIP library")
    config.addinivalue_line("markers", "slow: takes more than a few seconds of CPU time")


# Tests of refusals in which calls with made-up addresses pass every check of the arguments: they end with VC_ERR_DEVICE where
# there is no GPU, and would launch, and write to those addresses, where there is one.
WITHOUT_GPU_ONLY = ("test_blocks_abi.py::test_residual_pointers_and_combinations",)


def pytest_collection_modifyitems(config, items):
    # GPU tests run only where a GPU is present; never silently on CPU.
    try:
        import torch
        has_gpu = torch.cuda.is_available()
    except Exception:
        has_gpu = False
    if has_gpu:
        skip = pytest.mark.skip(reason="its calls would launch on made-up addresses; runs where there is no GPU")
        for it in items:
            if it.nodeid.endswith(WITHOUT_GPU_ONLY):
                it.add_marker(skip)
        return
    skip = pytest.mark.skip(reason="no GPU in this environment")
    for it in items:
        if "gpu" in it.keywords:
            it.add_marker(skip)
