"""The tests of refusals pass made-up addresses: beside a GPU too, none of their calls may reach it."""
import os
import subprocess
import sys

import pytest

TESTS = os.path.dirname(os.path.abspath(__file__))


@pytest.mark.parametrize("fn", ["test_abi.py", "test_tower_abi.py", "test_blocks_abi.py"])
def test_no_refusal_reaches_a_gpu(fn):
    import torch
    if torch.cuda.is_available():
        pytest.skip("shown on a machine without a GPU")
    env = dict(os.environ, PYTHONPATH=os.pathsep.join([TESTS, os.path.dirname(TESTS)]))
    res = subprocess.run([sys.executable, "-m", "pytest", os.path.join(TESTS, fn), "-q", "-m", "not gpu", "-p", "gpu_pretender", "-p", "no:cacheprovider"],
                         env=env, cwd=os.path.dirname(TESTS), capture_output=True, text=True, timeout=300)
    assert res.returncode == 0 and " passed" in res.stdout, res.stdout[-3000:] + res.stderr[-1000:]
