"""Properties of the compiled kernels around a block's attention (CPU: hipcc cross-compiles to assembly): no packed fp32
arithmetic, no vector spills."""
import re

import pytest

import test_kernel_asm as K
from test_kernel_asm import device_asm  # noqa: F401

FILES = ["residual.hip", "checkpoint.hip", "embedding.hip"]


@pytest.fixture(scope="module", autouse=True)
def block_sources():
    old, K.SOURCES = K.SOURCES, FILES
    yield
    K.SOURCES = old


def test_no_packed_arithmetic(device_asm):  # noqa: F811
    K.test_no_packed_fp32_arithmetic(device_asm)


@pytest.mark.parametrize("fn", FILES)
def test_no_vector_spills(device_asm, fn):  # noqa: F811
    found = re.findall(r"\.name:\s+(_Z\w+)\n(?:.*\n){0,40}?\s+\.vgpr_spill_count:\s+(\d+)", device_asm[fn])
    assert found and all(int(n) == 0 for _, n in found), [f for f in found if int(f[1])]
