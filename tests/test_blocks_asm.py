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
    # the residual's backward over more than 2,048 columns (its last flag) is at the limit of 256 registers
    wide = [n for n, _ in found if re.search(r"residual_bwd_kernelI.*Lb0EEEv", n)]
    assert found and all(int(n) == 0 or name in wide and int(n) <= 32 for name, n in found), [f for f in found if int(f[1])]
