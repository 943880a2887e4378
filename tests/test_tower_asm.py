"""Properties of the compiled packed-attention kernels (CPU: hipcc cross-compiles to assembly), with the detectors of
test_kernel_asm: M0 set by the LDS copies only, their scalar bases settled, no packed fp32 arithmetic, no waits among
copies, no spills in the walks."""
import re

import pytest

import test_kernel_asm as K
from test_kernel_asm import device_asm  # noqa: F401

FILES = ["packed_fwd.hip", "packed_bwd.hip", "norm.hip"]


@pytest.fixture(scope="module", autouse=True)
def tower_sources():
    old, K.SOURCES = K.SOURCES, FILES
    yield
    K.SOURCES = old


def test_copies_and_arithmetic(device_asm):  # noqa: F811
    K.test_m0_is_set_only_by_the_lds_copies(device_asm)
    K.test_scalar_bases_of_the_lds_copies_are_settled(device_asm)
    K.test_no_packed_fp32_arithmetic(device_asm)
    # apart from the waits written for the purpose (all but the copies just issued)
    own = {fn: re.sub(r";;#ASMSTART\n\ts_waitcnt \w+\(\d+\)\n\t;;#ASMEND\n", "", text) for fn, text in device_asm.items()}
    assert own["packed_fwd.hip"] != device_asm["packed_fwd.hip"]
    K.test_no_vector_memory_wait_among_lds_copies(own)


@pytest.mark.parametrize("fn", FILES)
def test_no_vector_spills(device_asm, fn):  # noqa: F811
    found = re.findall(r"\.name:\s+(_Z\w+)\n(?:.*\n){0,40}?\s+\.vgpr_spill_count:\s+(\d+)", device_asm[fn])
    assert found and all(int(n) == 0 for _, n in found), [f for f in found if int(f[1])]
