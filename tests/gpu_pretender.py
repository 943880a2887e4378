"""A pytest plugin for machines without a GPU: tests run as if one were there, and fail where a call of the library would go on to it.

Refusals are tested with addresses that are none. Where there is no GPU, a call that passes all checks of its arguments ends with
VC_ERR_DEVICE; where there is one it launches, and reads and writes those addresses."""
import torch

import paper_2501_08453_amd as vc

VC_ERR_DEVICE = -6


class _Watched:
    def __init__(self, name, f):
        self.name, self.f = name, f

    def __call__(self, *args):
        st = self.f(*args)
        if st == VC_ERR_DEVICE:
            raise RuntimeError("%s would reach the GPU" % self.name)
        return st


def pytest_configure(config):
    if torch.cuda.is_available():
        raise RuntimeError("for machines without a GPU")
    torch.cuda.is_available = lambda: True
    lib = vc._lib()
    for name, (restype, _) in vc._SIGS.items():
        if name.startswith("vc_") and restype is not None:
            setattr(lib, name, _Watched(name, getattr(lib, name)))
