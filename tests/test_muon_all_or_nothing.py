"""moe_muon makes all of its launches before it launches the first: where the device can not run one of them (here there is none), nothing of the step has been launched, and no momentum has taken a step
that its weights have not."""
import ctypes

import pytest
import torch

from paper_1701_06538_b200 import binding as B
from paper_1701_06538_b200 import build as moe_build


@pytest.mark.skipif(torch.cuda.is_available(), reason="of a machine without a device")
@pytest.mark.parametrize("shapes", [((2, 264, 200),), ((1, 16, 4096),), ((3, 64, 128),), ((3, 64, 128), (4, 264, 200), (1, 16, 4096)), tuple((1, 256 + 8 * i, 300) for i in range(9))], ids=str)
def test_nothing_is_launched(shapes):
    moe_build.build()
    lib = B.lib()
    at = lambda i: (1 << 30) + (i << 24)
    tensors = (B.moe_muon_tensor * len(shapes))(*[B.moe_muon_tensor(at(3 * i), at(3 * i + 1), None, at(3 * i + 2), *shape, 0, 0, 0, 0.0, 1.0) for i, shape in enumerate(shapes)])
    params = B.moe_muon_params(1e-3, 0.95, 1e-7, 1.0, 5, 1)
    before = B.moe_debug_launch_count()
    status = lib.moe_muon(tensors, ctypes.c_int32(len(shapes)), ctypes.byref(params), None, ctypes.c_void_p(1 << 20), None)
    assert status != 0 and B.moe_debug_launch_count() == before
