"""The bounded waits of the sliding-window kernels, in the test-only build that loads nothing: every wait runs out, the calls
return, the status word says so, and the context stays usable for the product library."""
import ctypes

import pytest
import torch

from paper_2604_16429_b200 import binding as mb
from paper_2604_16429_b200 import build as mbuild
from tests import test_gpu_window as T

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("d", [64, 128])
def test_window_calls_time_out_cleanly(d):
    L = ctypes.CDLL(mbuild.build_wait_test())
    vp = ctypes.c_void_p
    L.mosaic_bsa_window_fwd.argtypes = [vp] * 9 + [ctypes.c_size_t, vp]
    L.mosaic_bsa_window_bwd.argtypes = [vp] * 13 + [ctypes.c_size_t, vp]
    L.mosaic_bsa_last_status.argtypes = [vp, vp]
    q, k, v, d_o = T.make(1, 2, 1, 200, 200, d, seed=1)
    wp = mb.WindowParams(window=50, sinks=2)
    p = ctypes.byref(mb._WindowParams(1, 2, 1, 200, 200, d, 50, 2, 0.0, 0))
    o, lse, dq, dk, dv = torch.zeros_like(q), torch.zeros(1, 2, 200, device="cuda"), torch.zeros_like(q), torch.zeros_like(k), torch.zeros_like(v)
    ws = torch.zeros(mb.window_workspace_bytes(wp, q, k, mb.OP_BWD), dtype=torch.uint8, device="cuda")
    at = lambda x: ctypes.byref(mb._View(x.data_ptr(), *x.stride()[:3]))  # noqa: E731
    s = torch.cuda.current_stream().cuda_stream
    assert L.mosaic_bsa_window_fwd(p, at(q), at(k), at(v), None, None, at(o), lse.data_ptr(), ws.data_ptr(), ws.numel(), s) == 0
    assert L.mosaic_bsa_last_status(ws.data_ptr(), s) == -16
    assert L.mosaic_bsa_window_bwd(p, at(q), at(k), at(v), at(o), lse.data_ptr(), at(d_o), None, None, at(dq), at(dk), at(dv), ws.data_ptr(),
                                   ws.numel(), s) == 0
    assert L.mosaic_bsa_last_status(ws.data_ptr(), s) == -16
    T.check_bwd(wp, q, k, v, d_o)
