"""The bounded waits of the paged cache's attention, in the test-only build that loads nothing: every wait runs out, the calls return, the
status word says so, and the context stays usable for the product library."""
import ctypes

import pytest
import torch

from paper_2604_16429_b200 import binding as mb
from paper_2604_16429_b200 import build as mbuild
from tests import test_gpu_prefix as P

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("T", [1, 3])
def test_paged_calls_time_out_cleanly(d, T):
    L = ctypes.CDLL(mbuild.build_wait_test())
    vp = ctypes.c_void_p
    L.mosaic_bsa_paged_decode.argtypes = [vp] * 10 + [ctypes.c_size_t, vp]
    L.mosaic_bsa_prefix_decode.argtypes = [vp] * 11 + [ctypes.c_size_t, vp]
    L.mosaic_bsa_last_status.argtypes = [vp, vp]
    B, H, Hkv, page, width, n = 3, 8, 2, 16, 40, 200
    q, k, v, table, prefix = P.with_prefix(B, H, Hkv, T, d, page, width, n, seed=1)
    k_len = P.lens([600, 30, 3])
    o, lse = torch.zeros_like(q), torch.zeros(B, H, T, device="cuda")
    at = lambda x: ctypes.byref(mb._View(x.data_ptr(), *x.stride()[:3]))  # noqa: E731
    s = torch.cuda.current_stream().cuda_stream
    for shared in (0, n):
        ws = torch.zeros(mb.paged_workspace_bytes(mb.PagedParams(), q, k, table, shared), dtype=torch.uint8, device="cuda")
        p = ctypes.byref(mb._PagedParams(width, 0, B, H, Hkv, T, d, page, k.shape[0], width, 0, 0, shared, 0, 0.0, 0.0, 0))
        tables = (prefix.data_ptr(), table.data_ptr()) if shared else (table.data_ptr(),)
        call = L.mosaic_bsa_prefix_decode if shared else L.mosaic_bsa_paged_decode
        assert call(p, at(q), at(k), at(v), *tables, k_len.data_ptr(), None, at(o), lse.data_ptr(), ws.data_ptr(), ws.numel(), s) == 0
        assert L.mosaic_bsa_last_status(ws.data_ptr(), s) == -16
    P.check(mb.PagedParams(), q, k, v, table, [600, 30, 3], prefix, n)
