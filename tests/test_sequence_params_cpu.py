"""What the binding makes of parameters at and beyond the ends of their ranges (no GPU needed: the tensors are stand-ins and no entry
point that would launch is reached)."""
import ctypes
import math
import sys

import pytest
import torch

from paper_2604_16429_b200 import binding as mb
from paper_2604_16429_b200 import build as mbuild


@pytest.fixture(scope="module", autouse=True)
def built():
    mbuild.build()


class Tensor:
    """What the checks before a launch look at of a tensor on the device"""

    def __init__(self, *shape, dtype=torch.bfloat16):
        self.dtype, self.device, self.shape = dtype, "cuda:0", torch.Size(shape)
        self.strides = torch.empty(shape, device="meta").stride()

    def dim(self): return len(self.shape)
    def get_device(self): return 0
    def stride(self, i=None): return self.strides if i is None else self.strides[i]
    def is_contiguous(self): return True
    def data_ptr(self): return 256
    def numel(self): return 1 << 30


Q, K, LSE, WS = Tensor(1, 2, 1, 64), Tensor(1, 2, 500, 64), Tensor(1, 2, 1, dtype=torch.float32), Tensor(256, dtype=torch.uint8)


def window_calls(wp):
    yield lambda: mb.mosaic_bsa_window_fwd(wp, Q, K, K, o=Q, lse=LSE, ws=WS)
    yield lambda: mb.mosaic_bsa_window_bwd(wp, Q, K, K, Q, LSE, Q, dq=Q, dk=K, dv=K, ws=WS)
    yield lambda: mb.mosaic_bsa_window_decode(wp, Q, K, K, o=Q, lse=LSE)


@pytest.fixture
def seen(monkeypatch):
    """The parameter blocks that would have reached the library"""
    out = []
    monkeypatch.setattr(mb, "_call", lambda name, index, stream, at, *a: out.append(mb._WindowParams.from_buffer_copy(
        (ctypes.c_char * ctypes.sizeof(mb._WindowParams)).from_address(at))))
    return out


@pytest.mark.parametrize("window", [500, 501, 2 ** 31 - 1, 2 ** 31, sys.maxsize, 10 ** 30])
def test_any_window_beyond_the_keys_is_plain_causal(window, seen):
    wp = mb.WindowParams(window=window, sinks=3)
    for call in window_calls(wp):
        call()
    assert [p.window for p in seen] == [500] * 3 and all(p.sinks == 3 and p.Nk == 500 for p in seen)
    for op in (mb.OP_FWD, mb.OP_BWD):
        assert mb.window_workspace_bytes(wp, Q, K, op) == mb.window_workspace_bytes(mb.WindowParams(window=500, sinks=3), Q, K, op) > 0


@pytest.mark.parametrize("window", [-1, 0, 1, 499])
def test_other_windows_are_passed_on_as_they_are(window, seen):
    for call in window_calls(mb.WindowParams(window=window)):
        call()
    assert [p.window for p in seen] == [window] * 3


@pytest.mark.parametrize("kw", [dict(window=sys.maxsize, rolling=True), dict(window=-2 ** 31 - 1), dict(window=10, sinks=2 ** 31),
                                dict(window=10, sinks=2 ** 32 + 4), dict(window=10, scale=1e39)])
def test_numbers_that_no_field_holds_are_refused(kw, seen):
    wp = mb.WindowParams(**kw)
    for call in window_calls(wp):
        with pytest.raises(ValueError, match="out of range"):
            call()
    with pytest.raises(ValueError, match="out of range"):
        mb.window_workspace_bytes(wp, Q, K, mb.OP_BWD)
    assert seen == []


@pytest.mark.parametrize("kw,eps", [(dict(amplitude=1e39), 1e-6), (dict(), 1e300)])
def test_numbers_that_no_field_of_the_rotation_holds_are_refused(kw, eps, seen):
    rp = mb.RotaryParams(d=64, rot_dim=0, **kw)
    w = Tensor(64, dtype=torch.float32)
    with pytest.raises(ValueError, match="out of range"):
        mb.mosaic_bsa_qk_norm(rp, Q, Q, w, w, eps=eps, q_out=Q, k_out=Q)
    with pytest.raises(ValueError, match="out of range"):
        mb.mosaic_bsa_qk_norm_bwd(rp, Q, Q, w, w, None, None, Q, Q, eps=eps, dq=Q, dk=Q, dwq=w, dwk=w, ws=WS)
    if not kw:
        return
    pos, freqs = Tensor(1, dtype=torch.int64), Tensor(32, dtype=torch.float64)
    with pytest.raises(ValueError, match="out of range"):
        mb.mosaic_bsa_rotary(mb.RotaryParams(d=64, **kw), Q, Q, pos, freqs, q_out=Q, k_out=Q)
    with pytest.raises(ValueError, match="out of range"):
        mb.qk_norm_workspace_bytes(rp, Q, Q)
    assert math.isinf(ctypes.c_float(1e39).value) and seen == []
