"""Frequencies of the rotary positions against their definitions, and the refusals of the rotation and norm entry points
(no GPU needed: arguments are rejected before the device is touched)."""
import ctypes
import math

import numpy as np
import pytest

from paper_2604_16429_b200 import binding as mb
from paper_2604_16429_b200 import build as mbuild


@pytest.fixture(scope="module", autouse=True)
def built():
    mbuild.build()


def _f(**kw):
    return mb.rotary_freqs(mb.RotaryParams(**{**dict(d=256), **kw}), device="cpu").numpy()


@pytest.mark.parametrize("rot", [2, 16, 50, 128, 256])
def test_plain_linear_and_base(rot):
    i = np.arange(rot // 2)
    want = np.exp(-2.0 * i / rot * math.log(10000.0))
    # pow and exp/log in fp64: the exponent's own rounding, at most 9.3 * 2^-53, and a few ulp
    assert np.abs(_f(rot_dim=rot) / want - 1).max() < 1e-14
    assert np.abs(_f(rot_dim=rot, scaling=mb.ROTARY_LINEAR, factor=4.0) * 4 / want - 1).max() < 1e-14
    base = _f(rot_dim=rot, scaling=mb.ROTARY_BASE, factor=8.0)
    assert base[0] == 1.0 or rot == 2
    if rot > 2:  # the fastest pair keeps its speed, the slowest is slowed by the factor
        assert abs(base[-1] * 8.0 / want[-1] - 1) < 1e-13


def test_parts_ramps_over_the_pairs():
    rot, L, factor, fast, slow = 128, 8192.0, 8.0, 32.0, 1.0
    plain = _f(rot_dim=rot)
    got = _f(rot_dim=rot, scaling=mb.ROTARY_PARTS, factor=factor, length=L, fast=fast, slow=slow)
    turns = L * plain / (2 * math.pi)
    lo = np.nonzero(turns >= fast)[0].max()   # the last pair that still turns `fast` times
    hi = np.nonzero(turns >= slow)[0].max() + 1
    want = [p if i <= lo else p / factor if i >= hi else p * (1 - (i - lo) / (hi - lo)) + p / factor * (i - lo) / (hi - lo)
            for i, p in enumerate(plain)]
    assert np.abs(got / np.array(want) - 1).max() < 1e-13
    assert got[0] == plain[0] and abs(got[-1] * factor / plain[-1] - 1) < 1e-15


def test_bands_ramp_over_the_turns():
    rot, L, factor, fast, slow = 64, 8192.0, 4.0, 4.0, 1.0
    plain = _f(rot_dim=rot)
    got = _f(rot_dim=rot, scaling=mb.ROTARY_BANDS, factor=factor, length=L, fast=fast, slow=slow)
    for p, g in zip(plain, got):
        turns = L * p / (2 * math.pi)
        if turns > fast:
            assert g == p
        elif turns < slow:
            assert abs(g * factor / p - 1) < 1e-15
        else:
            t = (turns - slow) / (fast - slow)
            assert abs(g / ((1 - t) * p / factor + t * p) - 1) < 1e-13


@pytest.mark.parametrize("kw", [
    dict(rot_dim=3), dict(rot_dim=0), dict(theta=1.0), dict(theta=float("nan")), dict(theta=float("inf")), dict(scaling=5),
    dict(scaling=-1), dict(scaling=1, factor=0.5), dict(scaling=2, factor=float("nan")), dict(scaling=3, factor=2.0),
    dict(scaling=3, factor=2.0, length=100.0, fast=1.0, slow=1.0), dict(scaling=4, factor=2.0, length=100.0, slow=0.0),
    dict(scaling=4, factor=2.0, length=float("inf")),
])
def test_bad_scalings_are_refused(kw):
    with pytest.raises(mb.MosaicError) as e:
        _f(**kw)
    assert e.value.code == -1


def _call(name="rotary", ptr=256, strides=(64 * 8, 64, 64 * 4), pos_stride=0, ws=1 << 24, **kw):
    base = dict(B=1, H=4, Hkv=2, N=2, d=64, rot_dim=64, flags=0, amplitude=1.0, eps=1e-6)
    base.update(kw)
    p = ctypes.byref(mb._RotaryParams(*(base[k] for k, _ in mb._RotaryParams._fields_)))
    L = mb.lib()
    v = ctypes.byref(mb._View(ptr, *strides))
    good = ctypes.byref(mb._View(256, 64 * 8, 64, 64 * 4))
    if name == "rotary":
        return L.mosaic_bsa_rotary(p, v, good, 256, pos_stride, 256, good, good, None)
    if name == "norm":
        return L.mosaic_bsa_qk_norm(p, good, v, 256, 256, 256, pos_stride, 256, good, good, None)
    return L.mosaic_bsa_qk_norm_bwd(p, good, good, 256, 256, 256, pos_stride, 256, good, good, v, good, 256, 256, 256, ws, None)


@pytest.mark.parametrize("name", ["rotary", "norm", "bwd"])
@pytest.mark.parametrize("kw,code", [
    (dict(B=0), -1), (dict(N=0), -1), (dict(Hkv=3), -1), (dict(H=0), -1),
    (dict(rot_dim=66), -1), (dict(rot_dim=7), -1), (dict(rot_dim=-2), -1),
    (dict(flags=2 | 4), -1), (dict(flags=1), -1), (dict(flags=64), -1),
    (dict(amplitude=-1.0), -1), (dict(amplitude=float("inf")), -1),
    (dict(d=72, rot_dim=64), -2), (dict(d=272, rot_dim=64), -2), (dict(flags=8, rot_dim=24), -2),
    (dict(ptr=0), -1), (dict(ptr=256 + 8), -4), (dict(strides=(-64, 64, 256)), -1), (dict(strides=(512, 66, 256)), -4),
    (dict(strides=(512, 64, 68)), -4), (dict(pos_stride=-1), -1),
])
def test_bad_arguments_are_refused(name, kw, code):
    assert _call(name, **kw) == code


def test_what_only_one_entry_point_refuses():
    assert _call("rotary", rot_dim=0) == -1               # nothing to do
    assert _call("norm", flags=16) == -1                  # a norm has no inverse
    assert _call("norm", eps=-1.0) == -1
    assert _call("norm", eps=float("nan")) == -1
    assert _call("bwd", ws=16) == -3
    assert mb.lib().mosaic_bsa_rotary(None, None, None, None, 0, None, None, None, None) == -1
    p = ctypes.byref(mb._RotaryParams(1, 4, 2, 2, 64, 64, 0, 1.0, 1e-6))
    v = ctypes.byref(mb._View(256, 512, 64, 256))
    assert mb.lib().mosaic_bsa_rotary(p, v, v, None, 0, 256, v, v, None) == -1
    assert mb.lib().mosaic_bsa_rotary(p, v, v, 256, 0, 256 + 4, v, v, None) == -4
    assert mb.lib().mosaic_bsa_rotary(p, v, None, 256, 0, 256, v, v, None) == -1
    assert mb.lib().mosaic_bsa_qk_norm_workspace_bytes(ctypes.byref(mb._RotaryParams(1, 4, 3, 2, 64, 64, 0, 1.0, 1e-6))) == 0
    assert mb.lib().mosaic_bsa_qk_norm_workspace_bytes(p) % 256 == 0


def test_host_tensors_are_refused():
    import torch
    rp = mb.RotaryParams(d=64)
    x = torch.zeros(1, 2, 3, 64)
    with pytest.raises(ValueError):
        mb.mosaic_bsa_rotary(rp, x, x, torch.arange(3), mb.rotary_freqs(rp, "cpu"))
