"""Refusals, workspace sizes and registers of the sliding-window attention (no GPU needed)."""
import ctypes
import os
import re
import subprocess

import pytest

from paper_2604_16429_b200 import binding as mb
from paper_2604_16429_b200 import build as mbuild

NVCC = os.environ.get("NVCC", "/usr/local/cuda/bin/nvcc")
BASE = dict(B=2, H=4, Hkv=2, Nq=300, Nk=500, d=64, window=100, sinks=4, scale=0.0, flags=0)


@pytest.fixture(scope="module", autouse=True)
def built():
    mbuild.build()


def params(**kw):
    v = {**BASE, **kw}
    return ctypes.byref(mb._WindowParams(*(v[k] for k, _ in mb._WindowParams._fields_)))


def view(ptr=256, sb=1 << 20, sh=1 << 16, sn=64):
    return ctypes.byref(mb._View(ptr, sb, sh, sn))


def fwd(p=None, q=None, k=None, v=None, o=None, lse=256, ws=256, n=1 << 30, q_len=None, k_len=None):
    g = view()
    return mb.lib().mosaic_bsa_window_fwd(p or params(), q or g, k or g, v or g, q_len, k_len, o or g, lse, ws, n, None)


def bwd(p=None, x=None, at=0, lse=256, ws=256, n=1 << 30):
    vs = [view() for _ in range(8)]
    if x is not None:
        vs[at] = x
    q, k, v, o, d_o, dq, dk, dv = vs
    return mb.lib().mosaic_bsa_window_bwd(p or params(), q, k, v, o, lse, d_o, None, None, dq, dk, dv, ws, n, None)


def decode(p=None, q=None, k=None, lse=256, k_len=None):
    g = view()
    return mb.lib().mosaic_bsa_window_decode(p or params(Nq=1), q or g, k or g, g, k_len, g, lse, None)


@pytest.mark.parametrize("kw,code", [
    (dict(B=0), -1), (dict(H=3), -1), (dict(Hkv=0), -1), (dict(Nq=0), -1), (dict(Nk=-1), -1), (dict(window=0), -1), (dict(sinks=-1), -1),
    (dict(scale=float("nan")), -1), (dict(scale=float("inf")), -1), (dict(flags=1), -1), (dict(flags=4), -1), (dict(flags=64), -1),
    (dict(d=32), -2), (dict(d=256), -2), (dict(sinks=129), -2), (dict(Nk=1 << 30), -2),
])
def test_bad_params_are_refused(kw, code):
    assert fwd(params(**kw)) == code
    assert bwd(params(**kw)) == code
    if "Nq" not in kw:
        assert decode(params(Nq=1, **kw)) == code
    assert mb.lib().mosaic_bsa_window_workspace_bytes(params(**kw), mb.OP_FWD) == 0


def test_bad_tensors_are_refused():
    bad = [(view(0), -1), (view(256 + 8), -4), (view(sn=68), -4), (view(sh=4), -4), (view(sb=-64), -1), (view(sb=1 << 40), -2)]
    for x, code in bad:
        for at in ("q", "k", "v", "o"):
            assert fwd(**{at: x}) == code, at
        for at in range(8):
            assert bwd(x=x, at=at) == code, at
        assert decode(q=x) == code if x._obj.sn != 68 else True  # (one token: its stride is not looked at)
        assert decode(k=x) == code
    for at in ("q", "k", "v"):
        assert fwd(**{at: view(sn=0)}) == -2  # rows that all lie at one place
    assert mb.lib().mosaic_bsa_window_fwd(params(), None, view(), view(), None, None, view(), 256, 256, 256, None) == -1
    assert mb.lib().mosaic_bsa_window_fwd(None, view(), view(), view(), None, None, view(), 256, 256, 256, None) == -1


def test_bad_buffers_are_refused():
    assert fwd(lse=None) == -1 and fwd(ws=None) == -1 and fwd(lse=258) == -4 and fwd(ws=256 + 16) == -4 and fwd(n=255) == -3
    assert bwd(lse=None) == -1 and bwd(ws=None) == -1 and bwd(n=1 << 12) == -3
    assert fwd(q_len=258) == -4 and fwd(k_len=257) == -4 and decode(k_len=254) == -4 and decode(lse=None) == -1


def test_decode_takes_one_token_and_a_rolling_cache_holds_its_window():
    assert decode(params(Nq=2)) == -1
    assert decode(params(Nq=1, flags=mb.FLAG_ROLLING, window=497, sinks=4)) == -1     # 501 rows wanted, 500 there
    assert decode(params(Nq=1, flags=mb.FLAG_ROLLING, window=2 ** 31 - 1, sinks=4)) == -1
    assert fwd(params(flags=mb.FLAG_ROLLING)) == -1 and bwd(params(flags=mb.FLAG_ROLLING)) == -1


def test_workspaces():
    ws = mb.lib().mosaic_bsa_window_workspace_bytes
    assert ws(params(), mb.OP_FWD) == 256 and ws(params(), 7) == 0 and ws(params(), mb.OP_SELECT) == 0
    rows = 2 * 4 * 384 * 4  # [B, H, 384] fp32
    assert ws(params(window=500), mb.OP_BWD) == 256 + 2 * rows          # no row beyond the first tile's list
    assert ws(params(sinks=0), mb.OP_BWD) == 256 + 2 * rows
    assert ws(params(), mb.OP_BWD) > 256 + 2 * rows


@pytest.mark.skipif(not os.path.exists(NVCC), reason="needs nvcc")
@pytest.mark.parametrize("source,want", [("window_fwd.cu", {168}), ("window_bwd.cu", {128, 168})])
def test_kernels_are_launched_with_the_registers_that_they_share_out(source, want, tmp_path):
    """The warpgroups of these kernels raise and lower their registers; the sum of their shares is the launch's, and a launch with
    fewer would wait for good (the library refuses to)."""
    log = subprocess.run([NVCC, "-gencode", "arch=compute_100a,code=sm_100a", "-O3", "-std=c++17", "-lineinfo", "-Xptxas", "-v",
                          "-Xcompiler", "-fPIC", "-I", mbuild.INCLUDE, "-I", mbuild.CSRC, "-c", os.path.join(mbuild.CSRC, source),
                          "-o", str(tmp_path / "out.o")], check=True, capture_output=True, text=True).stderr
    found = re.findall(r"Compiling entry function '(\w+)'.*?Used (\d+) registers", log, re.S)
    used = {n: int(r) for n, r in found if "window_fwd_kernel" in n or "window_bwd_kernel" in n}
    assert len(used) >= 4 and set(used.values()) == want, used
    for name, regs in used.items():
        if "window_bwd_kernel" in name:
            assert regs == (168 if "Li128ELb0ELb1" in name or "Li128ELb1ELb1" in name else 128), name
