"""What the binding makes of the paged cache's arguments before any launch, and its kernels' registers (no GPU needed)."""
import ast
import ctypes
import inspect
import os
import re
import subprocess
import sys

import pytest
import torch

from paper_2604_16429_b200 import binding as mb
from paper_2604_16429_b200 import build as mbuild
from tests.test_sequence_params_cpu import Tensor

NVCC = os.environ.get("NVCC", "/usr/local/cuda/bin/nvcc")
I32 = torch.int32
Q, POOL, LSE, WS = Tensor(2, 4, 3, 64), Tensor(50, 2, 16, 64), Tensor(2, 4, 3, dtype=torch.float32), Tensor(256, dtype=torch.uint8)
KV, TABLE, LEN, PREFIX = Tensor(2, 2, 3, 64), Tensor(2, 7, dtype=I32), Tensor(2, dtype=I32), Tensor(5, dtype=I32)


@pytest.fixture(scope="module", autouse=True)
def built():
    mbuild.build()


@pytest.fixture
def seen(monkeypatch):
    """The parameter blocks that would have reached the library"""
    out = []
    monkeypatch.setattr(mb, "_call", lambda name, index, stream, at, *a: out.append((name, mb._PagedParams.from_buffer_copy(
        (ctypes.c_char * ctypes.sizeof(mb._PagedParams)).from_address(at)), a)))
    return out


def decode(pp=mb.PagedParams(), **kw):
    a = {**dict(q=Q, k_pages=POOL, v_pages=POOL, table=TABLE, k_len=LEN, o=Q, lse=LSE, ws=WS), **kw}
    return mb.mosaic_bsa_paged_decode(pp, **a)


def prefix(pp=mb.PagedParams(), n=70, **kw):
    a = {**dict(q=Q, k_pages=POOL, v_pages=POOL, prefix_table=PREFIX, table=TABLE, k_len=LEN, o=Q, lse=LSE, ws=WS), **kw}
    return mb.mosaic_bsa_prefix_decode(pp, prefix_len=n, **a)


def append(rp=mb.RotaryParams(d=64), **kw):
    a = {**dict(k=KV, v=KV, k_pages=POOL, v_pages=POOL, table=TABLE, k_len=LEN, freqs=Tensor(rp.rot // 2, dtype=torch.float64)), **kw}
    return mb.mosaic_bsa_paged_append(rp, **a)


def test_sizes_come_from_the_tensors(seen):
    decode(mb.PagedParams(window=20, sinks=3, scale=0.5))
    name, p, _ = seen.pop()
    assert name == "mosaic_bsa_paged_decode"
    assert (p.B, p.H, p.Hkv, p.Nq, p.d, p.page, p.pages, p.width, p.table_stride) == (2, 4, 2, 3, 64, 16, 50, 7, 7)
    assert (p.window, p.sinks, p.scale, p.prefix_len, p.flags) == (20, 3, 0.5, 0, 0)
    prefix()
    assert seen.pop()[1].prefix_len == 70
    assert append(mb.RotaryParams(d=64, rot_dim=32, half=True, amplitude=2.0), start=1 << 40) is None
    _, p, a = seen.pop()
    assert (p.start, p.rot_dim, p.amplitude, p.flags, p.H, p.Nq) == (1 << 40, 32, 2.0, mb.FLAG_HALF_PAIRS, 0, 3) and a[-1] == a[-2] == 0
    assert append(q=Q, q_out=Q) is Q
    assert seen.pop()[1].H == 4


@pytest.mark.parametrize("window", [112, 113, 2 ** 31, sys.maxsize, 10 ** 30])
def test_any_window_beyond_the_pages_is_none(window, seen):
    decode(mb.PagedParams(window=window, sinks=3))
    assert seen[0][1].window == 0


@pytest.mark.parametrize("window", [-1, 1, 111])
def test_other_windows_are_passed_on_as_they_are(window, seen):
    decode(mb.PagedParams(window=window))
    assert seen[0][1].window == window


def test_numbers_that_no_field_holds_are_refused(seen):
    for pp in (mb.PagedParams(window=-2 ** 31 - 1), mb.PagedParams(sinks=2 ** 31), mb.PagedParams(scale=1e39)):
        with pytest.raises(ValueError, match="out of range"):
            decode(pp)
        with pytest.raises(ValueError, match="out of range"):
            prefix(pp)
        with pytest.raises(ValueError, match="out of range"):
            mb.paged_workspace_bytes(pp, Q, POOL, TABLE)
    with pytest.raises(ValueError, match="out of range"):
        append(start=1 << 63)
    with pytest.raises(ValueError, match="out of range"):
        append(mb.RotaryParams(d=64, amplitude=1e39))
    assert seen == []


def test_what_does_not_fit_is_refused(seen):
    f32, f16 = torch.float32, torch.float16
    for kw in (dict(q=Tensor(2, 4, 3, 64, dtype=f32)), dict(k_pages=Tensor(50, 2, 16, 64, dtype=f16)), dict(v_pages=Tensor(50, 2, 32, 64)),
               dict(v_pages=Tensor(49, 2, 16, 64)), dict(table=Tensor(3, 7, dtype=I32)), dict(table=Tensor(2, 7)),
               dict(table=Tensor(14, dtype=I32)), dict(k_len=Tensor(3, dtype=I32)), dict(k_len=Tensor(2, dtype=torch.int64)),
               dict(q_len=Tensor(3, dtype=I32)), dict(o=Tensor(2, 4, 3, 128)), dict(lse=Tensor(2, 4, 3)), dict(ws=Tensor(9)),
               dict(k_pages=Tensor(50, 2, 16, 32))):
        for call in (decode, prefix):
            with pytest.raises(ValueError):
                call(**kw)
    for kw in (dict(n=0), dict(n=-5), dict(n=81), dict(prefix_table=Tensor(2, 5, dtype=I32)), dict(prefix_table=Tensor(5, dtype=torch.int64))):
        with pytest.raises(ValueError):
            prefix(**kw)
    for kw in (dict(k=Tensor(2, 2, 3, 64, dtype=f32)), dict(v=Tensor(2, 2, 4, 64)), dict(k=Tensor(2, 3, 3, 64)), dict(q=Tensor(2, 4, 2, 64)),
               dict(q_out=Q), dict(freqs=Tensor(31, dtype=torch.float64)), dict(freqs=Tensor(32, dtype=f32)), dict(k_pages=Tensor(50, 2, 16, 128)),
               dict(table=Tensor(2, 7, dtype=torch.int64)), dict(k_len=Tensor(1, dtype=I32)), dict(q=Tensor(2, 4, 3, 64, dtype=f16))):
        with pytest.raises(ValueError):
            append(**kw)
    assert seen == []


@pytest.mark.parametrize("name", ["mosaic_bsa_paged_append", "mosaic_bsa_paged_decode", "mosaic_bsa_prefix_decode", "_paged_attention", "_paged_ws"])
def test_no_call_allocates_past_its_stream(name):
    tree = ast.parse(inspect.getsource(getattr(mb, name)))
    for call in (n for n in ast.walk(tree) if isinstance(n, ast.Call)):
        assert ast.unparse(call.func) not in ("torch.empty", "torch.empty_like", "torch.empty_strided"), ast.unparse(call)


def compiled(source, tmp_path):
    log = subprocess.run([NVCC, "-gencode", "arch=compute_100a,code=sm_100a", "-O3", "-std=c++17", "-lineinfo", "-Xptxas", "-v",
                          "-Xcompiler", "-fPIC", "-I", mbuild.INCLUDE, "-I", mbuild.CSRC, "-c", os.path.join(mbuild.CSRC, source),
                          "-o", str(tmp_path / "out.o")], check=True, capture_output=True, text=True).stderr
    return re.findall(r"Compiling entry function '(\w+)'.*?(\d+) bytes spill stores, (\d+) bytes spill loads.*?Used (\d+) registers", log, re.S)


# most bytes a thread may spill (stores, loads)
@pytest.mark.skipif(not os.path.exists(NVCC), reason="needs nvcc")
@pytest.mark.parametrize("source,stores,loads", [("paged_append.cu", 0, 0), ("paged_decode.cu", 8, 8), ("prefix_fwd.cu", 4, 16)])
def test_kernels_do_not_spill_more(source, stores, loads, tmp_path):
    found = compiled(source, tmp_path)
    assert len(found) >= 4
    for name, st, ld, regs in found:
        assert int(st) <= stores and int(ld) <= loads, (name, st, ld)
        if "prefix_fwd_kernel" in name:  # what its warpgroups share out anew
            assert int(regs) == 168, name
