"""Spills of the sequence operators' kernels, as the compiler reports them (no GPU needed): their row threads hold a row's scores or two,
at the edge of their registers."""
import os
import re
import subprocess

import pytest

from paper_2604_16429_b200 import build as mbuild

NVCC = os.environ.get("NVCC", "/usr/local/cuda/bin/nvcc")

# most bytes a thread may spill (stores, loads), by what the kernel's mangled name holds; the first that fits
LIMITS = {
    "window_fwd.cu": [("window_fwd_kernel", 4, 20)],
    "window_bwd.cu": [("window_bwd_kernelILi64ELb0ELb1E", 84, 136),   # d = 64, bf16, key-stationary: the second product's operands
                      ("window_bwd_kernelILi64ELb1ELb1E", 28, 64), ("window_bwd_kernel", 12, 32), ("", 0, 0)],
    "window_decode.cu": [("", 0, 0)],
    "rotary.cu": [("", 0, 0)],
}


@pytest.mark.skipif(not os.path.exists(NVCC), reason="needs nvcc")
@pytest.mark.parametrize("source", sorted(LIMITS))
def test_kernels_of_the_sequence_operators_do_not_spill_more(source, tmp_path):
    log = subprocess.run([NVCC, "-gencode", "arch=compute_100a,code=sm_100a", "-O3", "-std=c++17", "-lineinfo", "-Xptxas", "-v",
                          "-Xcompiler", "-fPIC", "-I", mbuild.INCLUDE, "-I", mbuild.CSRC, "-c", os.path.join(mbuild.CSRC, source),
                          "-o", str(tmp_path / "out.o")], check=True, capture_output=True, text=True).stderr
    found = re.findall(r"Compiling entry function '(\w+)'.*?(\d+) bytes spill stores, (\d+) bytes spill loads", log, re.S)
    assert len(found) >= 4, log
    for name, stores, loads in found:
        most = next(x for x in LIMITS[source] if x[0] in name)
        assert int(stores) <= most[1] and int(loads) <= most[2], (name, stores, loads)
