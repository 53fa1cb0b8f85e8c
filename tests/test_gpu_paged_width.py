"""A member's bits do not depend on how many pages its table has room for, only on its own tokens."""
import pytest
import torch

from paper_2604_16429_b200 import binding as mb
from tests.test_gpu_paged_decode import lens, make
from tests.test_gpu_prefix import with_prefix

pytestmark = pytest.mark.gpu
CAPACITIES = (512, 4096, 4608, 8192, 8704, 32768, 33280, 70000)  # either side of 8, 16 and 64 chunks of 512


def widened(table, width):
    out = torch.full((table.shape[0], width), -1, dtype=torch.int32, device="cuda")
    out[:, :table.shape[1]] = table
    return out


@pytest.mark.parametrize("H,Hkv,T,d,dtype", [(8, 2, 1, 128, "bf16"), (6, 3, 2, 64, "fp16"), (32, 4, 16, 64, "fp16"), (32, 2, 8, 128, "fp16")])
@pytest.mark.parametrize("k_len", [[512, 3], [4000, 513], [8192, 4097], [9000, 30000], [33000, 5000]], ids=str)
def test_paged_attention(H, Hkv, T, d, dtype, k_len):
    page = 64
    q, kp, vp, table = make(2, H, Hkv, T, d, page, -(-max(k_len) // page), dtype, seed=d)
    got = [mb.mosaic_bsa_paged_decode(mb.PagedParams(), q, kp, vp, widened(table, -(-n // page)), lens(k_len)) for n in CAPACITIES if n >= max(k_len)]
    assert got
    for o, lse in got[1:]:
        assert torch.equal(o, got[0][0]) and torch.equal(lse, got[0][1])


@pytest.mark.parametrize("P", [500, 5000, 30000])
@pytest.mark.parametrize("k_len", [[0, 3, 700], [4000, 513, 8000]], ids=str)
def test_behind_a_prefix(P, k_len):
    """(From two own parts on: one part alone may be joined by the kernel that makes it, in another order.)"""
    page, H, Hkv, d = 32, 8, 2, 64
    q, kp, vp, table, prefix = with_prefix(3, H, Hkv, 1, d, page, -(-max(k_len) // page), P, seed=P)
    got = [mb.mosaic_bsa_prefix_decode(mb.PagedParams(), q, kp, vp, prefix, P, widened(table, -(-n // page)), lens(k_len))
           for n in (1024,) + CAPACITIES[1:] if n >= max(k_len)]
    for o, lse in got[1:]:
        assert torch.equal(o, got[0][0]) and torch.equal(lse, got[0][1])
