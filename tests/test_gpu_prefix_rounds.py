"""Behind a prefix of more parts than a row's lanes, the kernel of the members' own keys joins them in rounds of d / 4 parts, with a maximum
that moves from round to round, against the definition in 64 bits.  Tolerances: those of tests/test_gpu_prefix.py."""
import pytest
import torch

from paper_2604_16429_b200 import binding as mb
from tests.test_gpu_prefix import check, with_prefix

pytestmark = pytest.mark.gpu
CASES = [  # B, H, Hkv, T, d, page, P, k_len
    (3, 12, 3, 1, 64, 16, 1300, [3, 20, 0]),          # 21 parts: two rounds of 16
    (3, 12, 3, 1, 64, 32, 2500, [3, 20, 33]),         # 40: three rounds
    (2, 8, 4, 2, 64, 16, 2100, [2, 70]),
    (2, 8, 4, 1, 128, 16, 2300, [1, 100]),            # 36 and 40: two rounds of 32
    (3, 6, 3, 1, 128, 64, 2560, [0, 64, 7]),
]


def parts_of(q, kp, d, P):
    """(parts of the prefix, results come from the kernel that makes the own parts), from the workspaces"""
    B, H, T, _ = q.shape
    page, rows = kp.shape[2], q.shape[0] * q.shape[1] * q.shape[2]

    def parts(width):
        n = mb.paged_workspace_bytes(mb.PagedParams(), q, kp, torch.zeros((B, width), dtype=torch.int32, device="cuda"), P)
        return (n - 256) // (rows * (d * 4 + 8))

    shared = parts(-(-1024 // page)) - 2  # two own parts, which are joined apart
    return shared, parts(1) == shared


@pytest.mark.parametrize("scores", ["rising", "falling", "flat", "own", "holes", "all holes"])
@pytest.mark.parametrize("case", CASES, ids=str)
def test_parts_in_rounds(case, scores):
    B, H, Hkv, T, d, page, P, k_len = case
    q, kp, vp, table, prefix = with_prefix(B, H, Hkv, T, d, page, max(1, -(-max(k_len) // page)), P, seed=P, sharp=3.0)
    shared, direct = parts_of(q, kp, d, P)
    assert direct and d // 4 < shared <= 40, "not the join in rounds"
    n = len(prefix)
    if scores in ("rising", "falling"):  # the largest scores in the last parts, or in the first
        ramp = torch.linspace(0.1, 5, n, device="cuda")
        kp[prefix.long()] *= (ramp if scores == "rising" else ramp.flip(0)).to(kp.dtype)[:, None, None, None]
    elif scores == "own":  # or in the member's own keys
        kp[table.long().flatten()] *= 4
        kp[prefix.long()] *= 0.25
    elif scores == "holes":  # the whole first round, and some pages more
        prefix[:-(-(d // 4) * 64 // page)] = -1
        prefix[-2] = kp.shape[0]
    elif scores == "all holes":
        prefix[:] = -1
    check(mb.PagedParams(), q, kp, vp, table, k_len, prefix, P)


def test_a_value_in_the_last_round_counts():
    """A key of the last part that outweighs all others: its value is the result."""
    B, H, Hkv, T, d, page, P, k_len = CASES[1]
    q, kp, vp, table, prefix = with_prefix(B, H, Hkv, T, d, page, 2, P, seed=1)
    q[:] = 1
    kp[prefix.long()] *= 0.1
    at = P - 1
    kp[prefix[at // page], :, at % page] = 8
    o, _ = check(mb.PagedParams(), q, kp, vp, table, [3, 20, 33], prefix, P)
    want = vp[prefix[at // page], :, at % page].repeat_interleave(H // Hkv, 0)
    assert torch.equal(o[:, :, 0], want.expand(B, H, d))
