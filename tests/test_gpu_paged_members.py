"""Batches of more members than a CTA of the paged attention has threads (352): the list of items is then found in rounds.  Tolerances:
those of tests/test_gpu_paged_decode.py."""
import os
import re

import pytest
import torch

from paper_2604_16429_b200 import binding as mb
from paper_2604_16429_b200 import build as mbuild
from tests.test_gpu_paged_decode import NAN, check, lens, make
from tests.test_gpu_prefix import check as check_prefix
from tests.test_gpu_prefix import with_prefix

pytestmark = pytest.mark.gpu
THREADS = 352
CASES = [  # B, H, Hkv, T, d, page, longest, window, sinks
    (353, 3, 1, 1, 64, 16, 70, 0, 0),
    (704, 2, 2, 1, 128, 16, 40, 0, 0),
    (705, 2, 1, 2, 64, 32, 90, 30, 1),
    (1100, 1, 1, 1, 64, 16, 600, 0, 0),     # parts that are joined
    (400, 2, 1, 3, 64, 16, 1500, 700, 2),
]


def lengths(B, T, longest):
    """Members of very different lengths, some without rows, some without tokens; the first and last of a round have work"""
    k_len = [(37 * i) % (longest + 1) if i % 9 else longest for i in range(B)]
    q_len = [(0 if i % 7 == 3 else 1 + i % T) for i in range(B)]
    for i in (0, THREADS - 1, THREADS, 2 * THREADS - 1, 2 * THREADS, B - 1):
        if i < B:
            k_len[i], q_len[i] = longest, T
    return k_len, q_len


def test_the_members_are_more_than_the_threads():
    text = open(os.path.join(mbuild.CSRC, "paged_decode.cu")).read()
    warps = int(re.search(r"kWarps = (\d+);  // that take steps", text)[1]) + int(re.search(r"kThreads = 32 \* \(kWarps \+ (\d+)\)", text)[1])
    assert 32 * warps <= THREADS, "more threads: these batches are then found in one round"


@pytest.mark.parametrize("case", CASES, ids=str)
def test_many_members(case):
    B, H, Hkv, T, d, page, longest, window, sinks = case
    width = -(-longest // page)
    q, kp, vp, table = make(B, H, Hkv, T, d, page, width, seed=B)
    k_len, q_len = lengths(B, T, longest)
    for b in range(B):
        q[b, :, q_len[b]:] = NAN
    o, lse = check(mb.PagedParams(window=window, sinks=sinks), q, kp, vp, table, k_len, q_len)
    at = [i for i in (0, THREADS - 1, THREADS, B - 1) if i < B]  # alone they have the same bits
    one = mb.mosaic_bsa_paged_decode(mb.PagedParams(window=window, sinks=sinks), q[at].contiguous(), kp, vp, table[at].contiguous(),
                                     lens([k_len[i] for i in at]), q_len=lens([q_len[i] for i in at]))
    assert torch.equal(one[0], o[at]) and torch.equal(one[1], lse[at])


@pytest.mark.parametrize("B,H,Hkv,d,longest", [(353, 2, 1, 64, 20), (720, 2, 2, 128, 40), (360, 4, 1, 64, 700)])
def test_many_members_behind_a_prefix(B, H, Hkv, d, longest):
    page, P = 16, 150
    q, kp, vp, table, prefix = with_prefix(B, H, Hkv, 1, d, page, -(-longest // page), P, seed=B)
    k_len, q_len = lengths(B, 1, longest)
    for b in range(B):
        q[b, :, q_len[b]:] = NAN
    check_prefix(mb.PagedParams(), q, kp, vp, table, k_len, prefix, P, q_len)
