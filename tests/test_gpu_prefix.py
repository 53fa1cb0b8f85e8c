"""Attention of a batch behind a shared prefix against the definition in 64 bits.

Tolerances: those of the attention over a paged cache (tests/test_gpu_paged_decode.py).  Within a part of the prefix a row's sum of weights
takes 18 additions a step of 64 keys, rounded to 2^-24 each, and its weighted sums one of at most 2^-23 per 16 keys; the parts here have
1500 keys at most, so both stay below the (32 + 64) 2^-23 that the bound holds for a row's sums."""
import math

import pytest
import torch

from paper_2604_16429_b200 import binding as mb
from tests import gpu_util as G
from tests import paged_ref as ref
from tests.test_gpu_paged_decode import NAN, compare, lens, make, spoil

pytestmark = pytest.mark.gpu


def with_prefix(B, H, Hkv, T, d, page, width, P, dtype="bf16", layout="bhnd", pages="hpd", seed=0, sharp=1.0):
    """q, pools, table of the members' own pages, prefix table"""
    held = -(-P // page)
    q, kp, vp, table = make(B, H, Hkv, T, d, page, width, dtype, layout, pages, extra=held + 2, seed=seed, sharp=sharp)
    free = sorted(set(range(kp.shape[0])) - set(table.flatten().tolist()))
    g = torch.Generator().manual_seed(seed + 1)
    prefix = torch.tensor(free, dtype=torch.int32)[torch.randperm(len(free), generator=g)[:held]].cuda()
    return q, kp, vp, table, prefix


def check(pp, q, kp, vp, table, k_len, prefix, P, q_len=None, finite=None):
    clean = finite or (kp, vp)
    want = ref.attention(q, *clean, table, k_len, 0, 0, pp.scale, q_len, prefix, P)
    o, lse = G.Guarded(tuple(q.shape), q.dtype, fill=NAN), G.Guarded(tuple(q.shape[:3]), torch.float32, fill=NAN)
    ws = G.Guarded((mb.paged_workspace_bytes(pp, q, kp, table, P),), torch.uint8)
    mb.mosaic_bsa_prefix_decode(pp, q, kp, vp, prefix, P, table, lens(k_len), q_len=lens(q_len), o=o.t, lse=lse.t, ws=ws.t)
    mb.check_status(ws.t, "prefix_decode")
    for x, name in ((o, "o"), (lse, "lse"), (ws, "workspace")):
        x.check(name)
    compare(want, o.t, lse.t, q, clean[0], pp.scale, table.shape[1] * kp.shape[2] + P)
    return o.t, lse.t


CASES = [  # B, H, Hkv, T, d, page, P, k_len, q_len
    (1, 1, 1, 1, 64, 16, 1, [1], None),
    (1, 2, 1, 1, 128, 16, 64, [0], None),
    (2, 4, 2, 1, 64, 32, 100, [3, 40], None),
    (3, 16, 2, 1, 128, 64, 1000, [0, 1, 700], None),
    (5, 6, 6, 1, 64, 256, 2049, [9, 8, 7, 6, 600], None),
    (40, 8, 2, 1, 128, 16, 777, [i % 19 for i in range(40)], None),          # 160 rows: a tile and a quarter
    (70, 4, 1, 1, 64, 32, 333, [i % 37 for i in range(70)], None),           # 280 rows: the second pair has 24
    (4, 12, 3, 5, 64, 16, 500, [5, 50, 3, 0], [5, 2, 5, 3]),                 # drafts, more new tokens than tokens
    (9, 34, 2, 16, 128, 128, 4100, [16 + i for i in range(9)], None),        # 2448 rows
    (130, 2, 2, 1, 64, 512, 65, [1] * 130, [i % 2 for i in range(130)]),     # every other member has no rows
    (150, 2, 2, 1, 64, 16, 4000, [i % 50 for i in range(150)], None),        # one part each, but many items a CTA: joined apart
    (80, 8, 4, 2, 128, 32, 2500, [2 + i % 90 for i in range(80)], None),
]


@pytest.mark.parametrize("case", CASES, ids=lambda c: str(c)[:60])
@pytest.mark.parametrize("dtype,layout,pages", [("bf16", "bhnd", "phd"), ("fp16", "bnhd", "hpd")])
def test_prefix(case, dtype, layout, pages):
    B, H, Hkv, T, d, page, P, k_len, q_len = case
    width = max(1, -(-max(k_len) // page)) + 1
    q, kp, vp, table, prefix = with_prefix(B, H, Hkv, T, d, page, width, P, dtype, layout, pages, seed=P)
    clean = kp.clone(), vp.clone()
    both = torch.full((B + 1, max(width, len(prefix))), -1, dtype=torch.int32)
    both[:B, :width], both[B, :len(prefix)] = table.cpu(), prefix.cpu()
    spoil((kp, vp), both, list(k_len) + [P], page)  # what no row sees
    if q_len:
        for b in range(B):
            q[b, :, q_len[b]:] = NAN
    o, lse = check(mb.PagedParams(), q, kp, vp, table, k_len, prefix, P, q_len, clean)
    again = mb.mosaic_bsa_prefix_decode(mb.PagedParams(), q, kp, vp, prefix, P, table, lens(k_len), q_len=lens(q_len))
    same = ~torch.isnan(lse)
    assert torch.equal(again[0][same], o[same]) and torch.equal(again[1][same], lse[same])
    if B > 1:  # a member's bits depend neither on what the others hold nor on its place
        order = torch.arange(B - 1, -1, -1)
        turned = mb.mosaic_bsa_prefix_decode(mb.PagedParams(), q[order.cuda()], kp, vp, prefix, P, table[order.cuda()].contiguous(),
                                             lens([k_len[i] for i in order]), q_len=lens([q_len[i] for i in order]) if q_len else None)
        assert torch.equal(turned[0][order.cuda()][same], o[same]) and torch.equal(turned[1][order.cuda()][same], lse[same])


@pytest.mark.parametrize("page,holes", [(16, [0]), (16, [1, 5, 6, 7, 20]), (64, [2]), (32, list(range(100))), (256, [1])])
@pytest.mark.parametrize("d", [64, 128])
def test_prefix_pages_that_are_not_there_are_not_seen(page, holes, d):
    P = 700
    q, kp, vp, table, prefix = with_prefix(3, 4, 2, 1, d, page, 3, P, seed=page)
    for i, h in enumerate(holes):
        if h < len(prefix):
            prefix[h] = (-1, 2 ** 31 - 1, kp.shape[0], -(2 ** 31))[i % 4]
    check(mb.PagedParams(), q, kp, vp, table, [0, 5, 17], prefix, P)


def test_sharp_scores_and_scale():
    """Maxima that move all along the prefix."""
    q, kp, vp, table, prefix = with_prefix(20, 8, 1, 1, 64, 16, 2, 3000, seed=3, sharp=8.0)
    ramp = torch.linspace(0.1, 6, -(-3000 // 16), device="cuda").bfloat16()
    kp[prefix.long()] *= ramp[:, None, None, None]
    for scale in (0.0, 0.5):
        check(mb.PagedParams(scale=scale), q, kp, vp, table, [3] * 20, prefix, 3000)


def test_it_is_the_same_as_copies_of_the_prefix():
    """Behind a prefix, and with the prefix' pages at the head of every member's table."""
    B, H, Hkv, d, page, P = 6, 8, 2, 128, 32, 1024
    q, kp, vp, table, prefix = with_prefix(B, H, Hkv, 1, d, page, 4, P, seed=9)
    k_len = [1, 128, 60, 33, 32, 31]
    a = check(mb.PagedParams(), q, kp, vp, table, k_len, prefix, P)
    whole = torch.cat((prefix.expand(B, -1), table), 1).contiguous()
    want = ref.attention(q, kp, vp, table, k_len, 0, 0, 0.0, None, prefix, P)
    b = mb.mosaic_bsa_paged_decode(mb.PagedParams(), q, kp, vp, whole, lens([P + n for n in k_len]))
    compare(want, *b, q, kp, 0.0, P + 128)
    assert (a[0].double() - b[0].double()).abs().max() < 0.1


def test_a_long_prefix_behind_far_pages():
    B, H, Hkv, d, page, P = 3, 4, 2, 128, 64, 100000
    g = torch.Generator(device="cuda").manual_seed(1)
    pages = 140000  # 4.6 GB a pool
    kp, vp = (torch.zeros((pages, Hkv, page, d), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    held = -(-P // page)
    prefix = (pages - 1 - torch.randperm(held, generator=g, device="cuda")).to(torch.int32)
    table = torch.arange(B, dtype=torch.int32, device="cuda")[:, None]
    for x in (kp, vp):
        for at in (prefix.long(), table.long().view(-1)):
            x[at] = torch.randn((len(at), Hkv, page, d), generator=g, device="cuda").bfloat16()
    q = torch.randn((B, H, 1, d), generator=g, device="cuda").bfloat16()
    want = ref.attention(q, kp, vp, table, [64, 1, 0], prefix=prefix, prefix_len=P)
    o, lse = mb.mosaic_bsa_prefix_decode(mb.PagedParams(), q, kp, vp, prefix, P, table, lens([64, 1, 0]))
    compare(want, o, lse, q, kp[prefix.long()], 0.0, P + 64)
