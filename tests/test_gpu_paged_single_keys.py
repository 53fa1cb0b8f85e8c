"""Long caches and prefixes behind far pages, where single keys decide: every 512 positions hold one key that one row in 32 looks at, at
the first, the last or another place of the chunk, so that a row is an average of a few values and losing one of them, or a step of 64
keys, or a part, or taking another page's, is far outside the tolerance (which the test checks for each of them).  Pages that
belong to nobody, and slots behind the end, hold NaN.  Tolerances: those of tests/test_gpu_paged_decode.py."""
import math

import pytest
import torch

from paper_2604_16429_b200 import binding as mb
from tests import paged_ref as ref
from tests.test_gpu_paged_decode import NAN, compare, lens, tolerances

pytestmark = pytest.mark.gpu
ROWS = 32  # directions, one a row


def directions(d):
    """Rows of +-1 at right angles"""
    h = torch.ones(1, 1, device="cuda")
    while h.shape[0] < d:
        h = torch.cat((torch.cat((h, h), 1), torch.cat((h, -h), 1)))
    return h[1:ROWS + 1]


def chosen(n):
    """(position, direction) of the keys that count among n"""
    for c in range(-(-n // 512)):
        yield min(n - 1, 512 * c + (0, 511, 64, 447, 255, 130)[c % 6]), c % ROWS


def fill(pools, pages, n, g):
    """n tokens to the pages of one sequence.  Keys and values of normal values, and the chosen keys."""
    page, Hkv, d = pools[0].shape[2], pools[0].shape[1], pools[0].shape[3]
    held = -(-n // page)
    dirs = directions(d)
    for i, x in enumerate(pools):
        rows = torch.randn((held * page, Hkv, d), generator=g, device="cuda")
        if i == 0:
            for j, c in chosen(n):
                rows[j] = 16 / math.sqrt(d) * dirs[c]  # a score of 16, where a hundred thousand others together have e^12.3
        rows[n:] = NAN
        x[pages[:held].long()] = rows.view(held, page, Hkv, d).transpose(1, 2).to(x.dtype)


def queries(B, H, Hkv, d, call, g):
    """Row h of a group looks in the direction call * (H / Hkv) + h"""
    G = H // Hkv
    q = 0.3 * torch.randn((B, H, 1, d), generator=g, device="cuda")
    q += directions(d)[call * G:(call + 1) * G].repeat(Hkv, 1)[None, :, None]
    return q.bfloat16()


def look_that_every_key_counts(q, k, v, n, tol, call):
    """q [G, d] of one member and key head, k and v [n, d] in 64 bits; tol [G, d]: leaving out any step of 64 keys that holds a chosen
    key is seen"""
    G = q.shape[0]
    w = torch.softmax(q.double() @ k.T / math.sqrt(q.shape[1]), -1)
    for j, c in chosen(n):
        if call * G <= c < (call + 1) * G:
            s = slice(j // 64 * 64, min(n, j // 64 * 64 + 64))
            lost = (w[c - call * G, s] @ v[s]).abs()
            assert (lost > 2 * tol[c - call * G]).any(), f"the key at {j} may be lost unseen"


def far_pools(pages, Hkv, page, d):
    return [torch.full((pages, Hkv, page, d), NAN, dtype=torch.bfloat16, device="cuda") for _ in range(2)]


def test_a_long_cache():
    """263 and 137 parts a row, pages behind 2^32 bytes."""
    B, H, Hkv, d, page, width, pages = 2, 8, 2, 128, 64, 2100, 140000  # 4.6 GB a pool
    g = torch.Generator(device="cuda").manual_seed(1)
    pools = far_pools(pages, Hkv, page, d)
    table = (pages - 1 - torch.randperm(B * width, generator=g, device="cuda")).view(B, width).to(torch.int32)
    assert int(table.min()) * pools[0].stride(0) * 2 > 1 << 32
    k_len = [width * page - 7, 70001]
    for b in range(B):
        fill(pools, table[b], k_len[b], g)
    for call in range(ROWS // (H // Hkv)):
        q = queries(B, H, Hkv, d, call, g)
        want = ref.attention(q, *pools, table, k_len)
        o, lse = mb.mosaic_bsa_paged_decode(mb.PagedParams(), q, *pools, table, lens(k_len))
        compare(want, o, lse, q, pools[0][table[0].long()], 0.0, width * page)
        tol = tolerances(want, q, pools[0][table[0].long()], 0.0, width * page)[0]
        for b in range(B):
            for h in range(Hkv):
                k, v = (ref.gather(x, table, b, h, k_len[b], page)[0] for x in pools)
                rows = slice(h * (H // Hkv), (h + 1) * (H // Hkv))
                look_that_every_key_counts(q[b, rows, 0], k, v, k_len[b], tol[b, rows, 0], call)


def test_a_long_prefix():
    B, H, Hkv, d, page, P, pages = 3, 8, 2, 128, 64, 100000, 140000
    g = torch.Generator(device="cuda").manual_seed(2)
    pools = far_pools(pages, Hkv, page, d)
    held = -(-P // page)
    prefix = (pages - 1 - torch.randperm(held, generator=g, device="cuda")).to(torch.int32)
    assert int(prefix.min()) * pools[0].stride(0) * 2 > 1 << 32
    table, k_len = torch.arange(B, dtype=torch.int32, device="cuda")[:, None], [64, 1, 0]
    fill(pools, prefix, P, g)
    for x in pools:
        x[:B] = torch.randn((B, Hkv, page, d), generator=g, device="cuda").bfloat16()
    for call in range(ROWS // (H // Hkv)):
        q = queries(B, H, Hkv, d, call, g)
        want = ref.attention(q, *pools, table, k_len, prefix=prefix, prefix_len=P)
        o, lse = mb.mosaic_bsa_prefix_decode(mb.PagedParams(), q, *pools, prefix, P, table, lens(k_len))
        compare(want, o, lse, q, pools[0][prefix.long()], 0.0, P + 64)
        tol = tolerances(want, q, pools[0][prefix.long()], 0.0, P + 64)[0]
        for h in range(Hkv):
            k, v = (ref.gather(x, prefix[None], 0, h, P, page)[0] for x in pools)
            rows = slice(h * (H // Hkv), (h + 1) * (H // Hkv))
            look_that_every_key_counts(q[2, rows, 0], k, v, P, tol[2, rows, 0], call)
