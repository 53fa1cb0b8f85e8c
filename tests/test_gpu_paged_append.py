"""Appending to a paged cache against the definition in 64 bits.

Tolerances: those of the rotation by token index (tests/test_gpu_rotary.py: half a step of the storage type, and 6e-7 of the pair's
length for angle, cosine, sine and turn); values, and channels that do not turn, keep their bits."""
import pytest
import torch

from paper_2604_16429_b200 import binding as mb
from tests import gpu_util as G
from tests import paged_ref as ref
from tests.test_gpu_rotary import length, near, turn64

pytestmark = pytest.mark.gpu
DT = {"bf16": torch.bfloat16, "fp16": torch.float16}


def lens(x):
    return None if x is None else torch.tensor(x, dtype=torch.int32, device="cuda")


def heads(g, B, h, N, d, dtype, layout):
    x = torch.randn((B, N, h, d) if layout == "bnhd" else (B, h, N, d), generator=g).to(DT[dtype]).cuda()
    return x.transpose(1, 2) if layout == "bnhd" else x


def pool(pages, Hkv, page, d, dtype, layout, fill):
    """A guarded pool [pages, Hkv, page, d] in either memory order"""
    x = G.Guarded((pages, page, Hkv, d) if layout == "phd" else (pages, Hkv, page, d), DT[dtype], fill=fill)
    return x, x.t.transpose(1, 2) if layout == "phd" else x.t


def check(B, H, Hkv, N, d, rp, page, k_len, q_len=None, dtype="bf16", layout="bhnd", pages_layout="hpd", start=0, table=None, width=None,
          extra=3, seed=0, in_place=False):
    g = torch.Generator().manual_seed(seed)
    k, v = heads(g, B, Hkv, N, d, dtype, layout), heads(g, B, Hkv, N, d, dtype, layout)
    q = heads(g, B, H, N, d, dtype, layout) if H else None
    width = width or max(1, -(-max(k_len) // page))
    pages = B * width + extra
    if table is None:
        table = torch.randperm(pages, generator=g)[:B * width].view(B, width)
    table = torch.as_tensor(table, dtype=torch.int32).cuda()
    gk, kp = pool(pages, Hkv, page, d, dtype, pages_layout, 3.0)
    gv, vp = pool(pages, Hkv, page, d, dtype, pages_layout, -5.0)
    fr = mb.rotary_freqs(rp) if rp.rot else None
    out = None if q is None else q.clone() if in_place else torch.full_like(q, 7.0)
    got = mb.mosaic_bsa_paged_append(rp, k, v, kp, vp, table, lens(k_len), freqs=fr, start=start, q=out if in_place else q, q_len=lens(q_len),
                                     q_out=out)
    gk.check("k_pages"), gv.check("v_pages")
    kls, qls = ref.lengths(B, N, width * page, k_len, q_len)
    left_k, left_v = torch.ones((pages, page), dtype=torch.bool), torch.ones((pages, page), dtype=torch.bool)
    turn = lambda x, pos: turn64(x.double(), pos, rp) if rp.rot and len(pos) else x.double()  # noqa: E731
    for b in range(B):
        pos = start + torch.arange(kls[b] - qls[b], kls[b], device="cuda")
        if q is not None:
            near(got[b:b + 1, :, :qls[b]], turn(q[b:b + 1, :, :qls[b]], pos), 6e-7 * rp.amplitude, length(q[b:b + 1, :, :qls[b]].double()), "q") \
                if qls[b] else None
            assert torch.equal(got[b, :, :qls[b], rp.rot:], q[b, :, :qls[b], rp.rot:])
            if not in_place:
                assert (got[b, :, qls[b]:] == 7).all(), "rows that do not exist were written"
            else:
                assert torch.equal(got[b, :, qls[b]:], q[b, :, qls[b]:])
        want = turn(k[b:b + 1, :, :qls[b]], pos)
        for i in range(qls[b]):
            at = ref.place(table, b, kls[b] - qls[b] + i, page, pages)
            if at is None:
                continue
            left_k[at] = left_v[at] = False
            near(kp[at[0], :, at[1]], want[0, :, i], 6e-7 * rp.amplitude, length(k[b, :, i].double()), "k")
            assert torch.equal(kp[at[0], :, at[1], rp.rot:], k[b, :, i, rp.rot:])
            assert torch.equal(vp[at[0], :, at[1]], v[b, :, i])
    assert (kp.transpose(1, 2)[left_k.cuda()] == 3).all() and (vp.transpose(1, 2)[left_v.cuda()] == -5).all(), "other slots were written"


CASES = [  # B, H, Hkv, N, d, rot, half, page, k_len, q_len
    (1, 1, 1, 1, 64, 64, True, 16, [1], None),
    (3, 4, 2, 5, 64, 64, False, 16, [5, 21, 100], [5, 3, 0]),
    (2, 16, 4, 1, 128, 128, True, 16, [300, 17], None),
    (2, 12, 3, 70, 64, 48, False, 32, [70, 171], [70, 41]),
    (2, 0, 4, 33, 128, 32, True, 64, [64, 33], None),               # no queries
    (1, 6, 6, 40, 128, 0, False, 128, [1000], None),                # nothing turns
    (4, 5, 1, 9, 128, 34, False, 256, [9, 8, 700, 5], [9, 9, 2, 7]),  # more new tokens than tokens: the first have no place
    (2, 40, 8, 17, 64, 16, True, 16, [17, 160], None),
    (1, 0, 1, 300, 64, 64, True, 512, [300], None),
]


@pytest.mark.parametrize("case", CASES, ids=str)
@pytest.mark.parametrize("dtype,layout,pages", [("bf16", "bhnd", "phd"), ("fp16", "bnhd", "hpd")])
def test_append(case, dtype, layout, pages):
    B, H, Hkv, N, d, rot, half, page, k_len, q_len = case
    rp = mb.RotaryParams(d=d, rot_dim=rot, half=half, amplitude=1.25)
    check(B, H, Hkv, N, d, rp, page, k_len, q_len, dtype, layout, pages, start=1000, seed=N)


@pytest.mark.parametrize("start", [-7, 1 << 20, (1 << 31) + 5])
def test_positions_behind_a_prefix(start):
    check(2, 4, 2, 6, 64, mb.RotaryParams(d=64), 16, [6, 50], start=start)


def test_queries_in_place():
    check(2, 4, 2, 6, 64, mb.RotaryParams(d=64, half=True), 16, [6, 50], [3, 6], in_place=True)


def test_pages_that_are_not_there_are_not_written():
    big = 2 ** 31 - 1
    table = [[4, -1, 2], [big, 0, 7], [9, -big, 1]]  # nine pages: 9 is none either
    check(3, 2, 2, 40, 64, mb.RotaryParams(d=64), 16, [40, 41, 48], table=table, extra=0)


def test_lengths_beyond_the_table_are_clamped():
    check(2, 2, 1, 4, 64, mb.RotaryParams(d=64), 16, [100, -3], [9, -1], width=2)


def test_a_table_that_is_a_slice():
    g = torch.Generator().manual_seed(3)
    k = heads(g, 2, 2, 20, 64, "bf16", "bhnd")
    whole = torch.arange(12, dtype=torch.int32, device="cuda").view(2, 6)
    rp = mb.RotaryParams(d=64, rot_dim=0)
    pools = [torch.zeros((12, 2, 16, 64), dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    mb.mosaic_bsa_paged_append(rp, k, k, *pools, whole[:, 2:5], lens([20, 20]))
    for b in range(2):
        assert torch.equal(pools[0][whole[b, 2].long()], k[b, :, :16]) and torch.equal(pools[1][whole[b, 3].long(), :, :4], k[b, :, 16:])
    assert int((pools[0] != 0).any(-1).any(-1).any(-1).sum()) == 4


def test_infinities_and_numbers_that_are_none_keep_to_their_channels():
    rp = mb.RotaryParams(d=64, rot_dim=32)
    k = torch.randn(1, 1, 4, 64).bfloat16().cuda()
    k[..., 40] = float("nan")
    k[..., 50] = float("inf")
    pools = [torch.zeros((1, 1, 16, 64), dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    mb.mosaic_bsa_paged_append(rp, k, k, *pools, lens([[0]]), lens([4]), freqs=mb.rotary_freqs(rp))
    same = k[0, 0].view(torch.int16)
    assert torch.equal(pools[0][0, 0, :4, 32:].view(torch.int16), same[:, 32:]) and not pools[0][0, 0, :4, :32].isnan().any()
    assert torch.equal(pools[1][0, 0, :4].view(torch.int16), same)


def test_many_tokens_and_far_pages():
    """Offsets behind 2^31 bytes in the pools, more tokens than warps in flight."""
    B, Hkv, N, d, page, pages = 3, 8, 2500, 128, 64, 20000  # 2.6 GB a pool
    g = torch.Generator(device="cuda").manual_seed(1)
    k = torch.randn((B, Hkv, N, d), generator=g, device="cuda", dtype=torch.bfloat16)
    pools = [torch.zeros((pages, Hkv, page, d), dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    width = -(-N // page)
    table = (pages - 1 - torch.randperm(B * width, generator=g, device="cuda")).view(B, width).to(torch.int32)
    mb.mosaic_bsa_paged_append(mb.RotaryParams(d=d, rot_dim=0), k, k, *pools, table, lens([N] * B))
    for p in pools:
        got = p[table.long()].transpose(2, 3).reshape(B, width * page, Hkv, d)[:, :N].transpose(1, 2)
        assert torch.equal(got, k)
        assert int((p.view(pages, -1) != 0).any(-1).sum()) == B * width
