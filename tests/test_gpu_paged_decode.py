"""Attention over a paged cache against the definition in 64 bits.

Tolerances.  u = eps/2 of the 16-bit type bounds a rounding to nearest, relative.  Every weight rounds to 16 bits once (u of it) and the
result once; the rest is fp32: scores are sums of d exact products (d * 2^-24 of the sum of magnitudes, as an absolute error of the
exponent), exponentials are good to 3e-6, and a row's sums run through at most 8 steps of a warp, 3 shuffles, 8 warps and the parts,
each addition off by at most 2^-23.  So |o - o64| <= u |o| + (u + E) sum_j p_j |v_j|, E = 2 (d 2^-24 smax + 4e-6) + (32 + parts) 2^-23,
smax the largest sum of magnitudes in a score; |lse - lse64| <= E + 2^-22 |lse|.  fp16 has steps of 2^-25 for weights below its normal
range, relative to the row's largest weight, per key."""
import math

import pytest
import torch

from paper_2604_16429_b200 import binding as mb
from tests import gpu_util as G
from tests import paged_ref as ref

pytestmark = pytest.mark.gpu
DT = {"bf16": torch.bfloat16, "fp16": torch.float16}
NAN = float("nan")


def lens(x):
    return None if x is None else torch.tensor(x, dtype=torch.int32, device="cuda")


def make(B, H, Hkv, T, d, page, width, dtype="bf16", layout="bhnd", pages_layout="hpd", extra=2, seed=0, sharp=1.0):
    """q, pools, table: every member has pages of its own"""
    g = torch.Generator().manual_seed(seed)
    q = (sharp * torch.randn((B, T, H, d) if layout == "bnhd" else (B, H, T, d), generator=g)).to(DT[dtype]).cuda()
    pages = B * width + extra
    pools = [torch.randn((pages, page, Hkv, d) if pages_layout == "phd" else (pages, Hkv, page, d), generator=g).to(DT[dtype]).cuda()
             for _ in range(2)]
    if pages_layout == "phd":
        pools = [x.transpose(1, 2) for x in pools]
    table = torch.randperm(pages, generator=g)[:B * width].view(B, width).to(torch.int32).cuda()
    return q.transpose(1, 2) if layout == "bnhd" else q, *pools, table


def spoil(pools, table, k_len, page, first=None, sinks=0):
    """Slots that no row sees: NaN and infinities"""
    for n, x in zip((NAN, math.inf), pools):
        used = torch.zeros(x.shape[0], page, dtype=torch.bool)
        for b in range(table.shape[0]):
            for j in range(min(max(k_len[b], 0), table.shape[1] * page)):
                if first is None or j >= first[b] or j < sinks:
                    at = ref.place(table, b, j, page, x.shape[0])
                    if at:
                        used[at] = True
        x.transpose(1, 2)[~used.cuda()] = n


def tolerances(want, q, k_pages, scale, keys):
    d = q.shape[-1]
    k = torch.nan_to_num(k_pages.double(), 0.0, 0.0, 0.0).abs()
    smax = float(torch.nan_to_num(q.double()).abs().amax() * k.sum(-1).max()) * (scale or d ** -0.5)
    E = 2 * (d * 2.0 ** -24 * smax + 4e-6) + (32 + keys // 512 + 64) * 2.0 ** -23
    u = torch.finfo(q.dtype).eps / 2
    sub = 2.0 ** -25 * keys * 8 if q.dtype == torch.float16 else 0.0  # (values of at most 8)
    return u * want["o"].abs() + (u + E) * want["p_abs"] + sub + 1e-7, E + 2.0 ** -22 * want["lse"].abs()


def compare(want, o, lse, q, k_pages, scale, keys):
    there = ~torch.isnan(want["lse"])
    assert torch.isnan(o[~there]).all() and torch.isnan(lse[~there]).all(), "rows that do not exist were written"
    assert not torch.isnan(o[there]).any() and not torch.isnan(lse[there]).any()
    empty = there & (want["lse"] == -math.inf)
    assert (lse[empty] == -math.inf).all() and (o[empty] == 0).all()
    full = there & ~empty
    tol_o, tol_l = tolerances(want, q, k_pages, scale, keys)
    if full.any():
        off = (o.double() - want["o"]).abs() - tol_o
        assert off[full].max() <= 0, f"o: over by {float(off[full].max()):.3g}"
        off = (lse.double() - want["lse"]).abs() - tol_l
        assert off[full].max() <= 0, f"lse: over by {float(off[full].max()):.3g}"


def check(pp, q, kp, vp, table, k_len, q_len=None, finite=None):
    page = kp.shape[2]
    clean = finite or (kp, vp)
    want = ref.attention(q, *clean, table, k_len, pp.window, pp.sinks, pp.scale, q_len)
    o, lse = G.Guarded(tuple(q.shape), q.dtype, fill=NAN), G.Guarded(tuple(q.shape[:3]), torch.float32, fill=NAN)
    ws = G.Guarded((mb.paged_workspace_bytes(pp, q, kp, table),), torch.uint8)
    mb.mosaic_bsa_paged_decode(pp, q, kp, vp, table, lens(k_len), q_len=lens(q_len), o=o.t, lse=lse.t, ws=ws.t)
    mb.check_status(ws.t, "paged_decode")
    for x, name in ((o, "o"), (lse, "lse"), (ws, "workspace")):
        x.check(name)
    compare(want, o.t, lse.t, q, clean[0], pp.scale, table.shape[1] * page)
    return o.t, lse.t


CASES = [  # B, H, Hkv, T, d, page, k_len, q_len, window, sinks
    (1, 1, 1, 1, 64, 16, [1], None, 0, 0),
    (1, 2, 1, 1, 128, 16, [17], None, 5, 1),
    (2, 4, 2, 1, 64, 32, [300, 299], None, 64, 4),
    (3, 16, 2, 1, 128, 64, [0, 1, 1000], None, 0, 0),
    (2, 24, 2, 1, 128, 128, [777, 130], None, 0, 0),         # more than eight heads in a group
    (2, 34, 1, 1, 128, 16, [90, 4], None, 17, 3),            # more rows than a CTA takes
    (4, 6, 3, 1, 64, 256, [4099, 40, 33, 2000], None, 0, 0),
    (1, 8, 8, 1, 128, 16, [9000], None, 0, 0),
    (2, 8, 8, 1, 64, 32, [5000, 700], None, 1000, 128),
    (3, 4, 2, 5, 64, 16, [300, 5, 3], [5, 2, 5], 0, 0),      # drafts; more new tokens than tokens
    (2, 12, 3, 16, 128, 64, [1111, 16], None, 100, 4),
    (2, 6, 2, 3, 64, 512, [1537, 512], [3, 0], 513, 2),
    (1, 8, 1, 7, 128, 16, [2048], None, 2048, 7),
    (40, 2, 2, 1, 64, 16, [(37 * i) % 200 for i in range(40)], None, 0, 0),
    (300, 3, 1, 1, 64, 16, [(11 * i) % 70 for i in range(300)], None, 30, 1),  # more members than threads
]


@pytest.mark.parametrize("case", CASES, ids=lambda c: str(c)[:60])
@pytest.mark.parametrize("dtype,layout,pages", [("bf16", "bhnd", "phd"), ("fp16", "bnhd", "hpd")])
def test_paged_decode(case, dtype, layout, pages):
    B, H, Hkv, T, d, page, k_len, q_len, window, sinks = case
    width = max(1, -(-max(k_len) // page)) + 1
    q, kp, vp, table = make(B, H, Hkv, T, d, page, width, dtype, layout, pages, seed=d + B + window)
    pp = mb.PagedParams(window=window, sinks=sinks)
    clean = kp.clone(), vp.clone()
    kls, qls = ref.lengths(B, T, width * page, k_len, q_len)
    first = [max(0, kls[b] - qls[b] - window + 1) for b in range(B)] if window else None
    if B <= 40:
        spoil((kp, vp), table, k_len, page, first, sinks)
    if q_len:
        for b in range(B):
            q[b, :, q_len[b]:] = NAN
    o, lse = check(pp, q, kp, vp, table, k_len, q_len, clean)
    again = mb.mosaic_bsa_paged_decode(pp, q, kp, vp, table, lens(k_len), q_len=lens(q_len))
    same = ~torch.isnan(lse)
    assert torch.equal(again[0][same], o[same]) and torch.equal(again[1][same], lse[same])
    if 1 < B <= 40:  # a member's bits do not depend on the others
        one = mb.mosaic_bsa_paged_decode(pp, q[1:2], kp, vp, table[1:2], lens(k_len[1:2]), q_len=lens(q_len[1:2]) if q_len else None)
        assert torch.equal(one[0][0][same[1]], o[1][same[1]]) and torch.equal(one[1][0][same[1]], lse[1][same[1]])


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("T", [1, 4])
def test_pages_that_are_not_there_are_not_seen(d, T):
    big = 2 ** 31 - 1
    q, kp, vp, _ = make(4, 4, 2, T, d, 16, 1, seed=3, extra=60)
    table = torch.tensor([[3, -1, 7, big], [64, 1, -big, 2], [-1, -1, -1, -1], [63, 62, 61, 60]], dtype=torch.int32, device="cuda")
    for window in (0, 20):
        check(mb.PagedParams(window=window, sinks=2 if window else 0), q, kp, vp, table, [64, 50, 33, 61])


def test_lengths_beyond_the_table_are_clamped():
    q, kp, vp, table = make(2, 4, 2, 2, 64, 16, 3, seed=4)
    check(mb.PagedParams(), q, kp, vp, table, [1000, -5], [7, 2])


def test_pages_that_members_share():
    q, kp, vp, table = make(3, 8, 2, 1, 128, 32, 20, seed=5)
    table[1:, :10] = table[0, :10]
    table[2, 11] = table[2, 10]  # a page twice in a row
    check(mb.PagedParams(), q, kp, vp, table, [640, 333, 500])
    check(mb.PagedParams(), q, kp, vp, table[:1].expand(3, 20), [640, 333, 500])  # one table for all


def test_scale_and_sharp_scores():
    q, kp, vp, table = make(2, 4, 2, 1, 64, 16, 70, seed=6, sharp=6.0)
    for scale in (0.0, 0.02, 1.0):
        check(mb.PagedParams(scale=scale), q, kp, vp, table, [1100, 900])


def test_views_of_larger_pools():
    q, kp, vp, table = make(2, 4, 2, 1, 64, 16, 10, seed=7)
    wide = torch.full((kp.shape[0], 5, 16, 192), NAN, dtype=kp.dtype, device="cuda")  # heads 1 and 3, keys and values side by side
    wide[:, 1:5:2, :, :64], wide[:, 1:5:2, :, 64:128] = kp, vp
    want = mb.mosaic_bsa_paged_decode(mb.PagedParams(), q, kp, vp, table, lens([160, 99]))
    got = mb.mosaic_bsa_paged_decode(mb.PagedParams(), q, wide[:, 1:5:2, :, :64], wide[:, 1:5:2, :, 64:128], table, lens([160, 99]))
    assert torch.equal(want[0], got[0]) and torch.equal(want[1], got[1])


def test_a_long_cache_and_far_pages():
    """Two hundred and more parts a row, pages behind 2^32 bytes."""
    B, H, Hkv, d, page, width = 2, 8, 2, 128, 64, 2100
    g = torch.Generator(device="cuda").manual_seed(1)
    pages = 140000  # 4.6 GB a pool
    kp, vp = (torch.zeros((pages, Hkv, page, d), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    table = (pages - 1 - torch.randperm(B * width, generator=g, device="cuda")).view(B, width).to(torch.int32)
    for x in (kp, vp):
        x[table.long().view(-1)] = torch.randn((B * width, Hkv, page, d), generator=g, device="cuda").bfloat16()
    q = torch.randn((B, H, 1, d), generator=g, device="cuda").bfloat16()
    k_len = [width * page - 7, 70001]
    want = ref.attention(q, kp, vp, table, k_len)
    o, lse = mb.mosaic_bsa_paged_decode(mb.PagedParams(), q, kp, vp, table, lens(k_len))
    tol_o, tol_l = tolerances(want, q, kp[table[0].long()], 0.0, width * page)
    assert ((o.double() - want["o"]).abs() <= tol_o).all() and ((lse.double() - want["lse"]).abs() <= tol_l).all()


def test_it_is_the_linear_cache_in_pages():
    """The same keys in one tensor and in pages: the same results up to the order of sums."""
    B, H, Hkv, d, page, N = 3, 8, 2, 128, 16, 1000
    g = torch.Generator().manual_seed(2)
    q, k, v = (torch.randn((B, h, n, d), generator=g).bfloat16().cuda() for h, n in ((H, 1), (Hkv, N), (Hkv, N)))
    width = -(-N // page)
    table = torch.randperm(B * width, generator=g).view(B, width).to(torch.int32).cuda()
    kp, vp = (torch.zeros((B * width, Hkv, page, d), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    rp = mb.RotaryParams(d=d, rot_dim=0)
    mb.mosaic_bsa_paged_append(rp, k, v, kp, vp, table, lens([N] * B))
    kl = lens([1000, 1, 517])
    for window, sinks in ((0, 0), (200, 4)):
        a = mb.mosaic_bsa_window_decode(mb.WindowParams(window=window or N, sinks=sinks), q, k, v, k_len=kl)
        b = mb.mosaic_bsa_paged_decode(mb.PagedParams(window=window, sinks=sinks), q, kp, vp, table, kl)
        want = ref.attention(q, kp, vp, table, [1000, 1, 517], window, sinks)
        tol_o, tol_l = tolerances(want, q, kp, 0.0, N)  # both are this far from the definition
        assert ((a[0].double() - b[0].double()).abs() <= 2 * tol_o).all() and ((a[1].double() - b[1].double()).abs() <= 2 * tol_l).all()
