"""A run of the paged cache's calls as a server makes them: a shared prompt goes to pages once, every member's question behind it, then
tokens one by one and drafts, against the whole sequences' attention in 64 bits on what each stage before really gave."""
import math

import pytest
import torch

from paper_2604_16429_b200 import binding as mb
from tests import test_gpu_paged_decode as D
from tests import test_gpu_rotary as R

pytestmark = pytest.mark.gpu


def whole(q, k, v, pos, window=0, sinks=0):
    """o, lse, p_abs of rows q [H, T, d] at positions pos over keys k, v [Hkv, N, d] from position 0 on"""
    H, T, d = q.shape
    G = H // k.shape[0]
    j = torch.arange(k.shape[1], device=q.device)
    see = j <= pos[:, None]
    if window:
        see &= (pos[:, None] - j < window) | (j < sinks)
    s = (q.double() @ k.double().repeat_interleave(G, 0).transpose(1, 2) / math.sqrt(d)).masked_fill(~see, -math.inf)
    p = torch.softmax(s, -1)
    z = v.double().repeat_interleave(G, 0)
    return {"o": p @ z, "lse": torch.logsumexp(s, -1), "p_abs": p @ z.abs()}


def near(got, lse, want, q, k):
    want = {n: x[None] for n, x in want.items()}
    tol_o, tol_l = D.tolerances(want, q[None], k[:, None], 0.0, k.shape[1])
    assert ((got[None].double() - want["o"]).abs() <= tol_o).all() and ((lse[None].double() - want["lse"]).abs() <= tol_l).all()


@pytest.mark.parametrize("d,half,page,dtype", [(64, False, 16, "fp16"), (128, True, 32, "bf16")])
def test_a_server(d, half, page, dtype):
    B, H, Hkv, P, steps = 3, 8, 2, 77, 6
    asked = [5, 1, 40]  # lengths of the questions
    g = torch.Generator().manual_seed(d)
    rp = mb.RotaryParams(d=d, half=half)
    fr = mb.rotary_freqs(rp)
    new = lambda h, n, b=1: torch.randn((b, n, h, d), generator=g).to(D.DT[dtype]).cuda().transpose(1, 2)  # noqa: E731
    pages, width = 40, 6
    pools = [torch.full((pages, Hkv, page, d), float("nan"), dtype=D.DT[dtype], device="cuda") for _ in range(2)]
    ids = torch.randperm(pages, generator=g).to(torch.int32).cuda()
    held = -(-P // page)
    prefix, table = ids[:held].clone(), ids[held:held + B * width].view(B, width).clone()
    # the shared prompt: attention over itself, keys and values to their pages
    q, k, v = new(H, P), new(Hkv, P), new(Hkv, P)
    qr = mb.mosaic_bsa_paged_append(rp, k, v, *pools, prefix[None], D.lens([P]), freqs=fr, q=q)
    want_q, want_k = mb.mosaic_bsa_rotary(rp, q, k, torch.arange(P, device="cuda"), fr)
    assert torch.equal(qr, want_q)
    keys, values = [[want_k[0]] for _ in range(B)], [[v[0]] for _ in range(B)]  # every member's whole sequence
    o, lse = mb.mosaic_bsa_window_fwd(mb.WindowParams(window=P), qr, want_k, v)
    near(o[0], lse[0], whole(qr[0], want_k[0], v[0], torch.arange(P, device="cuda")), qr[0], want_k[0])
    # questions of different lengths and answers, new tokens in rows of up to 16
    k_len = [0] * B
    chunks = [[min(16, asked[b] - i) for i in range(0, asked[b], 16)] + [1] * steps for b in range(B)]
    chunks[0][3], chunks[2][5] = 4, 3  # drafts
    for n in range(max(len(c) for c in chunks)):
        now = [c[n] if n < len(c) else 0 for c in chunks]
        T = max(now)
        q, k, v = new(H, T, B), new(Hkv, T, B), new(Hkv, T, B)
        k_len = [a + b for a, b in zip(k_len, now)]
        at = D.lens(k_len)
        qr = mb.mosaic_bsa_paged_append(rp, k, v, *pools, table, at, freqs=fr, start=P, q=q, q_len=D.lens(now))
        o, lse = mb.mosaic_bsa_prefix_decode(mb.PagedParams(), qr, *pools, prefix, P, table, at, q_len=D.lens(now))
        for b in range(B):
            if not now[b]:
                continue
            pos = P + torch.arange(k_len[b] - now[b], k_len[b], device="cuda")
            R.near(qr[b:b + 1, :, :now[b]], R.turn64(q[b:b + 1, :, :now[b]].double(), pos, rp), 6e-7, R.length(q[b:b + 1, :, :now[b]].double()), "q")
            kr = mb.mosaic_bsa_rotary(rp, k[b:b + 1, :, :now[b]], k[b:b + 1, :, :now[b]], pos, fr)[1]
            keys[b].append(kr[0])
            values[b].append(v[b, :, :now[b]])
            kk, vv = torch.cat(keys[b], 1), torch.cat(values[b], 1)
            near(o[b, :, :now[b]], lse[b, :, :now[b]], whole(qr[b, :, :now[b]], kk, vv, pos), qr[b, :, :now[b]], kk)
    # the members part from the prefix: its last page, half full, is copied, the full ones are shared; then a window over the whole
    tail = P % page
    full = P // page
    spare = ids[held + B * width:held + B * width + B]
    for p in pools:
        p[spare.long()] = p[prefix[full].long()].clone()[None]
    own = torch.cat((prefix[:full].expand(B, -1), spare[:, None], torch.full((B, width), -1, dtype=torch.int32, device="cuda")), 1)
    assert tail and own.shape[1] == held + width
    for b in range(B):  # a member's own tokens follow in the copied page: append them anew
        kk, vv = torch.cat(keys[b][1:], 1)[None], torch.cat(values[b][1:], 1)[None]
        n = kk.shape[2]
        row = own[b:b + 1].clone()
        row[0, held:held + width] = table[b]
        still = mb.RotaryParams(d=d, rot_dim=0)
        mb.mosaic_bsa_paged_append(still, kk, vv, *pools, row, D.lens([P + n]))
        q1 = new(H, 1)
        for window, sinks in ((0, 0), (30, 4)):
            o, lse = mb.mosaic_bsa_paged_decode(mb.PagedParams(window=window, sinks=sinks), q1, *pools, row, D.lens([P + n]))
            kk_all, vv_all = torch.cat(keys[b], 1), torch.cat(values[b], 1)
            near(o[0], lse[0], whole(q1[0], kk_all, vv_all, torch.tensor([P + n - 1], device="cuda"), window, sinks), q1[0], kk_all)
