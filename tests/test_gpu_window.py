"""Sliding-window attention with sinks against the definition in 64 bits.

Tolerances.  u = eps/2 of the 16-bit type (2^-9 * 2 = 2^-8 for bf16, 2^-11 for fp16) bounds a rounding to nearest, relative.  The
forward rounds every weight to 16 bits once (u of it) and the result once, and works in fp32 otherwise: scores are sums of d
exact products (d * 2^-24 of the sum of magnitudes, as an absolute error of the exponent), exponentials are good to 3e-6.  So
|o - o64| <= u |o| + (u + E) sum_j p_j |v_j|, E = 2 (d 2^-24 smax + 4e-6), smax the largest sum of magnitudes in a score;
|lse - lse64| <= E + 2^-23 |lse|."""
import math

import pytest
import torch

from paper_2604_16429_b200 import binding as mb
from tests import gpu_util as G
from tests import window_ref as ref

pytestmark = pytest.mark.gpu
DT = {"bf16": torch.bfloat16, "fp16": torch.float16}
NAN = float("nan")


def make(B, H, Hkv, Nq, Nk, d, dtype="bf16", layout="bhnd", seed=0, sharp=1.0):
    g = torch.Generator().manual_seed(seed)

    def one(heads, N, f=1.0):
        x = (f * torch.randn((B, N, heads, d) if layout == "bnhd" else (B, heads, N, d), generator=g)).to(DT[dtype]).cuda()
        return x.transpose(1, 2) if layout == "bnhd" else x

    return one(H, Nq, sharp), one(Hkv, Nk), one(Hkv, Nk), one(H, Nq)


def lens(x):
    return None if x is None else torch.tensor(x, dtype=torch.int32, device="cuda")


def score_error(q, k, scale):
    d = q.shape[-1]
    smax = float(q.double().abs().amax(-1).max() * k.double().abs().sum(-1).max()) * (scale or d ** -0.5)
    return 2 * (d * 2.0 ** -24 * smax + 4e-6)


def check_fwd(wp, q, k, v, q_len=None, k_len=None, **kw):
    want = ref.attention(q, k, v, wp.window, wp.sinks, wp.scale, q_len, k_len)
    B, H, Nq, d = q.shape
    o, lse = G.Guarded((B, H, Nq, d), q.dtype, fill=NAN), G.Guarded((B, H, Nq), torch.float32, fill=NAN)
    ws = G.Guarded((mb.window_workspace_bytes(wp, q, k, mb.OP_FWD),), torch.uint8)
    mb.mosaic_bsa_window_fwd(wp, q, k, v, q_len=lens(q_len), k_len=lens(k_len), o=o.t, lse=lse.t, ws=ws.t, **kw)
    mb.check_status(ws.t, "window_fwd")
    for x, name in ((o, "o"), (lse, "lse"), (ws, "workspace")):
        x.check(name)
    there = ~torch.isnan(want["lse"])
    assert torch.isnan(o.t[~there]).all() and torch.isnan(lse.t[~there]).all(), "rows that do not exist were written"
    assert not torch.isnan(o.t[there]).any() and not torch.isnan(lse.t[there]).any()
    E, u = score_error(q, k, wp.scale), torch.finfo(q.dtype).eps / 2
    empty = there & (want["lse"] == -math.inf)
    assert (lse.t[empty] == -math.inf).all() and (o.t[empty] == 0).all()
    full = there & ~empty
    if full.any():
        tol = E + 2.0 ** -23 * want["lse"][full].abs()
        assert ((lse.t[full] - want["lse"][full]).abs() <= tol).all(), float(((lse.t[full] - want["lse"][full]).abs() - tol).max())
        tol = u * want["o"][full].abs() + (u + E) * want["p_abs"][full] + 1e-7
        off = (o.t[full].double() - want["o"][full]).abs()
        assert (off <= tol).all(), f"o: over by {float((off - tol).max()):.3g}"
    return o.t, lse.t


CASES = [  # B, H, Hkv, Nq, Nk, d, window, sinks
    (1, 1, 1, 1, 1, 64, 1, 0),
    (1, 1, 1, 1, 1, 128, 5, 3),
    (1, 2, 1, 128, 128, 64, 128, 0),
    (1, 2, 2, 129, 129, 64, 32, 4),
    (2, 4, 2, 300, 300, 128, 100, 7),
    (1, 3, 1, 400, 400, 64, 1000, 0),      # plain causal
    (1, 3, 1, 500, 500, 128, 1, 1),        # itself and the first token
    (1, 6, 2, 1000, 1000, 64, 127, 33),
    (1, 1, 1, 777, 777, 128, 129, 128),
    (1, 8, 1, 260, 2000, 64, 509, 64),     # a chunk behind a cache
    (1, 2, 1, 7, 1500, 128, 300, 5),
    (3, 5, 5, 257, 1025, 64, 256, 32),
]


@pytest.mark.parametrize("case", CASES, ids=str)
@pytest.mark.parametrize("dtype,layout", [("bf16", "bhnd"), ("fp16", "bnhd")])
def test_forward(case, dtype, layout):
    B, H, Hkv, Nq, Nk, d, window, sinks = case
    q, k, v, _ = make(B, H, Hkv, Nq, Nk, d, dtype, layout, seed=Nq + window)
    check_fwd(mb.WindowParams(window=window, sinks=sinks), q, k, v)


@pytest.mark.parametrize("q_len,k_len", [
    ([0, 1, 300, 17], [0, 1, 300, 900]),        # nothing, one token, a whole sequence, a chunk
    ([300, 200, 5, 128], [100, 0, 900, 128]),   # more queries than keys: the first rows see nothing
    ([1, 1, 1, 1], [900, 899, 1, 128]),
])
@pytest.mark.parametrize("d,G_", [(64, 1), (128, 3)])
def test_ragged_lengths_and_what_lies_behind_them(q_len, k_len, d, G_):
    q, k, v, _ = make(4, 2 * G_, 2, 300, 900, d, seed=5)
    for b in range(4):  # whatever lies behind a sequence's last row is never used
        q[b, :, q_len[b]:] = NAN
        k[b, :, k_len[b]:] = NAN
        v[b, :, k_len[b]:] = math.inf
    kc, vc, qc = k.clone(), v.clone(), q.clone()
    for b in range(4):
        qc[b, :, q_len[b]:] = kc[b, :, k_len[b]:] = vc[b, :, k_len[b]:] = 0
    wp = mb.WindowParams(window=150, sinks=3)
    want = mb.mosaic_bsa_window_fwd(wp, qc, kc, vc, q_len=lens(q_len), k_len=lens(k_len))
    E = score_error(qc, kc, 0)
    o = torch.full_like(q, 7.0)
    lse = torch.full(q.shape[:3], 7.0, device="cuda")
    mb.mosaic_bsa_window_fwd(wp, q, k, v, q_len=lens(q_len), k_len=lens(k_len), o=o, lse=lse)
    for b in range(4):
        assert torch.equal(o[b, :, :q_len[b]], want[0][b, :, :q_len[b]]) and torch.equal(lse[b, :, :q_len[b]], want[1][b, :, :q_len[b]])
        assert (o[b, :, q_len[b]:] == 7).all() and (lse[b, :, q_len[b]:] == 7).all()
    check_fwd(wp, qc, kc, vc, q_len, k_len)


def ring_of(x, kl, sinks, cap):
    """The rolling cache [.., cap, d] that keeps the sinks and the last positions of the first kl rows of x."""
    out = torch.full((*x.shape[:-2], cap, x.shape[-1]), NAN, dtype=x.dtype, device=x.device)
    for j in list(range(min(sinks, kl))) + list(range(max(sinks, kl - (cap - sinks)), kl)):
        out[..., j if j < sinks else sinks + (j - sinks) % (cap - sinks), :] = x[..., j, :]
    return out


DEC = [  # B, H, Hkv, Nk, d, window, sinks, k_len
    (1, 1, 1, 1, 64, 1, 0, None),
    (2, 4, 2, 300, 64, 64, 4, [300, 299]),
    (3, 16, 2, 1000, 128, 333, 7, [0, 1, 1000]),
    (2, 24, 2, 777, 128, 5000, 0, [777, 130]),        # more than eight heads in a group
    (1, 20, 1, 515, 64, 100, 128, [515]),
    (2, 34, 1, 90, 128, 17, 3, [90, 4]),              # more heads than a CTA takes
    (4, 6, 3, 4099, 64, 4000, 33, [4099, 40, 33, 2000]),
    (1, 8, 8, 9000, 128, 8999, 1, None),
]


@pytest.mark.parametrize("case", DEC, ids=str)
@pytest.mark.parametrize("dtype,layout", [("bf16", "bhnd"), ("fp16", "bnhd")])
@pytest.mark.parametrize("rolling", [False, True])
def test_decode(case, dtype, layout, rolling):
    B, H, Hkv, Nk, d, window, sinks, k_len = case
    q, k, v, _ = make(B, H, Hkv, 1, Nk, d, dtype, layout, seed=Nk)
    full = k_len or [Nk] * B
    want = ref.attention(q, k, v, window, sinks, 0.0, [1] * B, full)
    for b in range(B):  # never read
        k[b, :, full[b]:] = NAN
        v[b, :, full[b]:] = NAN
    E, u = score_error(q, torch.nan_to_num(k), 0), torch.finfo(q.dtype).eps / 2
    if rolling:
        cap = min(window, Nk) + min(sinks, Nk) + 5
        window, sinks = min(window, Nk), min(sinks, Nk)
        k, v = (torch.cat([ring_of(x[b:b + 1], full[b], sinks, cap) for b in range(B)]) for x in (k, v))
    wp = mb.WindowParams(window=window, sinks=sinks, rolling=rolling)
    o, lse = G.Guarded((B, H, 1, d), q.dtype, fill=NAN), G.Guarded((B, H, 1), torch.float32, fill=NAN)
    mb.mosaic_bsa_window_decode(wp, q, k, v, k_len=lens(k_len) if not rolling else lens(full), o=o.t, lse=lse.t)
    o.check("o"); lse.check("lse")
    for b in range(B):
        if full[b] == 0:
            assert (o.t[b] == 0).all() and (lse.t[b] == -math.inf).all()
            continue
        tol = E + 2.0 ** -22 * want["lse"][b].abs()
        assert ((lse.t[b] - want["lse"][b]).abs() <= tol).all()
        tol = u * want["o"][b].abs() + (u + E) * want["p_abs"][b] + 1e-7
        off = (o.t[b].double() - want["o"][b]).abs()
        assert (off <= tol).all(), float((off - tol).max())
    again = mb.mosaic_bsa_window_decode(wp, q, k, v, k_len=lens(full) if rolling or k_len else None)
    assert torch.equal(again[0], o.t) and torch.equal(again[1], lse.t)
    if B > 1:  # a member's bits do not depend on the others
        one = mb.mosaic_bsa_window_decode(wp, q[1:2], k[1:2], v[1:2], k_len=lens(full[1:2]))
        assert torch.equal(one[0], o.t[1:2]) and torch.equal(one[1], lse.t[1:2])


def check_bwd(wp, q, k, v, d_o, q_len=None, k_len=None):
    """dv: every weight rounds to 16 bits (u) and is off by E; dS: the same, and D comes from an o that rounded twice (2 u, its
    weights and itself); each result rounds once.  fp16 has steps of 2^-25 for weights below its normal range, per key or row."""
    want = ref.attention(q, k, v, wp.window, wp.sinks, wp.scale, q_len, k_len, d_o)
    o, lse = mb.mosaic_bsa_window_fwd(wp, q, k, v, q_len=lens(q_len), k_len=lens(k_len))
    outs = [G.Guarded(tuple(x.shape), x.dtype, fill=NAN) for x in (q, k, v)]
    ws = G.Guarded((mb.window_workspace_bytes(wp, q, k, mb.OP_BWD),), torch.uint8)
    mb.mosaic_bsa_window_bwd(wp, q, k, v, o, lse, d_o, q_len=lens(q_len), k_len=lens(k_len), dq=outs[0].t, dk=outs[1].t, dv=outs[2].t,
                             ws=ws.t)
    mb.check_status(ws.t, "window_bwd")
    ws.check("workspace")
    E, u = score_error(q, k, wp.scale), torch.finfo(q.dtype).eps / 2
    sc = wp.scale or q.shape[-1] ** -0.5
    n = q.shape[2] * (q.shape[1] // k.shape[1])
    sub = 2.0 ** -25 if q.dtype == torch.float16 else 0.0
    lo = {"dq": sub * sc * k.shape[2] * float(torch.nan_to_num(k).abs().max()), "dk": sub * sc * n * float(torch.nan_to_num(q).abs().max()),
          "dv": sub * n * float(torch.nan_to_num(d_o).abs().max())}
    for name, x in zip(("dq", "dk", "dv"), outs):
        x.check(name)
        there = ~torch.isnan(want[name])
        assert torch.isnan(x.t[~there]).all(), f"{name}: rows that do not exist were written"
        assert not torch.isnan(x.t[there]).any(), name
        f = (u + E) if name == "dv" else 2 * (u + E)
        tol = u * want[name][there].abs() + f * want[name + "_abs"][there] + lo[name] + 1e-7
        off = (x.t[there].double() - want[name][there]).abs()
        assert (off <= tol).all(), f"{name}: over by {float((off - tol).max()):.3g}, worst {float(off.max()):.3g}"
    again = mb.mosaic_bsa_window_bwd(wp, q, k, v, o, lse, d_o, q_len=lens(q_len), k_len=lens(k_len))
    for a, x, name in zip(again, outs, ("dq", "dk", "dv")):
        there = ~torch.isnan(want[name])
        assert torch.equal(a[there], x.t[there]), f"{name}: other bits the second time"
    return want, [x.t for x in outs]


BWD = CASES + [(1, 2, 1, 900, 900, 64, 64, 5), (1, 3, 1, 700, 1100, 128, 70, 100), (2, 2, 2, 1500, 1500, 64, 1, 3)]


@pytest.mark.parametrize("case", BWD, ids=str)
@pytest.mark.parametrize("dtype,layout", [("bf16", "bhnd"), ("fp16", "bnhd")])
def test_backward(case, dtype, layout):
    B, H, Hkv, Nq, Nk, d, window, sinks = case
    q, k, v, d_o = make(B, H, Hkv, Nq, Nk, d, dtype, layout, seed=Nq + window + 1)
    check_bwd(mb.WindowParams(window=window, sinks=sinks), q, k, v, d_o)


@pytest.mark.parametrize("q_len,k_len", [
    ([0, 1, 300, 17], [0, 1, 300, 900]),
    ([300, 200, 5, 128], [100, 0, 900, 128]),
    ([1, 1, 1, 299], [900, 899, 1, 900]),
])
@pytest.mark.parametrize("d,G_", [(64, 1), (128, 3)])
def test_backward_of_ragged_lengths(q_len, k_len, d, G_):
    q, k, v, d_o = make(4, 2 * G_, 2, 300, 900, d, seed=6)
    for b in range(4):
        q[b, :, q_len[b]:] = d_o[b, :, q_len[b]:] = NAN
        k[b, :, k_len[b]:] = NAN
        v[b, :, k_len[b]:] = math.inf
    for W, S in ((150, 3), (20, 70)):
        wp = mb.WindowParams(window=W, sinks=S)
        want = ref.attention(q, k, v, W, S, 0.0, q_len, k_len, d_o)
        o = torch.full_like(q, NAN)  # what lies behind the sequences is never used
        lse = torch.full(q.shape[:3], NAN, device="cuda")
        mb.mosaic_bsa_window_fwd(wp, q, k, v, q_len=lens(q_len), k_len=lens(k_len), o=o, lse=lse)
        got = [torch.full_like(x, 7.0) for x in (q, k, v)]
        mb.mosaic_bsa_window_bwd(wp, q, k, v, o, lse, d_o, q_len=lens(q_len), k_len=lens(k_len), dq=got[0], dk=got[1], dv=got[2])
        E, u = score_error(torch.nan_to_num(q), torch.nan_to_num(k), 0), torch.finfo(q.dtype).eps / 2
        for name, x in zip(("dq", "dk", "dv"), got):
            there = ~torch.isnan(want[name])
            assert (x[~there] == 7).all(), name
            tol = u * want[name][there].abs() + 2 * (u + E) * want[name + "_abs"][there] + 1e-7
            assert ((x[there].double() - want[name][there]).abs() <= tol).all(), name


@pytest.mark.parametrize("case", [
    (1, 3, 1, 700, 1100, 128, 70, 100, "fp16"),   # odd group, short last steps, two steps of sinks
    (2, 4, 2, 600, 600, 128, 20, 70, "bf16"),
    (2, 6, 2, 1500, 1500, 64, 100, 7, "bf16"),
    (1, 8, 2, 2048, 2048, 128, 1024, 4, "bf16"),
    (1, 8, 2, 2048, 2048, 64, 1024, 4, "fp16"),
], ids=str)
def test_the_same_bits_every_time(case):
    B, H, Hkv, Nq, Nk, d, window, sinks, dtype = case
    q, k, v, d_o = make(B, H, Hkv, Nq, Nk, d, dtype, "bnhd", seed=3)
    wp = mb.WindowParams(window=window, sinks=sinks)

    def both():
        o, lse = mb.mosaic_bsa_window_fwd(wp, q, k, v)
        return (o, lse) + mb.mosaic_bsa_window_bwd(wp, q, k, v, o, lse, d_o)

    first = both()
    for _ in range(25):
        for name, a, b in zip(("o", "lse", "dq", "dk", "dv"), first, both()):
            assert torch.equal(a, b), name


def test_a_scale_of_the_callers():
    q, k, v, d_o = make(1, 2, 1, 200, 200, 64, seed=7)
    check_bwd(mb.WindowParams(window=50, sinks=2, scale=0.3), q, k, v, d_o)


@pytest.mark.parametrize("d", [64, 128])
def test_large_scores(d):
    """Scores of some hundreds, falling and rising along the rows, so that the running maximum moves in most steps."""
    q, k, v, _ = make(1, 2, 1, 600, 600, d, seed=8, sharp=6.0)
    k *= (1 + torch.arange(600, device="cuda")[:, None] % 150 / 30).to(k.dtype)
    check_fwd(mb.WindowParams(window=333, sinks=9), q, k, v)


def test_slices_of_a_fused_projection_and_broadcast_heads():
    B, H, Hkv, N, d = 2, 4, 2, 270, 64
    g = torch.Generator().manual_seed(9)
    fused = torch.randn((B, N, H + 2 * Hkv, d), generator=g).bfloat16().cuda()
    q, k, v = (fused[:, :, a:b].transpose(1, 2) for a, b in ((0, H), (H, H + Hkv), (H + Hkv, H + 2 * Hkv)))
    d_o = torch.randn((B, N, H, d), generator=g).bfloat16().cuda().transpose(1, 2)
    wp = mb.WindowParams(window=77, sinks=3)
    check_bwd(wp, q, k, v, d_o)
    # one key head for all, broadcast by a stride of zero; the gradients then come a head each
    k1, v1 = k[:, :1].expand(B, H, N, d), v[:1, :1].expand(B, H, N, d)
    check_bwd(wp, q, k1, v1, d_o)
    o, lse = mb.mosaic_bsa_window_decode(wp, q[:, :, -1:], k1, v1)
    want = mb.mosaic_bsa_window_decode(wp, q[:, :, -1:].contiguous(), k1.contiguous(), v1.contiguous())
    assert torch.equal(o, want[0]) and torch.equal(lse, want[1])


def test_offsets_beyond_32_bits():
    """A cache of 2.4e9 elements: its last head starts at 4.3e9 bytes, its last rows lie at 4.8e9."""
    Hkv, Nk, d = 9, 1 << 21, 128
    k = torch.zeros((1, Hkv, Nk, d), dtype=torch.bfloat16, device="cuda")
    v = torch.zeros_like(k)
    n = 400
    qs, ks, vs, _ = make(1, Hkv, Hkv, 130, n, d, seed=10)
    k[:, :, -n:], v[:, :, -n:] = ks, vs
    wp = mb.WindowParams(window=250, sinks=0)
    want = mb.mosaic_bsa_window_fwd(wp, qs, ks, vs)
    got = mb.mosaic_bsa_window_fwd(wp, qs, k, v)
    # steps start at other keys here: the same sums in another order
    E, u = score_error(qs, ks, 0), torch.finfo(qs.dtype).eps / 2
    ref64 = ref.attention(qs[:, -1:], ks[:, -1:], vs[:, -1:], 250, 0)
    for o, lse in (want, got):
        tol = u * ref64["o"].abs() + (u + E) * ref64["p_abs"] + 1e-7
        assert ((o[:, -1:].double() - ref64["o"]).abs() <= tol).all()
        assert ((lse[:, -1:] - ref64["lse"]).abs() <= E + 2.0 ** -23 * ref64["lse"].abs()).all()
    one = mb.mosaic_bsa_window_decode(wp, qs[:, :, -1:].contiguous(), k, v)
    tol = u * ref64["o"][:, :, -1:].abs() + (u + E) * ref64["p_abs"][:, :, -1:] + 1e-7
    assert ((one[0][:, -1:].double() - ref64["o"][:, :, -1:]).abs() <= tol).all()


def test_on_another_stream_and_in_two_graphs():
    q, k, v, d_o = make(2, 4, 2, 300, 300, 64, seed=11)
    wp = mb.WindowParams(window=100, sinks=4)

    def all_of_it(**kw):
        o, lse = mb.mosaic_bsa_window_fwd(wp, q, k, v, **kw)
        return (o, lse) + mb.mosaic_bsa_window_bwd(wp, q, k, v, o, lse, d_o, **kw) + mb.mosaic_bsa_window_decode(wp, q[:, :, -1:], k, v, **kw)

    want = all_of_it()
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    got = all_of_it(stream=side)
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(want, got))
    ws = torch.empty(mb.window_workspace_bytes(wp, q, k, mb.OP_BWD), dtype=torch.uint8, device="cuda")
    graphs, outs = [], []
    for _ in range(2):  # two graphs on one workspace, replayed in turn on one stream
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[-1]):
            o, lse = mb.mosaic_bsa_window_fwd(wp, q, k, v, ws=ws)
            outs.append((o, lse) + mb.mosaic_bsa_window_bwd(wp, q, k, v, o, lse, d_o, ws=ws))
    for x in outs[0] + outs[1]:
        x.fill_(NAN)
    for i in (0, 1, 0):
        graphs[i].replay()
    torch.cuda.synchronize()
    for got in outs:
        assert all(torch.equal(a, b) for a, b in zip(want, got))


@pytest.mark.parametrize("d", [64, 128])
def test_gradients_of_the_sinks_round_once(d):
    """dv of the sinks' keys: weights as two 16-bit numbers (u^2 of them is left off), sums in fp32, one rounding of the result."""
    q, k, v, d_o = make(1, 4, 2, 1500, 1500, d, seed=18)
    wp = mb.WindowParams(window=100, sinks=7)
    want = ref.attention(q, k, v, 100, 7, 0.0, None, None, d_o)
    o, lse = mb.mosaic_bsa_window_fwd(wp, q, k, v)
    dv = mb.mosaic_bsa_window_bwd(wp, q, k, v, o, lse, d_o)[2][:, :, :7].double()
    E, u = score_error(q, k, 0.0), torch.finfo(q.dtype).eps / 2
    tol = u * want["dv"][:, :, :7].abs() + (u * u + E + 2.0 ** -20) * want["dv_abs"][:, :, :7]
    assert ((dv - want["dv"][:, :, :7]).abs() <= tol).all()


def test_more_units_than_a_grid_is_high():
    """66000 units are 600, checked against the definition, 110 times over."""
    x = make(1, 600, 300, 3, 3, 64, seed=14)
    wp = mb.WindowParams(window=2, sinks=1)
    _, want = check_bwd(wp, *x)
    o, lse = mb.mosaic_bsa_window_fwd(wp, *x[:3])
    q, k, v, d_o = (t.repeat(110, 1, 1, 1) for t in x)
    got = mb.mosaic_bsa_window_fwd(wp, q, k, v)
    for a, b in zip(got + mb.mosaic_bsa_window_bwd(wp, q, k, v, *got, d_o), [o, lse] + want):
        assert torch.equal(a, b.expand(a.shape))


@pytest.mark.parametrize("d,group", [(64, 4), (64, 12), (128, 4), (128, 12)])
def test_decode_of_many_has_the_bits_of_decode_of_one(d, group):
    """Few CTAs ask for rows ahead, many may not: a member's results are the same bits."""
    q, k, v, _ = make(64, 4 * group, 4, 1, 1001, d, seed=17)
    wp = mb.WindowParams(window=900, sinks=5)
    k_len = lens([1001 - 15 * b for b in range(64)])
    o, lse = mb.mosaic_bsa_window_decode(wp, q, k, v, k_len=k_len)
    for b in (0, 1, 31, 63):
        one = mb.mosaic_bsa_window_decode(wp, q[b:b + 1], k[b:b + 1], v[b:b + 1], k_len=k_len[b:b + 1])
        assert torch.equal(one[0], o[b:b + 1]) and torch.equal(one[1], lse[b:b + 1])


def test_calls_of_two_threads_at_once():
    """Each has its own stream, shapes and tensors; the results are those of calls one after the other."""
    import threading

    cases = [(make(2, 4, 2, 300, 300, 64, seed=15), mb.WindowParams(window=100, sinks=4)),
             (make(1, 6, 3, 777, 901, 128, "fp16", "bnhd", seed=16), mb.WindowParams(window=333, sinks=9))]

    def chain(x, wp, **kw):
        q, k, v, d_o = x
        o, lse = mb.mosaic_bsa_window_fwd(wp, q, k, v, **kw)
        return (o, lse) + mb.mosaic_bsa_window_bwd(wp, q, k, v, o, lse, d_o, **kw) + mb.mosaic_bsa_window_decode(wp, q[:, :, -1:], k, v, **kw)

    want = [chain(*c) for c in cases]
    torch.cuda.synchronize()
    got, streams = [None, None], [torch.cuda.Stream(), torch.cuda.Stream()]

    def work(i):
        for _ in range(20):
            with torch.cuda.stream(streams[i]):
                got[i] = chain(*cases[i])
        streams[i].synchronize()

    threads = [threading.Thread(target=work, args=(i,)) for i in (0, 1)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    for w, g in zip(want, got):
        assert all(torch.equal(a, b) for a, b in zip(w, g))


def test_refusals_of_the_binding():
    q, k, v, d_o = make(2, 4, 2, 30, 40, 64, seed=12)
    wp = mb.WindowParams(window=10)
    ln = lens([30, 30])
    for kw in (dict(q=q.float()), dict(k=k.half()), dict(v=v[:, :, :39]), dict(q=q[..., ::2]), dict(k=k[:1]), dict(q_len=ln.long()),
               dict(k_len=ln[:1]), dict(k_len=ln.cpu()), dict(o=q.float()), dict(lse=torch.empty(2, 4, 29, device="cuda")), dict(q=q.cpu()),
               dict(o=q[:1].expand_as(q)), dict(q=q.double()), dict(ws=torch.empty(256, device="cuda"))):
        with pytest.raises(ValueError):
            mb.mosaic_bsa_window_fwd(wp, **{**dict(q=q, k=k, v=v), **kw})
    o, lse = mb.mosaic_bsa_window_fwd(wp, q, k, v)
    for kw in (dict(d_o=d_o.half()), dict(lse=lse.double()), dict(dk=k[:, :1].expand_as(k)), dict(dv=q), dict(dq=q.transpose(0, 1))):
        with pytest.raises(ValueError):
            mb.mosaic_bsa_window_bwd(wp, **{**dict(q=q, k=k, v=v, o=o, lse=lse, d_o=d_o), **kw})
    with pytest.raises(mb.MosaicError) as e:
        mb.mosaic_bsa_window_decode(wp, q, k, v)  # thirty tokens at once
    assert e.value.code == -1
    with pytest.raises(mb.MosaicError) as e:
        mb.mosaic_bsa_window_fwd(wp, q, k, v, ws=torch.empty(128, dtype=torch.uint8, device="cuda"))
    assert e.value.code == -3


@pytest.mark.parametrize("d,half", [(64, False), (128, True)])
def test_a_layer_in_training(d, half):
    """Norm and rotation, attention, and both backward passes, as a layer chains them, each stage against 64 bits on what the stage
    before it really gave."""
    from tests import test_gpu_rotary as R
    B, H, Hkv, N = 2, 6, 2, 333
    q, k, v, d_o = make(B, H, Hkv, N, N, d, "bf16", "bnhd", seed=13)
    rp = mb.RotaryParams(d=d, half=half, scaling=mb.ROTARY_PARTS, factor=4.0, length=4096.0)
    pos, fr = torch.arange(N, device="cuda") + 5000, mb.rotary_freqs(rp)
    wq, wk = 1 + 0.1 * torch.randn(d, device="cuda"), 1 + 0.1 * torch.randn(d, device="cuda")
    wp = mb.WindowParams(window=90, sinks=4)
    qn, kn = mb.mosaic_bsa_qk_norm(rp, q, k, wq, wk, pos, fr)
    for x, w, y in ((q, wq, qn), (k, wk, kn)):
        n = R.norm64(x.double(), w, 1e-6)
        R.near(y, R.turn64(n, pos, rp), 2e-6, R.length(n), "norm")
    want, (dqn, dkn, dv) = check_bwd(wp, qn, kn, v, d_o)
    dq, dk, dwq, dwk = mb.mosaic_bsa_qk_norm_bwd(rp, q, k, wq, wk, pos, fr, dqn, dkn)
    for x, w, dy, dx, dw in ((q, wq, dqn, dq, dwq), (k, wk, dkn, dk, dwk)):
        ref_dx, ref_dw, size, terms = R.grads64(x, w, dy, pos, rp, 1e-6)
        R.near(dx, ref_dx, 4e-6, size, "dx")
        assert ((dw.double() - ref_dw).abs() <= 1.2e-5 * terms).all()


def test_tokens_one_by_one_over_a_rolling_cache_are_the_prompt():
    """A stream of 300 tokens, rotated at its true positions, whose cache keeps 3 sinks and 40 places."""
    H, Hkv, d, N, W, S = 4, 2, 64, 300, 40, 3
    q, k, v, _ = make(1, H, Hkv, N, N, d, seed=14)
    rp = mb.RotaryParams(d=d, half=True)
    fr = mb.rotary_freqs(rp)
    qr, kr = mb.mosaic_bsa_rotary(rp, q, k, torch.arange(N, device="cuda"), fr)
    wp = mb.WindowParams(window=W, sinks=S, rolling=True)
    o, lse = mb.mosaic_bsa_window_fwd(mb.WindowParams(window=W, sinks=S), qr, kr, v)
    want = ref.attention(qr, kr, v, W, S)
    kc, vc = torch.full((1, Hkv, W + S, d), NAN, dtype=k.dtype, device="cuda"), torch.full((1, Hkv, W + S, d), NAN, dtype=k.dtype, device="cuda")
    E, u = score_error(qr, kr, 0), torch.finfo(q.dtype).eps / 2
    for j in range(N):
        q1, k1 = mb.mosaic_bsa_rotary(rp, q[:, :, j:j + 1], k[:, :, j:j + 1], torch.tensor([j], device="cuda"), fr)
        assert torch.equal(q1, qr[:, :, j:j + 1]) and torch.equal(k1, kr[:, :, j:j + 1])
        slot = j if j < S else S + (j - S) % W
        kc[:, :, slot], vc[:, :, slot] = k1[:, :, 0], v[:, :, j]
        if j in (0, 1, 2, 3, 42, 43, 44, 150, 299):
            o1, l1 = mb.mosaic_bsa_window_decode(wp, q1, kc, vc, k_len=lens([j + 1]))
            for a, b in ((o1, o[:, :, j:j + 1]),):
                tol = u * want["o"][:, :, j:j + 1].abs() + (u + E) * want["p_abs"][:, :, j:j + 1] + 1e-7
                assert ((a.double() - want["o"][:, :, j:j + 1]).abs() <= tol).all() and ((b.double() - want["o"][:, :, j:j + 1]).abs() <= tol).all()
            assert ((l1[..., 0] - want["lse"][:, :, j]).abs() <= E + 2.0 ** -22 * want["lse"][:, :, j].abs()).all()


def test_gradients_against_differences():
    """Central differences of the 64-bit forward along random directions: a step of 1e-4 leaves some 1e-8 of third derivatives, and a
    gradient of n elements that are off by tol each is off by tol times the direction's sum of magnitudes."""
    q, k, v, d_o = make(1, 2, 1, 40, 40, 64, "fp16", seed=15)
    wp = mb.WindowParams(window=9, sinks=2)
    o, lse = mb.mosaic_bsa_window_fwd(wp, q, k, v)
    grads = mb.mosaic_bsa_window_bwd(wp, q, k, v, o, lse, d_o)
    want = ref.attention(q, k, v, 9, 2, 0.0, None, None, d_o)
    E, u = score_error(q, k, 0), torch.finfo(q.dtype).eps / 2
    g = torch.Generator().manual_seed(16)
    x = [q.double(), k.double(), v.double()]
    loss = lambda y: (ref.attention(*y, 9, 2)["o"] * d_o.double()).sum()  # noqa: E731
    for i, name in enumerate(("dq", "dk", "dv")):
        t = torch.randn(x[i].shape, generator=g).double().cuda()
        up, down = ([y + s * 1e-4 * t if j == i else y for j, y in enumerate(x)] for s in (1, -1))
        diff = float(loss(up) - loss(down)) / 2e-4
        tol = u * want[name].abs() + 2 * (u + E) * want[name + "_abs"] + 40 * 2.0 ** -25 * 4
        assert abs(float((grads[i].double() * t).sum()) - diff) <= float((tol * t.abs()).sum()) + 1e-5, name
