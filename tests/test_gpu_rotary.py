"""Rotary positions by token index and the norms of query and key heads, against the formulas in 64 bits.

Tolerances.  Everything is computed in fp32 from an angle that fp64 reduced and one rounding to fp32 (2^-25 of half a turn,
9.4e-8 radians), cosines and sines good to 2 ulp (2.4e-7), three roundings of the turn: below 6e-7 of the pair's length.  A
norm adds half the error of a sum of d squares (at most 2V + 5 roundings in a row, V <= 8) and a reciprocal root good to
2 ulp: below 1e-6.  The store rounds by at most eps/2 of the value.  So: eps/2 |y| + F * (length), with F = 6e-7 for the
rotation, 2e-6 with the norm and 4e-6 for the difference of two such terms in the backward."""
import math

import pytest
import torch

from paper_2604_16429_b200 import binding as mb
from tests import gpu_util as G

pytestmark = pytest.mark.gpu
DT = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}


def make(B, H, Hkv, N, d, dtype, layout, seed):
    g = torch.Generator().manual_seed(seed)

    def one(heads):
        x = torch.randn((B, N, heads, d) if layout == "bnhd" else (B, heads, N, d), generator=g).to(DT[dtype]).cuda()
        return x.transpose(1, 2) if layout == "bnhd" else x

    return one(H), one(Hkv), g


def turn64(x, pos, rp, back=False):
    """The rotation of x [B,h,N,d] (fp64) by the definition, channel by channel."""
    r, i = rp.rot, torch.arange(rp.rot // 2, device=x.device)
    f = mb.rotary_freqs(rp, "cpu").to(x.device)
    a = pos.double().reshape(-1, 1, pos.shape[-1], 1) * f * (-1 if back else 1)
    lo, hi = (i, i + r // 2) if rp.half else (2 * i, 2 * i + 1)
    y = x.clone()
    y[..., lo] = rp.amplitude * (x[..., lo] * a.cos() - x[..., hi] * a.sin())
    y[..., hi] = rp.amplitude * (x[..., lo] * a.sin() + x[..., hi] * a.cos())
    return y


def near(got, want, factor, length, what):
    """|got - want| <= eps/2 |want| + factor * length (the length of the row that takes part)"""
    tol = torch.finfo(got.dtype).eps / 2 * want.abs() * (1 + 1e-6) + factor * length
    if got.dtype == torch.float16:
        tol = tol + 2.0 ** -25  # half a step of its subnormal numbers
    off = ((got.double() - want).abs() - tol).max()
    assert not torch.isnan(got).any() and off <= 0, f"{what}: over by {off:.3g}"


def length(x):
    return x.abs().amax(-1, keepdim=True) * math.sqrt(2)


CASES = [  # B, H, Hkv, N, d, rot, half, dtype, layout
    (1, 1, 1, 1, 64, 64, True, "bf16", "bhnd"),
    (2, 4, 2, 7, 64, 64, False, "bf16", "bnhd"),
    (3, 12, 3, 130, 64, 32, True, "fp16", "bhnd"),
    (1, 16, 4, 65, 128, 128, True, "bf16", "bnhd"),
    (2, 6, 2, 33, 128, 34, False, "fp16", "bnhd"),
    (2, 5, 1, 19, 80, 48, True, "bf16", "bhnd"),      # ten pieces of a row on lanes for sixteen
    (1, 3, 3, 40, 96, 2, False, "fp32", "bnhd"),
    (2, 8, 8, 21, 256, 256, True, "fp32", "bhnd"),
    (1, 40, 2, 9, 256, 256, False, "bf16", "bhnd"),
    (5, 2, 1, 3, 16, 16, True, "fp32", "bnhd"),
    (1, 33, 11, 5, 16, 10, False, "bf16", "bhnd"),
    (64, 16, 4, 1, 128, 128, True, "bf16", "bnhd"),
]


@pytest.mark.parametrize("case", CASES, ids=str)
@pytest.mark.parametrize("inverse", [False, True])
def test_rotation(case, inverse):
    B, H, Hkv, N, d, rot, half, dtype, layout = case
    q, k, g = make(B, H, Hkv, N, d, dtype, layout, seed=N + d)
    rp = mb.RotaryParams(d=d, rot_dim=rot, half=half, amplitude=1.25)
    pos = torch.randint(-5, 100000, (B, N), generator=g).cuda()
    fr = mb.rotary_freqs(rp)
    gq, gk = G.Guarded((B, H, N, d), q.dtype, fill=float("nan")), G.Guarded((B, Hkv, N, d), q.dtype, fill=float("nan"))
    mb.mosaic_bsa_rotary(rp, q, k, pos, fr, inverse=inverse, q_out=gq.t, k_out=gk.t)
    for x, y in ((q, gq), (k, gk)):
        y.check("out")
        near(y.t, turn64(x.double(), pos, rp, inverse), 6e-7 * 1.25, length(x.double()), "rotation")
        assert torch.equal(y.t[..., rot:], x[..., rot:])  # channels that do not turn come through as they are


@pytest.mark.parametrize("far", [0, 1 << 17, 1 << 24, 10 ** 9, -(10 ** 9)])
def test_far_positions_keep_their_angle(far):
    q, k, _ = make(1, 2, 1, 50, 64, "fp32", "bhnd", seed=1)
    rp = mb.RotaryParams(d=64, half=True)
    pos = far + torch.arange(50).cuda()
    qo, ko = mb.mosaic_bsa_rotary(rp, q, k, pos, mb.rotary_freqs(rp))
    # two fp64 roundings of the angle (and the reference's one): 3 * 2^-53 * 1e9 = 3.4e-7 radians at the farthest
    near(qo, turn64(q.double(), pos, rp), 6e-7 + 3 * 2.0 ** -53 * abs(far), length(q.double()), "q")
    near(ko, turn64(k.double(), pos, rp), 6e-7 + 3 * 2.0 ** -53 * abs(far), length(k.double()), "k")


def test_products_depend_on_the_distance_alone():
    q, k, _ = make(1, 1, 1, 40, 64, "fp32", "bhnd", seed=3)
    q, k = q[:, :, :1].expand(1, 1, 40, 64), k[:, :, :1].expand(1, 1, 40, 64)  # (inputs may be broadcast)
    rp = mb.RotaryParams(d=64)
    pos, fr = torch.arange(40).cuda(), mb.rotary_freqs(rp)
    a, b = mb.mosaic_bsa_rotary(rp, q, k, pos, fr)
    z = a[0, 0].double() @ b[0, 0].double().T
    for shift in (0, 1, 7):
        diag = torch.diagonal(z, shift)
        # 64 products of elements that are off by 6e-7 of their pair each
        assert (diag - diag[0]).abs().max() <= 2 * 6e-7 * float(q[0, 0, 0].double().norm() * k[0, 0, 0].double().norm()) * 2


def test_in_place_shared_positions_and_slices():
    B, H, Hkv, N, d = 2, 4, 2, 37, 64
    g = torch.Generator().manual_seed(5)
    fused = torch.randn((B, N, H + 2 * Hkv, d), generator=g).bfloat16().cuda()
    before = fused.clone()
    q, k = fused[:, :, :H].transpose(1, 2), fused[:, :, H:H + Hkv].transpose(1, 2)
    rp = mb.RotaryParams(d=d, rot_dim=32, half=True)
    pos = torch.arange(N).cuda()
    q0, k0 = q.double(), k.double()
    mb.mosaic_bsa_rotary(rp, q, k, pos, mb.rotary_freqs(rp), q_out=q, k_out=k)
    near(q, turn64(q0, pos, rp), 6e-7, length(q0), "q")
    near(k, turn64(k0, pos, rp), 6e-7, length(k0), "k")
    assert torch.equal(fused[:, :, H + Hkv:], before[:, :, H + Hkv:])  # the values beside them are untouched


def norm64(x, w, eps):
    return x * torch.rsqrt((x * x).mean(-1, keepdim=True) + eps) * w.double()


@pytest.mark.parametrize("case", CASES, ids=str)
def test_norm_and_rotation(case):
    B, H, Hkv, N, d, rot, half, dtype, layout = case
    q, k, g = make(B, H, Hkv, N, d, dtype, layout, seed=N + d + 1)
    q *= 7.0
    k[:, :, N // 2] *= 1e-3  # where eps counts
    rp = mb.RotaryParams(d=d, rot_dim=rot, half=half)
    pos = torch.randint(0, 5000, (B, N), generator=g).cuda()
    wq, wk = (1 + 0.3 * torch.randn(d, generator=g)).cuda(), (1 + 0.3 * torch.randn(d, generator=g)).cuda()
    gq, gk = G.Guarded((B, H, N, d), q.dtype, fill=float("nan")), G.Guarded((B, Hkv, N, d), q.dtype, fill=float("nan"))
    mb.mosaic_bsa_qk_norm(rp, q, k, wq, wk, pos, mb.rotary_freqs(rp), eps=1e-5, q_out=gq.t, k_out=gk.t)
    for x, w, y in ((q, wq, gq), (k, wk, gk)):
        y.check("out")
        n = norm64(x.double(), w, 1e-5)
        near(y.t, turn64(n, pos, rp), 2e-6, length(n), "norm and rotation")


def test_norm_alone_and_zero_rows():
    q, k, g = make(2, 4, 2, 9, 96, "bf16", "bhnd", seed=2)
    q[:, 1] = 0
    w = torch.ones(96, device="cuda")
    rp = mb.RotaryParams(d=96, rot_dim=0)
    qo, ko = mb.mosaic_bsa_qk_norm(rp, q, k, w, w)
    near(qo, norm64(q.double(), w, 1e-6), 2e-6, length(norm64(q.double(), w, 1e-6)), "q")
    assert (qo[:, 1] == 0).all()
    d_q, d_k = torch.randn_like(q), torch.randn_like(k)
    dq, dk, dwq, dwk = mb.mosaic_bsa_qk_norm_bwd(rp, q, k, w, w, None, None, d_q, d_k)
    want = d_q.double()[:, 1] / math.sqrt(1e-6)  # a zero row's norm is a factor of 1 / sqrt(eps)
    near(dq[:, 1], want, 4e-6, length(want), "gradient of a zero row")


def grads64(x, w, dy, pos, rp, eps):
    g = turn64(dy.double(), pos, rp, back=True)
    x = x.double()
    r = torch.rsqrt((x * x).mean(-1, keepdim=True) + eps)
    gw = g * w.double()
    back = r * r * (gw * x).mean(-1, keepdim=True)
    return r * (gw - x * back), (g * x * r).sum((0, 1, 2)), length(r * gw) + length(r * x) * length(r * gw), (g * x * r).abs().sum((0, 1, 2))


@pytest.mark.parametrize("case", CASES + [(2, 8, 2, 3000, 128, 128, True, "bf16", "bnhd")], ids=str)
def test_gradients(case):
    B, H, Hkv, N, d, rot, half, dtype, layout = case
    q, k, g = make(B, H, Hkv, N, d, dtype, layout, seed=N + d + 2)
    rp = mb.RotaryParams(d=d, rot_dim=rot, half=half, amplitude=0.75)
    pos = torch.randint(0, 5000, (B, N), generator=g).cuda()
    wq, wk = (1 + 0.3 * torch.randn(d, generator=g)).cuda(), (1 + 0.3 * torch.randn(d, generator=g)).cuda()
    d_q, d_k, _ = make(B, H, Hkv, N, d, dtype, "bnhd", seed=N + d + 3)
    outs = [G.Guarded(s, t, fill=float("nan")) for s, t in (((B, H, N, d), q.dtype), ((B, Hkv, N, d), q.dtype), ((d,), torch.float32),
                                                            ((d,), torch.float32))]
    ws = G.Guarded((mb.qk_norm_workspace_bytes(rp, q, k),), torch.uint8)
    args = dict(zip(("dq", "dk", "dwq", "dwk"), (o.t for o in outs)), ws=ws.t, eps=1e-5)
    mb.mosaic_bsa_qk_norm_bwd(rp, q, k, wq, wk, pos, mb.rotary_freqs(rp), d_q, d_k, **args)
    ws.check("workspace")
    for (x, w, dy), dx, dw in (((q, wq, d_q), outs[0], outs[2]), ((k, wk, d_k), outs[1], outs[3])):
        dx.check("dx"); dw.check("dw")
        want, dw_want, size, terms = grads64(x, w, dy, pos, rp, 1e-5)
        near(dx.t, want, 4e-6, size, "dx")
        # fp32 sums: at most 80 additions in a row in a lane at these sizes, 5 in the warp, 8 in the CTA, 19 + 5 over CTAs, and
        # 4e-6 of every term: below 1.2e-5 of the terms' sum
        assert ((dw.t.double() - dw_want).abs() <= 1.2e-5 * terms + 1e-30).all(), "dw"
    first = [o.t.clone() for o in outs]
    mb.mosaic_bsa_qk_norm_bwd(rp, q, k, wq, wk, pos, mb.rotary_freqs(rp), d_q, d_k, **args)
    assert all(torch.equal(a, o.t) for a, o in zip(first, outs))  # the same bits again


def test_gradients_against_differences():
    """Central differences of the 64-bit forward, in a few directions: the step h leaves h^2 / 6 of a third derivative of
    order one and 2^-53 / h of rounding."""
    q, k, g = make(1, 2, 1, 5, 64, "fp32", "bhnd", seed=11)
    rp = mb.RotaryParams(d=64, rot_dim=32, half=True)
    pos = torch.arange(5).cuda() * 17
    wq, wk = (1 + 0.3 * torch.randn(64, generator=g)).cuda(), (1 + 0.3 * torch.randn(64, generator=g)).cuda()
    d_q, d_k, _ = make(1, 2, 1, 5, 64, "fp32", "bhnd", seed=12)
    dq, dk, dwq, dwk = mb.mosaic_bsa_qk_norm_bwd(rp, q, k, wq, wk, pos, mb.rotary_freqs(rp), d_q, d_k)
    loss = lambda x, w, dy: (turn64(norm64(x, w, 1e-6), pos, rp) * dy.double()).sum()  # noqa: E731
    h = 1e-5
    for x, w, dy, dx, dw in ((q, wq, d_q, dq, dwq), (k, wk, d_k, dk, dwk)):
        for s in range(3):
            u = torch.randn(x.shape, generator=g).double().cuda()
            v = torch.randn(64, generator=g).double().cuda()
            a = (loss(x.double() + h * u, w, dy) - loss(x.double() - h * u, w, dy)) / (2 * h)
            b = (loss(x.double(), w.double() + h * v, dy) - loss(x.double(), w.double() - h * v, dy)) / (2 * h)
            # 4e-6 of every term of a sum of `numel` products
            assert abs(float((dx.double() * u).sum() - a)) <= 4e-6 * float((dx.double().abs() * u.abs()).sum()) * 2 + 1e-6
            assert abs(float((dw.double() * v).sum() - b)) <= 1.2e-5 * float((dw.double().abs() * v.abs()).sum()) * 2 + 1e-6


def test_on_another_stream_and_captured():
    q, k, g = make(2, 4, 2, 100, 64, "bf16", "bhnd", seed=21)
    rp = mb.RotaryParams(d=64, half=True)
    pos, fr = torch.arange(100).cuda(), mb.rotary_freqs(rp)
    w = torch.ones(64, device="cuda")
    want = mb.mosaic_bsa_qk_norm(rp, q, k, w, w, pos, fr)
    grads = mb.mosaic_bsa_qk_norm_bwd(rp, q, k, w, w, pos, fr, q, k)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    got = mb.mosaic_bsa_qk_norm(rp, q, k, w, w, pos, fr, stream=side)
    got2 = mb.mosaic_bsa_qk_norm_bwd(rp, q, k, w, w, pos, fr, q, k, stream=side)
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(want + grads, got + got2))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = mb.mosaic_bsa_qk_norm(rp, q, k, w, w, pos, fr) + mb.mosaic_bsa_qk_norm_bwd(rp, q, k, w, w, pos, fr, q, k)
    for t in out:
        t.fill_(float("nan"))
    for _ in range(2):
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(want + grads, out))


def test_refusals_of_the_binding():
    q, k, _ = make(2, 4, 2, 10, 64, "bf16", "bhnd", seed=31)
    rp = mb.RotaryParams(d=64)
    pos, fr, w = torch.arange(10).cuda(), mb.rotary_freqs(rp), torch.ones(64, device="cuda")
    bad = [
        dict(q=q.double()), dict(k=k.half()), dict(q=q[..., ::2]), dict(k=k[:, :, :9]), dict(pos=pos.int()), dict(pos=pos[:9]),
        dict(pos=pos.cpu()), dict(freqs=fr.float()), dict(freqs=fr[:31]), dict(q_out=q.float()), dict(k_out=k[:1].expand_as(k)),
        dict(q=q[0]), dict(q_out=torch.empty_like(q).transpose(2, 3)),
    ]
    for kw in bad:
        args = {**dict(q=q, k=k, pos=pos, freqs=fr), **kw}
        with pytest.raises(ValueError):
            mb.mosaic_bsa_rotary(rp, **args)
    with pytest.raises(ValueError):
        mb.mosaic_bsa_qk_norm(rp, q, k, w.bfloat16(), w, pos, fr)
    with pytest.raises(mb.MosaicError) as e:  # a row that does not start on 16 bytes
        shifted = torch.zeros(2 * 4 * 10 * 64 + 4, dtype=torch.bfloat16, device="cuda")[4:].view(2, 4, 10, 64)
        mb.mosaic_bsa_rotary(rp, shifted, k, pos, fr)
    assert e.value.code == -4
