"""Channels from rot_dim on: what they hold, whatever it is, comes through and reaches no other channel."""
import math

import pytest
import torch

from paper_2604_16429_b200 import binding as mb
from tests import test_gpu_rotary as R

pytestmark = pytest.mark.gpu
ODD = (math.inf, -math.inf, math.nan, -0.0, 0.0)

CASES = [  # d, rot, half
    (64, 32, True), (64, 32, False), (64, 2, False), (128, 34, False), (128, 126, False), (80, 48, True), (80, 38, False), (256, 16, True),
    (256, 130, False), (16, 6, False),
]


def bits(x):
    return x.contiguous().view(torch.int32 if x.dtype == torch.float32 else torch.int16)


@pytest.mark.parametrize("case", CASES, ids=str)
@pytest.mark.parametrize("dtype", ["bf16", "fp16", "fp32"])
@pytest.mark.parametrize("inverse", [False, True])
def test_rotation_copies_them_bit_for_bit(case, dtype, inverse):
    d, rot, half = case
    q, k, g = R.make(2, 6, 2, 37, d, dtype, "bnhd", seed=d + rot)
    clean_q, clean_k = q.clone(), k.clone()
    for x in (q, k):
        for i in range(rot, d):  # each channel has each of them in some row, and ordinary numbers in others
            for j, odd in enumerate(ODD):
                x[:, (i + j) % x.shape[1], (3 * i + 5 * j) % 37, i] = odd
        x[0, 0, 0, rot:] = bits(x)[0, 0, 0, rot:].random_(generator=torch.Generator("cuda").manual_seed(1)).view(x.dtype)  # any bits at all
    rp = mb.RotaryParams(d=d, rot_dim=rot, half=half, amplitude=1.5)
    pos, fr = torch.arange(37, device="cuda") + 99, mb.rotary_freqs(rp)
    got = mb.mosaic_bsa_rotary(rp, q, k, pos, fr, inverse=inverse)
    want = mb.mosaic_bsa_rotary(rp, clean_q, clean_k, pos, fr, inverse=inverse)
    for x, y, z in zip((q, k), got, want):
        assert torch.equal(bits(y)[..., rot:], bits(x)[..., rot:])
        assert torch.equal(bits(y)[..., :rot], bits(z)[..., :rot])


@pytest.mark.parametrize("case", CASES, ids=str)
@pytest.mark.parametrize("dtype", ["bf16", "fp16", "fp32"])
def test_norm_does_not_mix_them(case, dtype):
    """A weight that is infinite or no number makes its own channel so, and in the backward an incoming gradient its own channel's
    weight gradient; the row's mean takes every channel, so the gradients of the rows are not looked at."""
    d, rot, half = case
    q, k, g = R.make(2, 6, 2, 37, d, dtype, "bnhd", seed=d + rot + 1)
    rp = mb.RotaryParams(d=d, rot_dim=rot, half=half)
    pos, fr = torch.arange(37, device="cuda") + 99, mb.rotary_freqs(rp)
    w = (1 + 0.3 * torch.randn(d, generator=g)).cuda()
    plain = mb.mosaic_bsa_qk_norm(rp, q, k, w, w, pos, fr)
    grads = mb.mosaic_bsa_qk_norm_bwd(rp, q, k, w, w, pos, fr, q, k)
    for at in {rot, rot + 1, d - 1}:
        rest = torch.arange(d, device="cuda") != at
        for odd in (math.inf, math.nan):
            bad = w.clone()
            bad[at] = odd
            for x, y, z in zip((q, k), plain, mb.mosaic_bsa_qk_norm(rp, q, k, bad, bad, pos, fr)):
                assert torch.equal(bits(y)[..., rest], bits(z)[..., rest])
                assert not torch.isfinite(z[..., at][x[..., at] != 0]).any()
            dq, dk = q.clone(), k.clone()
            dq[0, 0, 5, at] = dk[0, 0, 5, at] = odd
            for a, b in zip(grads[2:], mb.mosaic_bsa_qk_norm_bwd(rp, q, k, w, w, pos, fr, dq, dk)[2:]):
                assert torch.equal(bits(a)[rest], bits(b)[rest]) and not torch.isfinite(b[at])
