"""Inputs on which one rounding of the weights shows in the sinks' gradients, their exact gradients, and what a backward that rounds P
or dS once to 16 bits would give.

All keys are zero, so every score is 0 and a row that sees n keys weighs each by 1/n.  n = 255 (2047 in fp16) for all rows but the
first, whose q and dO are zero: 1/n lies just above the middle between two 16-bit numbers, so that its rounding is off by 0.99 u of it,
in every row to the same side.  The values are zero but for channel 0 of the sinks, +1 and -1 in turn, and dO is 1 there: o is zero,
dP_ij = +-1, and dS_ij = +-1/n rounds like the weight.  The other channels of dO and all of q are positive, so no sum cancels."""
import torch

SINKS = 8


def inputs(d, dtype, device="cpu", H=4, Hkv=2):
    """wp's window, and q, k, v, d_o"""
    seen, N = (255, 1500) if dtype == torch.bfloat16 else (2047, 2447)
    g = torch.Generator().manual_seed(d)
    q = (0.5 + torch.rand((1, H, N, d), generator=g)).to(dtype)
    k, v = torch.zeros((1, Hkv, N, d), dtype=dtype), torch.zeros((1, Hkv, N, d), dtype=dtype)
    v[:, :, :SINKS:2, 0], v[:, :, 1:SINKS:2, 0] = 1, -1
    d_o = (0.5 + torch.rand((1, H, N, d), generator=g)).to(dtype)
    d_o[..., 0] = 1
    q[:, :, :seen - 1] = d_o[:, :, :seen - 1] = 0
    return seen - SINKS, [x.to(device) for x in (q, k, v, d_o)]


def gradients(window, q, k, v, d_o, once=()):
    """(dk, dv) [1, Hkv, SINKS, d] of the sinks in 64 bits; `once`: which of "P", "dS" are rounded to the inputs' type, the results too
    then."""
    _, H, N, d = q.shape
    Hkv, dtype = k.shape[1], q.dtype
    p = torch.arange(N, device=q.device)
    n = torch.minimum(p + 1, torch.full_like(p, window + SINKS)).double()
    sees = (torch.arange(SINKS, device=q.device) <= p[:, None]).double()
    P = sees / n[:, None]
    sign = v[0, 0, :SINKS, 0].double()
    dS = P * sign  # (in the rows that count dO_i . o_i is zero)
    if "P" in once:
        P = P.to(dtype).double()
    if "dS" in once:
        dS = dS.to(dtype).double()
    group = lambda x: x.double().view(1, Hkv, H // Hkv, N, d).sum(2)  # noqa: E731
    dk, dv = d ** -0.5 * torch.einsum("ij,bhid->bhjd", dS, group(q)), torch.einsum("ij,bhid->bhjd", P, group(d_o))
    return (dk.to(dtype).double(), dv.to(dtype).double()) if once else (dk, dv)


def tolerance(window, q, want):
    """One rounding of the result (u), weights as two 16-bit numbers (u^2), an exponential good to 4e-6 and twice as much of its
    logarithm, and fp32 sums of one addition a row that counts and head of the group, each off by at most 2^-23 of a sum whose terms
    have one sign."""
    u = torch.finfo(q.dtype).eps / 2
    return want.abs() * (u + u * u + 1.2e-5 + 2 * (q.shape[2] - window - SINKS + 1) * 2.0 ** -23)
