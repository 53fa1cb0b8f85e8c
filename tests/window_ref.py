"""Sliding-window attention with sinks in 64 bits, from the definition, a batch member and head at a time."""
import math

import torch


def mask(pos, nk, window, sinks):
    j = torch.arange(nk, device=pos.device)
    p = pos[:, None]
    return (j <= p) & ((p - j < window) | (j < sinks))


def attention(q, k, v, window, sinks, scale=0.0, q_len=None, k_len=None, d_o=None):
    """o, lse (rows that do not exist: NaN), and with d_o also dq, dk, dv; inputs [B, heads, tokens, d] of any type."""
    B, H, Nq, d = q.shape
    Hkv, Nk = k.shape[1:3]
    sc = scale if scale > 0 else 1 / math.sqrt(d)
    nan = lambda *s: torch.full(s, math.nan, dtype=torch.float64, device=q.device)  # noqa: E731
    out = {"o": nan(B, H, Nq, d), "lse": nan(B, H, Nq), "p_abs": nan(B, H, Nq, d)}
    if d_o is not None:
        out.update(dq=nan(B, H, Nq, d), dk=nan(B, Hkv, Nk, d), dv=nan(B, Hkv, Nk, d),
                   dq_abs=nan(B, H, Nq, d), dk_abs=nan(B, Hkv, Nk, d), dv_abs=nan(B, Hkv, Nk, d))
    for b in range(B):
        ql = Nq if q_len is None else int(q_len[b])
        kl = Nk if k_len is None else int(k_len[b])
        see = mask(torch.arange(ql, device=q.device) + kl - ql, kl, window, sinks)
        if d_o is not None:
            for n in ("dk", "dv", "dk_abs", "dv_abs"):
                out[n][b, :, :kl] = 0
        for h in range(H):
            x, y, z = q[b, h, :ql].double(), k[b, h * Hkv // H, :kl].double(), v[b, h * Hkv // H, :kl].double()
            s = (x @ y.T * sc).masked_fill(~see, -math.inf)
            lse = torch.logsumexp(s, -1) if kl else s.new_full((ql,), -math.inf)
            p = torch.exp(s - lse[:, None]).masked_fill(~see, 0.0)
            out["o"][b, h, :ql], out["lse"][b, h, :ql] = p @ z, lse
            out["p_abs"][b, h, :ql] = p @ z.abs()
            if d_o is not None:
                g = d_o[b, h, :ql].double()
                o = out["o"][b, h, :ql]
                dp = g @ z.T
                D = (g * o).sum(-1, keepdim=True)
                ds = p * (dp - D) * sc
                # what a rounding of P, of dS and of O in D can move: sums of the magnitudes
                ds_abs = p * (dp.abs() + D.abs()) * sc
                D_abs = p * (g.abs() * out["p_abs"][b, h, :ql]).sum(-1, keepdim=True) * sc
                hk = h * Hkv // H
                out["dq"][b, h, :ql], out["dq_abs"][b, h, :ql] = ds @ y, (ds_abs + D_abs) @ y.abs()
                out["dk"][b, hk, :kl] += ds.T @ x
                out["dk_abs"][b, hk, :kl] += (ds_abs + D_abs).T @ x.abs()
                out["dv"][b, hk, :kl] += p.T @ g
                out["dv_abs"][b, hk, :kl] += p.T @ g.abs()
    return out
