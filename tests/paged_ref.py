"""A paged cache and attention over it in 64 bits, from the definition: token by token, member by member, head by head."""
import math

import torch


def place(table, b, j, page, pages):
    """(page, slot) of token j of member b, or None where there is none"""
    if j < 0 or j // page >= table.shape[1]:
        return None
    t = int(table[b, j // page])
    return (t, j % page) if 0 <= t < pages else None


def lengths(B, T, cap, k_len, q_len):
    """(tokens, new tokens) of every member, clamped"""
    kl = [min(max(int(x), 0), cap) for x in k_len]
    ql = [T] * B if q_len is None else [min(max(int(x), 0), T) for x in q_len]
    return kl, ql


def rotate(x, pos, freqs, half, amplitude=1.0):
    """A row [.., d] in 64 bits at one position"""
    y = x.clone()
    r = 2 * len(freqs)
    for i in range(r // 2):
        a, b = (i, i + r // 2) if half else (2 * i, 2 * i + 1)
        c, s = math.cos(pos * freqs[i]) * amplitude, math.sin(pos * freqs[i]) * amplitude
        y[..., a], y[..., b] = x[..., a] * c - x[..., b] * s, x[..., a] * s + x[..., b] * c
    return y


def gather(pool, table, b, h, n, page):
    """The first n tokens of member b's head h in 64 bits, and which of them are there"""
    pages = pool.shape[0]
    out = torch.zeros((n, pool.shape[-1]), dtype=torch.float64, device=pool.device)
    there = torch.zeros(n, dtype=torch.bool, device=pool.device)
    for i in range(-(-n // page)):
        t, m = int(table[b, i]), min(page, n - i * page)
        if 0 <= t < pages:
            out[i * page:i * page + m] = pool[t, h, :m].double()
            there[i * page:i * page + m] = True
    return out, there


def attention(q, k_pages, v_pages, table, k_len, window=0, sinks=0, scale=0.0, q_len=None, prefix=None, prefix_len=0):
    """o, lse and p_abs (sum of weight times magnitude of the values); rows that do not exist: NaN"""
    B, H, T, d = q.shape
    pages, Hkv, page, _ = k_pages.shape
    sc = scale if scale > 0 else 1 / math.sqrt(d)
    kls, qls = lengths(B, T, table.shape[1] * page, k_len, q_len)
    nan = lambda *s: torch.full(s, math.nan, dtype=torch.float64, device=q.device)  # noqa: E731
    out = {"o": nan(B, H, T, d), "lse": nan(B, H, T), "p_abs": nan(B, H, T, d)}
    for b in range(B):
        kl, ql = kls[b], qls[b]
        for hk in range(Hkv):
            k, there = gather(k_pages, table, b, hk, kl, page)
            v, _ = gather(v_pages, table, b, hk, kl, page)
            p = torch.arange(kl - ql, kl, device=q.device)[:, None]
            j = torch.arange(kl, device=q.device)
            see = (j <= p) & there
            if window:
                see &= (p - j < window) | (j < sinks)
            if prefix is not None:
                kp, held = gather(k_pages, prefix[None], 0, hk, prefix_len, page)
                vp, _ = gather(v_pages, prefix[None], 0, hk, prefix_len, page)
                k, v, see = torch.cat((kp, k)), torch.cat((vp, v)), torch.cat((held.expand(ql, -1), see), 1)
            for h in range(hk * H // Hkv, (hk + 1) * H // Hkv):
                s = (q[b, h, :ql].double() @ k.T * sc).masked_fill(~see, -math.inf)
                lse = torch.logsumexp(s, -1) if len(k) else s.new_full((ql,), -math.inf)
                w = torch.exp(s - lse[:, None]).masked_fill(~see, 0.0)
                out["o"][b, h, :ql], out["lse"][b, h, :ql], out["p_abs"][b, h, :ql] = w @ v, lse, w @ v.abs()
    return out
