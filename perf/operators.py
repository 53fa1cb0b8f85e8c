"""The operators on queries, keys and values of token sequences, as cases that can be timed and compared.

* ``rotary``       one-dimensional rotary positions of Q and K: interleaved or half pairs, the whole head or its first
                   channels, frequencies of a scaled context; ``inverse`` is the transpose that a backward applies
* ``qk_norm``      root-mean-square norm of every query and key head, its weight, and the rotation, in one pass
* ``qk_norm_bwd``  the gradients of that pass: of Q, K and both weights
* ``window``       causal attention inside a sliding window whose first tokens (sinks) stay visible
* ``window_train`` the same with its backward
* ``decode``       the same for one new token per sequence, over a linear or a rolling cache

``own`` says which side ``run`` takes: elementary torch operations in 32 bits (angles in 64), or this library's calls.
"""
from __future__ import annotations

import math

import numpy as np
import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}
EPS = 1e-6


def _rot(name, op, B, H, Hkv, N, d, rot, **over):
    c = dict(name=name, op=op, B=B, H=H, Hkv=Hkv, N=N, d=d, rot=rot, half=True, dtype="bf16", layout="bnhd", scaling="plain",
             factor=1.0, far=0, inverse=False)
    c.update(over)
    return c


def _win(name, op, B, H, Hkv, Nq, Nk, d, window, sinks, **over):
    c = dict(name=name, op=op, B=B, H=H, Hkv=Hkv, Nq=Nq, Nk=Nk, d=d, window=window, sinks=sinks, dtype="bf16", layout="bnhd",
             ragged=False, rolling=False)
    c.update(over)
    return c


def listed():
    return [
        # one new token of 64 sequences, far into a context that by-parts scaling stretched eightfold: the smallest call
        _rot("rotary_decode", "rotary", 64, 16, 4, 1, 128, 128, scaling="parts", factor=8.0, far=60000),
        # a training batch, a quarter of the head turned in adjacent pairs, as the projection lays its heads out
        _rot("rotary_partial", "rotary", 2, 16, 4, 8192, 128, 32, half=False, dtype="fp16"),
        # the backward of the rotation for a batch of odd length, frequencies stretched by bands, the library's own layout
        _rot("rotary_inverse_odd", "rotary", 3, 12, 3, 4099, 64, 64, scaling="bands", factor=4.0, layout="bhnd", inverse=True),
        # queries and keys of a layer of 12288 tokens and 16 heads, inference
        _rot("qk_norm_12288", "qk_norm", 1, 16, 16, 12288, 64, 64, half=False, layout="bhnd"),
        # the gradients of that pass in a training batch with grouped-query heads
        _rot("qk_norm_bwd_train", "qk_norm_bwd", 2, 16, 4, 8192, 128, 128),
        # a short odd batch in 32 bits, three quarters of the head turned
        _rot("qk_norm_bwd_odd", "qk_norm_bwd", 3, 6, 2, 1021, 64, 48, half=False, dtype="fp32", layout="bhnd"),
        # the prompt of one sequence
        _win("window_8192", "window", 1, 16, 4, 8192, 8192, 128, 1024, 4),
        # the next chunk of five prompts of different lengths, each behind what its cache holds already
        _win("window_chunk_ragged", "window", 5, 12, 3, 1021, 4099, 64, 509, 7, dtype="fp16", ragged=True, layout="bhnd"),
        # a layer of 49152 tokens in training: a long sequence, a wide window
        _win("window_train_49152", "window_train", 1, 12, 3, 49152, 49152, 64, 2048, 16),
        # a layer of a training batch
        _win("window_train_4096", "window_train", 2, 16, 4, 4096, 4096, 128, 1024, 4),
        # one token of one sequence over a long linear cache: latency
        _win("decode_one", "decode", 1, 16, 4, 1, 16384, 128, 4096, 4, layout="bhnd"),
        # one token of 64 streams of different lengths, each over a rolling cache that forgets what left the window
        _win("decode_rolling", "decode", 64, 16, 4, 1, 4100, 128, 4096, 4, ragged=True, rolling=True, layout="bhnd"),
    ]


def _log(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    """Any operator, type, layout and head grouping; lengths from one token to 32768 (window attention to 16384), caches to
    32768; at most half a million (token, query head) pairs per call."""
    op = rng.choice(["rotary", "qk_norm", "qk_norm_bwd", "window", "window", "window_train", "window_train", "decode"])
    d = rng.choice([64, 128])
    Hkv = rng.choice([1, 2, 3, 4, 8])
    H = Hkv * rng.choice([1, 2, 3, 4, 6, 8])
    layout = rng.choice(["bhnd", "bnhd"])
    if op in ("rotary", "qk_norm", "qk_norm_bwd"):
        N = _log(rng, 1, 32768)
        B = _log(rng, 1, max(1, min(32, (1 << 19) // (H * N))))
        rot = rng.choice([d, d, d // 2, d // 4])
        scaling = rng.choice(["plain", "linear", "base", "parts", "bands"])
        c = _rot("", op, B, H, Hkv, N, d, rot, half=rng.random() < 0.5, dtype=rng.choice(["bf16", "bf16", "fp16", "fp32"]),
                 layout=layout, scaling=scaling, factor=1.0 if scaling == "plain" else rng.choice([2.0, 4.0, 8.0]),
                 far=rng.choice([0, 0, _log(rng, 1, 1 << 20)]), inverse=op == "rotary" and rng.random() < 0.4)
    elif op == "decode":
        Nk = _log(rng, 16, 32768)
        B = _log(rng, 1, max(1, min(64, (1 << 20) // (Hkv * Nk))))
        sinks = rng.randint(0, min(64, Nk // 2))
        rolling = rng.random() < 0.4
        window = Nk - sinks if rolling else _log(rng, 1, Nk)
        c = _win("", op, B, H, Hkv, 1, Nk, d, window, sinks, dtype=rng.choice(["bf16", "fp16"]), layout=layout,
                 ragged=rng.random() < 0.5, rolling=rolling)
    else:
        N = _log(rng, 1, 16384)
        B = _log(rng, 1, max(1, min(8, (1 << (19 if op == "window" else 18)) // (H * N))))
        ragged = rng.random() < 0.4
        more = _log(rng, 1, 4096) if ragged else 0
        c = _win("", op, B, H, Hkv, N, N + more, d, _log(rng, 1, 4096), rng.randint(0, 64), dtype=rng.choice(["bf16", "fp16"]),
                 layout=layout, ragged=ragged)
    del c["name"]
    return c


# ---------------------------------------------------------------------------------------------------- inputs
def _freqs(c):
    """Radians per position of every turned pair, in 64 bits."""
    rot, theta, length, fast, slow = c["rot"], 10000.0, 8192.0, 32.0, 1.0
    i = np.arange(rot // 2, dtype=np.float64)
    if c["scaling"] == "base" and rot > 2:  # the base grows until the slowest pair is slowed by the factor
        theta *= c["factor"] ** (rot / (rot - 2))
    f = theta ** (-2.0 * i / rot)
    if c["scaling"] == "linear":
        f = f / c["factor"]
    elif c["scaling"] == "parts":  # a ramp over the pairs between those that turn `fast` and `slow` times in the length
        at = lambda turns: rot * math.log(length / (2 * math.pi * turns)) / (2 * math.log(theta))  # noqa: E731
        lo, hi = max(math.floor(at(fast)), 0), min(math.ceil(at(slow)), rot - 1)
        ramp = np.clip((i - lo) / max(hi - lo, 1e-3), 0.0, 1.0)
        f = f * (1 - ramp) + f / c["factor"] * ramp
    elif c["scaling"] == "bands":  # a ramp over the number of turns itself
        keep = np.clip((length * f / (2 * math.pi) - slow) / (fast - slow), 0.0, 1.0)
        f = f * keep + f / c["factor"] * (1 - keep)
    return f


def _amplitude(c):
    return 0.1 * math.log(c["factor"]) + 1.0 if c["scaling"] == "parts" else 1.0


def _tensor(gen, c, heads, N, mean=None, scale=1.0):
    """[B, heads, N, d] of normal values about `mean`, in the case's layout and type."""
    shape = (c["B"], N, heads, c["d"]) if c["layout"] == "bnhd" else (c["B"], heads, N, c["d"])
    x = torch.randn(shape, generator=gen, device="cuda") * scale
    x = x.transpose(1, 2) if c["layout"] == "bnhd" else x
    if mean is not None:
        x += mean
    return x.to(DTYPES[c["dtype"]])


def _heads_mean(gen, c, share):
    """A direction that all keys' queries share: [1, heads, 1, d] for the query heads, and the key heads' own."""
    u = torch.randn((1, c["Hkv"], 1, c["d"]), generator=gen, device="cuda")
    return share * u.repeat_interleave(c["H"] // c["Hkv"], dim=1), share * u


def prepare(case, seed):
    c = case
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    s = {"c": c}
    if c["op"] in ("rotary", "qk_norm", "qk_norm_bwd"):
        s["q"], s["k"] = _tensor(gen, c, c["H"], c["N"]), _tensor(gen, c, c["Hkv"], c["N"])
        pos = torch.arange(c["N"], device="cuda")[None].repeat(c["B"], 1)
        if c["far"]:  # every sequence at its own place
            pos = pos + torch.randint(0, c["far"] + 1, (c["B"], 1), generator=gen, device="cuda")
        s["pos"], s["freqs"] = pos.contiguous(), torch.from_numpy(_freqs(c)).cuda()
        if c["op"] != "rotary":
            s["wq"] = 1.0 + 0.2 * torch.randn(c["d"], generator=gen, device="cuda")
            s["wk"] = 1.0 + 0.2 * torch.randn(c["d"], generator=gen, device="cuda")
        if c["op"] == "qk_norm_bwd":
            s["dq_out"], s["dk_out"] = _tensor(gen, c, c["H"], c["N"]), _tensor(gen, c, c["Hkv"], c["N"])
        return s
    mq, mk = _heads_mean(gen, c, 0.6)
    s["q"] = _tensor(gen, c, c["H"], c["Nq"], mq)
    s["k"], s["v"] = _tensor(gen, c, c["Hkv"], c["Nk"]), _tensor(gen, c, c["Hkv"], c["Nk"])
    s["k"][:, :, :c["sinks"]] += mk.to(s["k"].dtype)  # what makes the first tokens sinks: every query leans towards them
    if c["op"] == "decode":
        k_len = torch.full((c["B"],), c["Nk"], device="cuda")
        if c["ragged"]:  # a stream may be empty, or (rolling) have forgotten most of what it saw
            most = 4 * c["Nk"] if c["rolling"] else c["Nk"]
            k_len = torch.randint(0, most + 1, (c["B"],), generator=gen, device="cuda")
        s["k_len"] = k_len.to(torch.int32)
        return s
    s["q_len"] = s["k_len"] = None
    if c["ragged"]:  # rows behind a sequence's last are left as they were
        ql = torch.randint(max(1, c["Nq"] // 2), c["Nq"] + 1, (c["B"],), generator=gen, device="cuda")
        cached = torch.randint(0, c["Nk"] - c["Nq"] + 1, (c["B"],), generator=gen, device="cuda")
        s["q_len"], s["k_len"] = ql.to(torch.int32), (ql + cached).to(torch.int32)
        s["o"] = torch.zeros_like(s["q"])
        s["lse"] = torch.zeros(s["q"].shape[:3], device="cuda")
    if c["op"] == "window_train":
        s["d_o"] = _tensor(gen, c, c["H"], c["Nq"])
        if c["ragged"]:
            s["dq"], s["dk"], s["dv"] = torch.zeros_like(s["q"]), torch.zeros_like(s["k"]), torch.zeros_like(s["v"])
    return s


# ---------------------------------------------------------------------------------------------------- plain forms
def _cos_sin(s, c):
    a = s["pos"].double()[..., None] * s["freqs"]  # [B, N, rot / 2]
    amp = _amplitude(c)
    sin = -torch.sin(a) if c["inverse"] or c["op"] == "qk_norm_bwd" else torch.sin(a)
    return (torch.cos(a) * amp).float()[:, None], (sin * amp).float()[:, None]


def _turn(x, cos, sin, half):
    r = 2 * cos.shape[-1]
    a, b = (x[..., :r // 2], x[..., r // 2:r]) if half else (x[..., 0:r:2], x[..., 1:r:2])
    y, z = a * cos - b * sin, a * sin + b * cos
    turned = torch.cat((y, z), -1) if half else torch.stack((y, z), -1).flatten(-2)
    return torch.cat((turned, x[..., r:]), -1)


def _plain_rotary(s, c):
    cos, sin = _cos_sin(s, c)
    return {n + "_out": _turn(s[n].float(), cos, sin, c["half"]).to(s[n].dtype) for n in ("q", "k")}


def _plain_qk_norm(s, c):
    cos, sin = _cos_sin(s, c)
    out = {}
    for n, w in (("q", s["wq"]), ("k", s["wk"])):
        x = s[n].float()
        y = x * torch.rsqrt((x * x).mean(-1, keepdim=True) + EPS) * w
        out[n + "_out"] = _turn(y, cos, sin, c["half"]).to(s[n].dtype)
    return out


def _plain_qk_norm_bwd(s, c):
    cos, sin = _cos_sin(s, c)
    out = {}
    for n, w in (("q", s["wq"]), ("k", s["wk"])):
        x = s[n].float()
        g = _turn(s["d" + n + "_out"].float(), cos, sin, c["half"])
        r = torch.rsqrt((x * x).mean(-1, keepdim=True) + EPS)
        out["dw" + n] = (g * x * r).sum((0, 1, 2))
        g = g * w
        out["d" + n] = (r * (g - x * r * r * (g * x).mean(-1, keepdim=True))).to(s[n].dtype)
    return out


def _blocks(s, c):
    """Query rows in blocks of C, and for each block the keys that any of its rows sees: the sinks, then the window."""
    B, H, Nq, d = s["q"].shape
    Hkv, Nk = s["k"].shape[1:3]
    C = min(512, Nq)
    n, S = -(-Nq // C), min(c["sinks"], Nk)
    W = min(c["window"], Nk)
    row = torch.arange(n * C, device="cuda")
    ql = torch.full((B,), Nq, device="cuda") if s["q_len"] is None else s["q_len"].long()
    kl = torch.full((B,), Nk, device="cuda") if s["k_len"] is None else s["k_len"].long()
    pos = (kl - ql)[:, None] + row  # [B, n * C]
    real = (row < ql[:, None]) & (row < Nq)
    j = torch.cat((torch.arange(S, device="cuda").expand(B, n, S),
                   pos.view(B, n, C)[:, :, :1] - (W - 1) + torch.arange(C + W - 1, device="cuda")), -1)  # [B, n, S + C + W - 1]
    jj, pp = j[:, :, None, :], pos.view(B, n, C, 1)
    first = torch.arange(j.shape[-1], device="cuda") < S
    see = (jj <= pp) & (jj >= 0) & (jj < kl[:, None, None, None]) & real.view(B, n, C, 1)
    see &= torch.where(first, torch.ones_like(see), (jj >= S) & (pp - jj < W))
    at = j.clamp(0, Nk - 1).view(B, -1)
    take = lambda x: x.float().transpose(1, 2)[torch.arange(B, device="cuda")[:, None], at].view(B, n, -1, Hkv, d)  # noqa: E731

    def rows(x):
        x = torch.cat((x.float(), torch.zeros((B, H, n * C - Nq, d), device="cuda")), 2) if n * C > Nq else x.float()
        return x.view(B, Hkv, H // Hkv, n, C, d)

    return rows, take, see[:, None, None], at, real[:, None, :Nq]


def _plain_window(s, c):
    rows, take, see, at, real = _blocks(s, c)
    B, H, Nq, d = s["q"].shape
    Hkv, dtype = s["k"].shape[1], s["q"].dtype
    q, k, v = rows(s["q"]), take(s["k"]), take(s["v"])
    p = (torch.einsum("bhgncd,bnshd->bhgncs", q, k) * d ** -0.5).masked_fill_(~see, -math.inf)
    m = p.amax(-1, keepdim=True)
    p = torch.exp_(p.sub_(m.clamp(min=-1e30)))
    total = p.sum(-1, keepdim=True)
    p /= total.clamp(min=1e-30)
    o = torch.einsum("bhgncs,bnshd->bhgncd", p, v)
    flat = lambda x: x.reshape(B, H, -1, x.shape[-1])[:, :, :Nq]  # noqa: E731
    lse = flat(m + torch.log(total))[..., 0]
    out = {"o": torch.where(real[..., None], flat(o), 0.0).to(dtype), "lse": torch.where(real, lse, 0.0)}
    if c["op"] == "window_train":
        do = rows(torch.where(real[..., None], s["d_o"], torch.zeros_like(s["d_o"])))
        ow = rows(out["o"])  # the forward's output as it is kept
        ds = torch.einsum("bhgncd,bnshd->bhgncs", do, v).sub_((do * ow).sum(-1, keepdim=True)).mul_(p).mul_(d ** -0.5)
        out["dq"] = flat(torch.einsum("bhgncs,bnshd->bhgncd", ds, k)).to(dtype)
        b = torch.arange(B, device="cuda")[:, None]
        for name, g in (("dk", torch.einsum("bhgncs,bhgncd->bnshd", ds, q)), ("dv", torch.einsum("bhgncs,bhgncd->bnshd", p, do))):
            full = torch.zeros((B, s["k"].shape[2], Hkv, d), device="cuda")
            full.index_put_((b, at), g.reshape(B, -1, Hkv, d), accumulate=True)
            out[name] = full.transpose(1, 2).to(dtype)
    return out


def _plain_decode(s, c):
    B, H, _, d = s["q"].shape
    Hkv, Nk = s["k"].shape[1:3]
    S, W = c["sinks"], c["window"]
    t = torch.arange(min(S + W, Nk), device="cuda")  # the sinks, then what the window holds
    kl = s["k_len"].long()[:, None]
    j = torch.where(t < S, t, torch.maximum(kl - W, torch.full_like(kl, S)) + t - S)  # positions, [B, S + W]
    see = j < kl
    slot = torch.where(j < S, j, S + (j - S) % (Nk - S)) if c["rolling"] else j
    at = slot.clamp(0, Nk - 1)[:, None, :, None].expand(B, Hkv, -1, d)
    k, v = s["k"].gather(2, at).float(), s["v"].gather(2, at).float()
    q = s["q"].float().reshape(B, Hkv, H // Hkv, d)
    p = (torch.einsum("bhgd,bhsd->bhgs", q, k) * d ** -0.5).masked_fill(~see[:, None, None], -math.inf)
    m = p.amax(-1, keepdim=True)
    p = torch.exp(p - m.clamp(min=-1e30))
    total = p.sum(-1, keepdim=True)
    o = torch.einsum("bhgs,bhsd->bhgd", p / total.clamp(min=1e-30), v)
    return {"o": o.reshape(B, H, 1, d).to(s["q"].dtype), "lse": (m + torch.log(total)).reshape(B, H, 1)}


# ---------------------------------------------------------------------------------------------------- the library's calls
def _own(s, c):
    from paper_2604_16429_b200 import binding as mb
    if c["op"] in ("rotary", "qk_norm", "qk_norm_bwd"):
        rp = mb.RotaryParams(d=c["d"], rot_dim=c["rot"], half=c["half"], amplitude=_amplitude(c))
        if c["op"] == "rotary":
            q, k = mb.mosaic_bsa_rotary(rp, s["q"], s["k"], s["pos"], s["freqs"], inverse=c["inverse"])
            return {"q_out": q, "k_out": k}
        if c["op"] == "qk_norm":
            q, k = mb.mosaic_bsa_qk_norm(rp, s["q"], s["k"], s["wq"], s["wk"], s["pos"], s["freqs"], eps=EPS)
            return {"q_out": q, "k_out": k}
        dq, dk, dwq, dwk = mb.mosaic_bsa_qk_norm_bwd(rp, s["q"], s["k"], s["wq"], s["wk"], s["pos"], s["freqs"], s["dq_out"],
                                                     s["dk_out"], eps=EPS)
        return {"dq": dq, "dk": dk, "dwq": dwq, "dwk": dwk}
    wp = mb.WindowParams(window=c["window"], sinks=c["sinks"], rolling=c["rolling"])
    if c["op"] == "decode":
        o, lse = mb.mosaic_bsa_window_decode(wp, s["q"], s["k"], s["v"], s["k_len"])
        return {"o": o, "lse": lse}
    o, lse = mb.mosaic_bsa_window_fwd(wp, s["q"], s["k"], s["v"], q_len=s["q_len"], k_len=s["k_len"], o=s.get("o"), lse=s.get("lse"))
    out = {"o": o, "lse": lse}
    if c["op"] == "window_train":
        out["dq"], out["dk"], out["dv"] = mb.mosaic_bsa_window_bwd(wp, s["q"], s["k"], s["v"], o, lse, s["d_o"], q_len=s["q_len"],
                                                                   k_len=s["k_len"], dq=s.get("dq"), dk=s.get("dk"), dv=s.get("dv"))
    return out


def run(state):
    s, c = state, state["c"]
    if own:
        return _own(s, c)
    plain = {"rotary": _plain_rotary, "qk_norm": _plain_qk_norm, "qk_norm_bwd": _plain_qk_norm_bwd, "window": _plain_window,
             "window_train": _plain_window, "decode": _plain_decode}
    return plain[c["op"]](s, c)


# ---------------------------------------------------------------------------------------------------- what a pass needs
def _pairs(c, Nq, cached):
    """(query, key) pairs that Nq rows behind `cached` tokens see."""
    pos = np.arange(cached, cached + Nq, dtype=np.int64)
    return float((np.minimum(c["window"], pos + 1) + np.minimum(c["sinks"], np.maximum(pos + 1 - c["window"], 0))).sum())


def work(case):
    """Every input read once, every output written once, and the products of the visible pairs (ragged cases: at the lengths'
    means)."""
    c = case
    size = 4 if c["dtype"] == "fp32" else 2
    if c["op"] in ("rotary", "qk_norm", "qk_norm_bwd"):
        n = float(c["B"] * (c["H"] + c["Hkv"]) * c["N"] * c["d"])
        streams, flops = {"rotary": (2, 3), "qk_norm": (2, 7), "qk_norm_bwd": (3, 14)}[c["op"]]
        return {"bytes": streams * n * size + 8.0 * c["B"] * c["N"], "flops": flops * n}
    B, H, Hkv, d = c["B"], c["H"], c["Hkv"], c["d"]
    if c["op"] == "decode":
        keys = float(min(c["sinks"] + c["window"], c["Nk"]))
        if c["ragged"] and c["rolling"]:  # lengths of 0 to 4 Nk
            keys = keys * 7 / 8
        elif c["ragged"]:                 # lengths of 0 to Nk
            keys = keys - keys * keys / (2.0 * c["Nk"])
        return {"bytes": 2.0 * size * B * Hkv * keys * d + 2.0 * size * B * H * d, "flops": 4.0 * B * H * keys * d}
    Nq, cached = c["Nq"], c["Nk"] - c["Nq"]
    if c["ragged"]:
        Nq, cached = max(1, 3 * Nq // 4), cached // 2
    rows, kv = float(B * H * Nq), float(B * Hkv * min(Nq + cached, c["window"] + c["sinks"] + Nq))
    pairs = B * H * _pairs(c, Nq, cached)
    if c["op"] == "window":
        return {"bytes": size * d * (2 * rows + 2 * kv) + 4 * rows, "flops": 4.0 * d * pairs}
    return {"bytes": size * d * (4 * rows + 4 * kv) + 4 * rows, "flops": 14.0 * d * pairs}


# ---------------------------------------------------------------------------------------------------- 64 bits
def _exact_turn(x, s, c, back):
    """The rotation as a product of complex numbers."""
    r = c["rot"]
    a, b = (x[..., :r // 2], x[..., r // 2:r]) if c["half"] else (x[..., :r].unflatten(-1, (-1, 2)).unbind(-1))
    angle = s["pos"].to(torch.float64).unsqueeze(-1) * torch.from_numpy(_freqs(c)).cuda()
    z = torch.complex(a, b) * torch.polar(torch.full_like(angle, _amplitude(c)), -angle if back else angle).unsqueeze(1)
    y = x.clone()
    if c["half"]:
        y[..., :r // 2], y[..., r // 2:r] = z.real, z.imag
    else:
        y[..., 0:r:2], y[..., 1:r:2] = z.real, z.imag
    return y


def _exact_rotary(s, c):
    if c["op"] == "rotary":
        return {n + "_out": _exact_turn(s[n].double(), s, c, c["inverse"]) for n in ("q", "k")}
    if c["op"] == "qk_norm":
        out = {}
        for n in ("q", "k"):
            x = s[n].double()
            out[n + "_out"] = _exact_turn(x / (x.pow(2).sum(-1, keepdim=True) / c["d"] + EPS).sqrt() * s["w" + n].double(), s, c, False)
        return out
    out = {}
    for n in ("q", "k"):
        x, w = s[n].double(), s["w" + n].double()
        g = _exact_turn(s["d" + n + "_out"].double(), s, c, True)
        rms = (x.pow(2).sum(-1, keepdim=True) / c["d"] + EPS).sqrt()
        unit = x / rms
        out["dw" + n] = (g * unit).flatten(0, 2).sum(0)
        gw = g * w
        out["d" + n] = (gw - unit * (gw * unit).sum(-1, keepdim=True) / c["d"]) / rms
    return out


def _exact_attention(s, c):
    """Row after row of the masked score matrix, a head and 1024 query rows at a time."""
    B, H, Nq, d = s["q"].shape
    G = H // s["k"].shape[1]
    train = c["op"] == "window_train"
    out = {"o": torch.zeros((B, H, Nq, d), dtype=torch.float64, device="cuda"), "lse": torch.zeros((B, H, Nq), dtype=torch.float64, device="cuda")}
    if train:
        out["dq"] = torch.zeros_like(out["o"])
        out["dk"] = torch.zeros(s["k"].shape, dtype=torch.float64, device="cuda")
        out["dv"] = torch.zeros_like(out["dk"])
    for b in range(B):
        kl = c["Nk"] if s["k_len"] is None else int(s["k_len"][b])
        ql = c["Nq"] if s.get("q_len") is None else int(s["q_len"][b])
        held = torch.arange(kl, device="cuda")
        slot = held
        if c["rolling"]:
            held = held[(held < c["sinks"]) | (held >= kl - c["window"])]
            slot = torch.where(held < c["sinks"], held, c["sinks"] + (held - c["sinks"]) % (c["Nk"] - c["sinks"]))
        for h in range(H):
            for lo in range(0, ql, 1024):
                i = torch.arange(lo, min(lo + 1024, ql), device="cuda")
                p = (i + kl - ql)[:, None]
                some = (held <= p.max()) & ((held < c["sinks"]) | (held > p.min() - c["window"]))
                j, at = held[some], slot[some]
                k, v = s["k"][b, h // G, at].double(), s["v"][b, h // G, at].double()
                q = s["q"][b, h, i].double()
                z = q @ k.T / math.sqrt(d)
                z[(j > p) | ((j >= c["sinks"]) & (p - j >= c["window"]))] = -math.inf
                lse = torch.logsumexp(z, -1) if len(j) else torch.full((len(i),), -math.inf, dtype=torch.float64, device="cuda")
                a = torch.nan_to_num(torch.exp(z - lse[:, None]), nan=0.0)
                o = a @ v
                out["o"][b, h, i], out["lse"][b, h, i] = o, lse
                if train:
                    g = s["d_o"][b, h, i].double()
                    dz = a * (g @ v.T - (g * o).sum(-1, keepdim=True)) / math.sqrt(d)
                    out["dq"][b, h, i] = dz @ k
                    out["dk"][b, h // G].index_add_(0, at, dz.T @ q)
                    out["dv"][b, h // G].index_add_(0, at, a.T @ g)
    if c["op"] == "decode" and c["ragged"]:
        out["lse"][(s["k_len"] == 0)] = -math.inf
    return out


def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] in ("rotary", "qk_norm", "qk_norm_bwd"):
        return _exact_rotary(s, case)
    return _exact_attention(s, case)
