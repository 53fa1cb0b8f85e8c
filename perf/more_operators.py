"""The operators on a paged cache of keys and values, as cases that can be timed and compared.

* ``append``  new tokens' keys and values go to their places in a paged cache, keys (and queries) turned to their positions
              on the way
* ``paged``   attention of one or a few new tokens per sequence over such a cache, with or without a window and sinks
* ``prefix``  the same for a batch whose sequences all begin with one long prefix, which lies in the cache once

``own`` says which side ``run`` takes: elementary torch operations in 32 bits (angles in 64), or this library's calls.
"""
from __future__ import annotations

import math

import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "fp16": torch.float16}


def _append(name, B, H, Hkv, N, d, rot, page, cached, **over):
    """N new tokens a sequence behind `cached` ones; `start`: position of the cache's first token."""
    c = dict(name=name, op="append", B=B, H=H, Hkv=Hkv, N=N, d=d, rot=rot, page=page, cached=cached, half=True, dtype="bf16",
             layout="bnhd", pages="hpd", ragged=False, start=0, queries=True)
    c.update(over)
    return c


def _attend(name, op, B, H, Hkv, T, N, d, page, **over):
    """T new tokens a sequence, the last of up to N in its pages, behind P of a prefix that all share; window 0: none."""
    c = dict(name=name, op=op, B=B, H=H, Hkv=Hkv, T=T, N=N, d=d, page=page, P=0, window=0, sinks=0, dtype="bf16", layout="bhnd",
             pages="hpd", ragged=False)
    c.update(over)
    return c


def listed():
    return [
        # the next token of 64 sequences of 4096: the smallest call, one a layer and step
        _append("append_decode", 64, 16, 4, 1, 128, 128, 16, 4096),
        # two prompts go to an empty cache, as the projection lays their heads out
        _append("append_prompt", 2, 16, 4, 8192, 128, 128, 64, 0, pages="phd"),
        # the next chunk of five prompts of different lengths behind a shared prefix, three quarters of the head turned in adjacent
        # pairs; the queries are turned elsewhere
        _append("append_chunk_ragged", 5, 12, 3, 1021, 64, 48, 32, 3000, half=False, dtype="fp16", layout="bhnd", ragged=True,
                start=32768, queries=False),
        # one token of one sequence: latency
        _attend("paged_one", "paged", 1, 16, 4, 1, 16384, 128, 16),
        # one token of 64 sequences of very different lengths, pages that hold a token's heads side by side
        _attend("paged_ragged", "paged", 64, 16, 4, 1, 8192, 128, 64, pages="phd", ragged=True),
        # eight long documents, eight query heads a key head
        _attend("paged_long", "paged", 8, 32, 4, 1, 65536, 128, 128),
        # five drafted tokens of 32 sequences are checked at once, inside a window
        _attend("paged_window_drafts", "paged", 32, 12, 3, 5, 16384, 64, 32, window=2048, sinks=4, dtype="fp16", ragged=True),
        # eight short answers to one question: the smallest batch with a prefix
        _attend("prefix_short", "prefix", 8, 16, 4, 1, 64, 128, 16, P=2048),
        # 64 members of an ensemble or as many questions on one long document
        _attend("prefix_long", "prefix", 64, 16, 4, 1, 512, 128, 64, P=32768, ragged=True),
        # drafts of 33 sequences behind a prefix of odd length
        _attend("prefix_drafts_odd", "prefix", 33, 12, 3, 4, 300, 64, 32, P=8191, dtype="fp16", ragged=True, layout="bnhd"),
        # a wide batch whose own answers have grown long
        _attend("prefix_wide", "prefix", 256, 16, 4, 1, 1024, 128, 128, P=16384, ragged=True, pages="phd"),
    ]


def _log(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    """Any operator, type, layout, page size and head grouping; appended tokens to 16384, caches to 65536 tokens (two million
    (token, key head) pairs in all), prefixes to 32768; batches to 256, 67 million (query row, key) pairs at most."""
    op = rng.choice(["append", "paged", "paged", "prefix", "prefix"])
    d = rng.choice([64, 128])
    Hkv = rng.choice([1, 2, 3, 4, 8])
    H = Hkv * rng.choice([1, 2, 3, 4, 6, 8])
    both = dict(dtype=rng.choice(["bf16", "fp16"]), layout=rng.choice(["bhnd", "bnhd"]), pages=rng.choice(["hpd", "phd"]),
                ragged=rng.random() < 0.6)
    page = rng.choice([16, 32, 64, 128, 256])
    if op == "append":
        N = _log(rng, 1, 16384)
        B = _log(rng, 1, max(1, min(256, (1 << 18) // (H * N))))
        c = _append("", B, H, Hkv, N, d, rng.choice([d, d, d // 2, d // 4, 0]), page, rng.choice([0, _log(rng, 1, 8192)]),
                    half=rng.random() < 0.5, start=rng.choice([0, 0, _log(rng, 1, 1 << 20)]), queries=rng.random() < 0.7, **both)
    else:
        T = rng.choice([1, 1, 1, 2, 3, 5, 8])
        if op == "paged":
            N = _log(rng, T, 65536)
            B = _log(rng, 1, max(1, min(256, (1 << 21) // (Hkv * N), (1 << 26) // (H * T * N))))
            P, window, sinks = 0, rng.choice([0, 0, _log(rng, 1, 8192)]), 0
            sinks = rng.randint(0, 64) if window else 0
        else:
            N = _log(rng, T, 2048)
            P, window, sinks = _log(rng, 64, 32768), 0, 0
            B = _log(rng, 1, max(1, min(256, (1 << 26) // (H * T * (P + N)))))
        c = _attend("", op, B, H, Hkv, T, N, d, page, P=P, window=window, sinks=sinks, **both)
    del c["name"]
    return c


# ---------------------------------------------------------------------------------------------------- inputs
def _tensor(gen, c, heads, N):
    """[B, heads, N, d] of normal values, in the case's layout and type."""
    shape = (c["B"], N, heads, c["d"]) if c["layout"] == "bnhd" else (c["B"], heads, N, c["d"])
    x = torch.randn(shape, generator=gen, device="cuda", dtype=torch.float32).to(DTYPES[c["dtype"]])
    return x.transpose(1, 2) if c["layout"] == "bnhd" else x


def _pool(gen, c, pages):
    """[pages, Hkv, page, d], whose memory holds a page's heads or its tokens side by side."""
    shape = (pages, c["page"], c["Hkv"], c["d"]) if c["pages"] == "phd" else (pages, c["Hkv"], c["page"], c["d"])
    x = torch.empty(shape, device="cuda", dtype=DTYPES[c["dtype"]])
    for part in x.split(max(1, (1 << 26) // (c["page"] * c["Hkv"] * c["d"]))):  # (normal values in 32 bits take their time and room)
        part.copy_(torch.randn(part.shape, generator=gen, device="cuda"))
    return x.transpose(1, 2) if c["pages"] == "phd" else x


def _freqs(c):
    i = torch.arange(c["rot"] // 2, dtype=torch.float64)
    return (10000.0 ** (-2.0 * i / max(c["rot"], 1))).cuda()


def _table(gen, c, lens, most, pages, first):
    """[B, most / page] of page numbers, drawn from a pool where sequences have come and gone; -1 behind a sequence's last."""
    width = -(-most // c["page"])
    ids = first + torch.randperm(pages - first, generator=gen, device="cuda")[:c["B"] * width]
    at = torch.arange(width, device="cuda") * c["page"]
    return torch.where(at < lens[:, None], ids.view(c["B"], width), -1).to(torch.int32)


def prepare(case, seed):
    c = case
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    s = {"c": c}
    B, page = c["B"], c["page"]
    if c["op"] == "append":
        s["k"], s["v"] = _tensor(gen, c, c["Hkv"], c["N"]), _tensor(gen, c, c["Hkv"], c["N"])
        s["q"] = _tensor(gen, c, c["H"], c["N"]) if c["queries"] else None
        s["q_len"] = None
        new = torch.full((B,), c["N"], device="cuda")
        cached = torch.full((B,), c["cached"], device="cuda")
        if c["ragged"]:
            new = torch.randint(max(1, c["N"] // 2), c["N"] + 1, (B,), generator=gen, device="cuda")
            cached = torch.randint(0, c["cached"] + 1, (B,), generator=gen, device="cuda")
            s["q_len"] = new.to(torch.int32)
            s["q_out"] = None if s["q"] is None else torch.zeros_like(s["q"])  # rows behind a sequence's last are left as they were
        most = c["cached"] + c["N"]
        # what the call writes, and as much again that belongs to others (the pages between hold nothing that is looked at); the
        # last page is nobody's
        touched = -(-c["N"] // page) + 1
        width = -(-most // page)
        pages = 2 * B * min(touched, width) + 2
        ids = torch.randperm(pages - 1, generator=gen, device="cuda")[:B * min(touched, width)].view(B, -1)
        at = torch.arange(width, device="cuda") - (cached // page)[:, None]
        table = torch.where((at >= 0) & (at < ids.shape[1]), ids.gather(1, at.clamp(0, ids.shape[1] - 1)), -1)
        s["table"], s["k_len"] = table.to(torch.int32).contiguous(), (cached + new).to(torch.int32)
        s["k_pages"], s["v_pages"] = _pool(gen, c, pages), _pool(gen, c, pages)
        s["freqs"] = _freqs(c)
        return s
    T, N = c["T"], c["N"]
    s["q"] = _tensor(gen, c, c["H"], T)
    lens = torch.full((B,), N, device="cuda")
    if c["ragged"]:  # behind a prefix a sequence may have nothing of its own but its new tokens
        lens = torch.randint(T, N + 1, (B,), generator=gen, device="cuda")
    shared = -(-c["P"] // page)
    pages = shared + B * -(-N // page) + 3
    s["table"] = _table(gen, c, lens, N, pages, shared)
    s["prefix"] = torch.randperm(shared, generator=gen, device="cuda").to(torch.int32) if shared else None
    s["k_len"] = lens.to(torch.int32)
    s["k_pages"], s["v_pages"] = _pool(gen, c, pages), _pool(gen, c, pages)
    # what makes the first tokens sinks: every query leans towards them
    lean = 0.6 * torch.randn((c["Hkv"], c["d"]), generator=gen, device="cuda")
    s["q"] += lean.repeat_interleave(c["H"] // c["Hkv"], 0)[None, :, None].to(s["q"].dtype)
    first = s["prefix"][:1] if shared else s["table"][:, 0]
    s["k_pages"][first.long(), :, :4] += lean[None, :, None].to(s["q"].dtype)
    return s


# ---------------------------------------------------------------------------------------------------- plain forms
def _turn(x, cos, sin, half):
    r = 2 * cos.shape[-1]
    a, b = (x[..., :r // 2], x[..., r // 2:r]) if half else (x[..., 0:r:2], x[..., 1:r:2])
    y, z = a * cos - b * sin, a * sin + b * cos
    turned = torch.cat((y, z), -1) if half else torch.stack((y, z), -1).flatten(-2)
    return torch.cat((turned, x[..., r:]), -1)


def _plain_append(s, c):
    B, N, page = c["B"], c["N"], c["page"]
    row = torch.arange(N, device="cuda")
    new = torch.full((B,), N, device="cuda") if s["q_len"] is None else s["q_len"].long()
    at = (s["k_len"].long() - new)[:, None] + row  # [B, N]
    real = row < new[:, None]
    angle = (c["start"] + at).double()[..., None] * s["freqs"]
    cos, sin = torch.cos(angle).float()[:, None], torch.sin(angle).float()[:, None]
    width = s["table"].shape[1]
    pages = s["table"].long().gather(1, (at // page).clamp(0, width - 1))
    real_at = torch.where(real, pages, s["k_pages"].shape[0] - 1)  # (rows that do not exist write what the last page has already)
    slot = torch.where(real, at % page, torch.zeros_like(at))
    out = {}
    for n in ("k", "v"):
        x = s[n].float()
        x = _turn(x, cos, sin, c["half"]) if n == "k" and c["rot"] else x
        pool = s[n + "_pages"]
        x = torch.where(real[:, None, :, None], x.to(pool.dtype), pool[-1, :, 0][None, :, None])
        pool[real_at, :, slot] = x.transpose(1, 2)
        out[n + "_pages"] = pool
    if s["q"] is not None:
        q = s["q"].float()
        q = (_turn(q, cos, sin, c["half"]) if c["rot"] else q).to(s["q"].dtype)
        out["q"] = torch.where(real[:, None, :, None], q, torch.zeros_like(q))
    return out


def _plain_attend(s, c):
    B, H, T, d = s["q"].shape
    Hkv, page = c["Hkv"], c["page"]
    q = s["q"].float().reshape(B, Hkv, H // Hkv, T, d)
    width = s["table"].shape[1]
    take = lambda x: x[s["table"].long().clamp(min=0)].transpose(1, 2).reshape(B, Hkv, width * page, d).float()  # noqa: E731
    p = torch.einsum("bhgtd,bhsd->bhgts", q, take(s["k_pages"])) * d ** -0.5
    j = torch.arange(width * page, device="cuda")
    at = (s["k_len"].long()[:, None] - T + torch.arange(T, device="cuda"))[..., None]  # [B, T, 1]
    see = j <= at
    if c["window"]:
        see &= (at - j < c["window"]) | (j < c["sinks"])
    p.masked_fill_(~see[:, None, None], -math.inf)
    if c["P"]:
        held = lambda x: x[s["prefix"].long()].transpose(0, 1).reshape(Hkv, -1, d)[:, :c["P"]].float()  # noqa: E731
        p = torch.cat((torch.einsum("bhgtd,hsd->bhgts", q, held(s["k_pages"])) * d ** -0.5, p), -1)
    m = p.amax(-1, keepdim=True)
    p = torch.exp_(p.sub_(m))
    total = p.sum(-1, keepdim=True)
    o = torch.einsum("bhgts,bhsd->bhgtd", p[..., c["P"]:], take(s["v_pages"]))
    if c["P"]:
        o += torch.einsum("bhgts,hsd->bhgtd", p[..., :c["P"]], held(s["v_pages"]))
    o /= total
    return {"o": o.reshape(B, H, T, d).to(s["q"].dtype), "lse": (m + torch.log(total)).reshape(B, H, T)}


# ---------------------------------------------------------------------------------------------------- the library's calls
def _own(s, c):
    from paper_2604_16429_b200 import binding as mb
    if c["op"] == "append":
        rp = mb.RotaryParams(d=c["d"], rot_dim=c["rot"], half=c["half"])
        q = mb.mosaic_bsa_paged_append(rp, s["k"], s["v"], s["k_pages"], s["v_pages"], s["table"], s["k_len"], freqs=s["freqs"],
                                       start=c["start"], q=s["q"], q_len=s["q_len"], q_out=s.get("q_out"))
        out = {"k_pages": s["k_pages"], "v_pages": s["v_pages"]}
        return out if q is None else {**out, "q": q}
    if c["op"] == "paged":
        pp = mb.PagedParams(window=c["window"], sinks=c["sinks"])
        o, lse = mb.mosaic_bsa_paged_decode(pp, s["q"], s["k_pages"], s["v_pages"], s["table"], s["k_len"])
    else:
        o, lse = mb.mosaic_bsa_prefix_decode(mb.PagedParams(), s["q"], s["k_pages"], s["v_pages"], s["prefix"], c["P"], s["table"],
                                             s["k_len"])
    return {"o": o, "lse": lse}


def run(state):
    s, c = state, state["c"]
    if own:
        return _own(s, c)
    return _plain_append(s, c) if c["op"] == "append" else _plain_attend(s, c)


# ---------------------------------------------------------------------------------------------------- what a pass needs
def work(case):
    """Every input read once, every output written once, and the products of the visible pairs (ragged cases: at the lengths'
    means)."""
    c = case
    B, H, Hkv, d = c["B"], c["H"], c["Hkv"], c["d"]
    if c["op"] == "append":
        n = B * c["N"] * d * (0.75 if c["ragged"] and c["N"] > 1 else 1.0)
        heads = 2 * Hkv + (H if c["queries"] else 0)
        turned = Hkv + (H if c["queries"] else 0)
        return {"bytes": 4.0 * n * heads, "flops": 3.0 * n * turned * c["rot"] / d}
    T, N = c["T"], c["N"]
    keys = 0.5 * (N + T) if c["ragged"] else float(N)
    if c["window"]:
        w = float(min(N, c["window"] + c["sinks"]))
        keys = w - w * w / (2.0 * N) if c["ragged"] else w
    rows = float(B * H * T)
    return {"bytes": 4.0 * d * Hkv * (B * keys + c["P"]) + 4.0 * d * rows + 4.0 * rows, "flops": 4.0 * d * rows * (keys + c["P"])}


# ---------------------------------------------------------------------------------------------------- 64 bits
def _exact_append(s, c):
    """A token at a time's worth of bookkeeping on the host, the rotation as a product of complex numbers."""
    out = {"k_pages": s["k_pages"].double(), "v_pages": s["v_pages"].double()}
    if s["q"] is not None:
        out["q"] = torch.zeros(s["q"].shape, dtype=torch.float64, device="cuda")
    r = c["rot"]
    f = _freqs(c)

    def turned(x, pos):
        x = x.double()
        if not r:
            return x
        a, b = (x[..., :r // 2], x[..., r // 2:r]) if c["half"] else x[..., :r].unflatten(-1, (-1, 2)).unbind(-1)
        angle = pos.double()[:, None] * f
        z = torch.complex(a, b) * torch.polar(torch.ones_like(angle), angle)
        y = x.clone()
        if c["half"]:
            y[..., :r // 2], y[..., r // 2:r] = z.real, z.imag
        else:
            y[..., 0:r:2], y[..., 1:r:2] = z.real, z.imag
        return y

    for b in range(c["B"]):
        kl = int(s["k_len"][b])
        n = c["N"] if s["q_len"] is None else int(s["q_len"][b])
        j = torch.arange(kl - n, kl, device="cuda")
        page = s["table"][b].long()[torch.div(j, c["page"], rounding_mode="floor")]
        slot = j - c["page"] * torch.div(j, c["page"], rounding_mode="floor")
        out["k_pages"][page, :, slot] = turned(s["k"][b, :, :n], c["start"] + j).transpose(0, 1)
        out["v_pages"][page, :, slot] = s["v"][b, :, :n].double().transpose(0, 1)
        if s["q"] is not None:
            out["q"][b, :, :n] = turned(s["q"][b, :, :n], c["start"] + j)
    return out


def _exact_attend(s, c):
    """A sequence and key head at a time: its keys in a row, the prefix in front."""
    B, H, T, d = s["q"].shape
    G = H // c["Hkv"]
    out = {"o": torch.zeros((B, H, T, d), dtype=torch.float64, device="cuda"), "lse": torch.zeros((B, H, T), dtype=torch.float64, device="cuda")}

    def held(x, pages, h, n):
        return x[pages.long(), h].reshape(-1, d)[:n].double()

    for h in range(c["Hkv"]):
        if c["P"]:
            kp, vp = held(s["k_pages"], s["prefix"], h, c["P"]), held(s["v_pages"], s["prefix"], h, c["P"])
        for b in range(B):
            n = int(s["k_len"][b])
            pages = s["table"][b, :-(-n // c["page"])]
            k, v = held(s["k_pages"], pages, h, n), held(s["v_pages"], pages, h, n)
            x = s["q"][b, h * G:(h + 1) * G].double()  # [G, T, d]
            z = x @ k.T / math.sqrt(d)
            dist = torch.arange(n - T, n, device="cuda")[:, None] - torch.arange(n, device="cuda")
            hidden = dist < 0
            if c["window"]:
                hidden |= (dist >= c["window"]) & (torch.arange(n, device="cuda") >= c["sinks"])
            z[:, hidden] = -math.inf
            if c["P"]:
                z, v = torch.cat((x @ kp.T / math.sqrt(d), z), -1), torch.cat((vp, v))
            lse = torch.logsumexp(z, -1)
            out["o"][b, h * G:(h + 1) * G] = torch.exp(z - lse[..., None]) @ v
            out["lse"][b, h * G:(h + 1) * G] = lse
    return out


def exact(case, seed):
    s = prepare(case, seed)
    return _exact_append(s, case) if case["op"] == "append" else _exact_attend(s, case)
