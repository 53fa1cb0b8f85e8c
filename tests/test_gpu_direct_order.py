"""A call reads what the kernel right ahead of it on the stream writes last, with nothing at all between the two.

The writer is that of tests/test_gpu_stream_order.py, a rotation whose last words are the call's lengths, table, frequencies or rows.  A
kernel of torch's between the two (a clone, a fill, a copy) would not start before the rotation is complete, nor let the next one in
early, and so hide a read that comes too soon: outputs, workspaces and views are made ahead of the rotation, and a call that
dispatches any operation of torch's fails."""
import pytest
import torch
from torch.utils._python_dispatch import TorchDispatchMode

from paper_2604_16429_b200 import binding as mb
from tests import test_gpu_window as W
from tests.test_gpu_paged_decode import lens, make
from tests.test_gpu_prefix import with_prefix
from tests.test_gpu_stream_order import Writer

pytestmark = pytest.mark.gpu


class NothingOfTorch(TorchDispatchMode):
    def __torch_dispatch__(self, func, types, args=(), kwargs=None):
        raise AssertionError(f"{func} stands between the writer and the call")


def check(value, stale, outputs, call, view=lambda x: x):
    """`call(x, out)` runs the operator on x, which holds `value` (or on a view of it), into what `outputs()` makes; `stale` stands in x
    until the rotation ahead of the call is done."""
    words, old_words = (x.contiguous().view(-1).view(torch.int32) for x in (value, stale))
    w = Writer(words)
    x, want, old = view(w.at.view(value.dtype).view(value.shape)), outputs(), outputs()
    call(view(value), want)
    call(view(stale), old)
    torch.cuda.synchronize()
    assert not all(torch.equal(a, b) for a, b in zip(want, old)), "what stood there before gives the same"
    for _ in range(6):
        got = outputs()
        w.go(old_words)
        with NothingOfTorch():
            call(x, got)
        torch.cuda.synchronize()
        assert torch.equal(w.at, words)
        for a, b in zip(got, want):
            assert torch.equal(a, b)


B, T, D, PAGE, P = 4, 2, 64, 16, 300
LENGTHS = {"k_len": [190, 100, 17, 64], "q_len": [2, 1, 2, 2]}


def stale_of(what, x):
    return lens({"k_len": [2] * B, "q_len": [0] * B}[what]) if what in LENGTHS else torch.full_like(x, -1)


@pytest.mark.parametrize("what", ["k_len", "q_len", "table", "freqs"])
@pytest.mark.parametrize("heads", [2, 32])  # one part of a token a warp, and several
def test_append(what, heads):
    q, kp, vp, table = make(B, heads, 2, T, D, PAGE, 12, seed=3)
    k = torch.randn((B, 2, T, D), generator=torch.Generator().manual_seed(4)).bfloat16().cuda()
    rp = mb.RotaryParams(d=D, rot_dim=32)
    values = {"k_len": lens(LENGTHS["k_len"]), "q_len": lens(LENGTHS["q_len"]), "table": table, "freqs": mb.rotary_freqs(rp)}

    def call(x, out):
        a = {**values, what: x}
        mb.mosaic_bsa_paged_append(rp, k, k, out[0], out[1], a["table"], a["k_len"], freqs=a["freqs"], q=q, q_len=a["q_len"], q_out=out[2])

    check(values[what], stale_of(what, values[what]), lambda: (kp.clone(), vp.clone(), torch.zeros_like(q)), call)


def attention(a, q, pools, out, ws, shared):
    if shared:
        mb.mosaic_bsa_prefix_decode(mb.PagedParams(), q, *pools, a["prefix"], shared, a["table"], a["k_len"], q_len=a["q_len"], o=out[0],
                                    lse=out[1], ws=ws)
    else:
        mb.mosaic_bsa_paged_decode(mb.PagedParams(), q, *pools, a["table"], a["k_len"], q_len=a["q_len"], o=out[0], lse=out[1], ws=ws)


def results(q):
    return torch.zeros_like(q), torch.zeros(q.shape[:3], device="cuda")


def workspace(q, k_pages, table, shared):
    return torch.zeros(mb.paged_workspace_bytes(mb.PagedParams(), q, k_pages, table, shared), dtype=torch.uint8, device="cuda")


@pytest.mark.parametrize("what,shared", [("k_len", 0), ("q_len", 0), ("table", 0), ("k_len", P), ("q_len", P), ("table", P), ("prefix", P)])
@pytest.mark.parametrize("width", [12, 40])  # results from the kernel that makes the parts, and joined apart
def test_attention(what, shared, width):
    q, kp, vp, table, prefix = with_prefix(B, 8, 2, T, D, PAGE, width, P, seed=3)
    if what == "table" and width > 12:  # (what the writer has room for: one row for all members)
        table = table[:1]
    values = {"k_len": lens(LENGTHS["k_len"]), "q_len": lens(LENGTHS["q_len"]), "table": table.contiguous(), "prefix": prefix}
    view = (lambda x: x.expand(B, width)) if what == "table" else (lambda x: x)
    ws = workspace(q, kp, table.expand(B, width), shared)
    check(values[what], stale_of(what, values[what]), lambda: results(q),
          lambda x, out: attention({**values, what: x}, q, (kp, vp), out, ws, shared), view)


@pytest.mark.parametrize("width", [12, 40])
@pytest.mark.parametrize("shared", [0, P])
def test_attention_reads_the_queries(width, shared):
    """One member, one head: the row of q is what the writer writes."""
    q, kp, vp, table, prefix = with_prefix(1, 1, 1, 1, D, PAGE, width, P, seed=5)
    a = {"k_len": lens([190]), "q_len": None, "table": table, "prefix": prefix}
    ws = workspace(q, kp, table, shared)
    check(q, torch.zeros_like(q), lambda: results(q), lambda x, out: attention(a, x, (kp, vp), out, ws, shared))


@pytest.mark.parametrize("what", ["q_len", "k_len"])
@pytest.mark.parametrize("op", ["fwd", "bwd", "decode"])
def test_window(op, what):
    if op == "decode" and what == "q_len":
        return  # it has none
    wp = mb.WindowParams(window=100, sinks=4)
    q, k, v, d_o = W.make(4, 4, 2, 300, 300, 64, seed=1)
    full, short = lens([300, 290, 280, 299]), lens([1, 0, 2, 1])
    o, lse = mb.mosaic_bsa_window_fwd(wp, q, k, v)
    q1 = q[:, :, :1].contiguous()
    size = {"fwd": mb.OP_FWD, "bwd": mb.OP_BWD}
    n = mb.window_workspace_bytes(wp, q, k, size[op]) if op in size else 0
    ws = torch.zeros(max(n, 256), dtype=torch.uint8, device="cuda")

    def outputs():
        return [torch.zeros_like(x) for x in {"fwd": (q, lse), "bwd": (q, k, v), "decode": (q1, lse[:, :, :1].contiguous())}[op]]

    def call(x, out):
        kw = {what: x}
        if op == "decode":
            mb.mosaic_bsa_window_decode(wp, q1, k, v, o=out[0], lse=out[1], **kw)
        elif op == "fwd":
            mb.mosaic_bsa_window_fwd(wp, q, k, v, o=out[0], lse=out[1], ws=ws, **kw)
        else:
            mb.mosaic_bsa_window_bwd(wp, q, k, v, o, lse, d_o, dq=out[0], dk=out[1], dv=out[2], ws=ws, **kw)

    check(full, short, outputs, call)
