"""The paged cache's calls on streams: memory of a named stream, what the kernel right ahead writes, captured graphs, calls of two
threads at once."""
import threading

import pytest
import torch

from paper_2604_16429_b200 import binding as mb
from tests import test_gpu_stream_order as order
from tests import test_gpu_streams as streams
from tests.test_gpu_paged_decode import lens, make
from tests.test_gpu_prefix import with_prefix

pytestmark = pytest.mark.gpu
NAMES = ("append", "paged_decode", "prefix_decode")


def calls(B=3, H=8, Hkv=2, T=2, d=64, page=16, P=300, seed=1):
    """name -> a call that makes all its outputs, its own workspace too"""
    q, kp, vp, table, prefix = with_prefix(B, H, Hkv, T, d, page, 70, P, seed=seed)
    g = torch.Generator().manual_seed(seed + 7)
    k, v = (torch.randn((B, Hkv, T, d), generator=g).bfloat16().cuda() for _ in range(2))
    k_len = lens([1100, 700, 2])
    rp, pp = mb.RotaryParams(d=d, half=True), mb.PagedParams()
    fr = mb.rotary_freqs(rp)
    return {
        "append": lambda **kw: mb.mosaic_bsa_paged_append(rp, k, v, kp, vp, table, k_len, freqs=fr, start=P, q=q, **kw),
        "paged_decode": lambda **kw: mb.mosaic_bsa_paged_decode(pp, q, kp, vp, table, k_len, **kw),
        "prefix_decode": lambda **kw: mb.mosaic_bsa_prefix_decode(pp, q, kp, vp, prefix, P, table, k_len, **kw),
    }


@pytest.mark.parametrize("name", NAMES)
def test_memory_of_the_stream(name):
    streams.check_memory_of_the_stream(calls()[name])


@pytest.mark.parametrize("name", NAMES)
def test_queued_work_is_left_alone(name):
    streams.check_queued_work_is_left_alone(calls()[name])


@pytest.mark.parametrize("name", NAMES)
def test_results_last(name):
    streams.check_results_last_as_long_as_the_caller_needs_them(calls()[name])


@pytest.mark.parametrize("name", NAMES)
def test_captured_on_a_forked_stream(name):
    streams.check_captured_on_a_forked_stream(calls()[name])


@pytest.mark.parametrize("what", ["k_len", "q_len", "table", "prefix", "freqs"])
@pytest.mark.parametrize("op", NAMES)
def test_what_the_kernel_ahead_writes_is_read(op, what):
    B, H, Hkv, T, d, page, P = 4, 8, 2, 2, 64, 16, 300
    q, kp, vp, table, prefix = with_prefix(B, H, Hkv, T, d, page, 12, P, seed=3)
    k = torch.randn((B, Hkv, T, d), generator=torch.Generator().manual_seed(4)).bfloat16().cuda()
    rp, pp = mb.RotaryParams(d=d), mb.PagedParams()
    values = {"k_len": lens([190, 100, 17, 64]), "q_len": lens([2, 1, 2, 2]), "table": table, "prefix": prefix,
              "freqs": (2.0 ** -torch.arange(32, dtype=torch.float64)).cuda()}
    if (what == "prefix" and op != "prefix_decode") or (what == "freqs" and op != "append"):
        return  # it has none
    if what == "freqs":
        rp, values["freqs"] = mb.RotaryParams(d=d, rot_dim=32), values["freqs"][:16]
    words = values[what].contiguous().view(-1).view(torch.int32)
    stale = {"k_len": lens([2, 2, 2, 2]), "q_len": lens([0, 0, 0, 0])}.get(what, torch.zeros_like(words) - 1)

    def call(x):
        x = x.view(values[what].dtype).view(values[what].shape)
        a = {**values, what: x}
        if op == "append":
            pools = kp.clone(), vp.clone()
            out = torch.zeros_like(q)
            mb.mosaic_bsa_paged_append(rp, k, k, *pools, a["table"], a["k_len"], freqs=a["freqs"] if what == "freqs" else mb.rotary_freqs(rp),
                                       q=q, q_len=a["q_len"], q_out=out)
            return (*pools, out)
        out = torch.zeros_like(q), torch.zeros(q.shape[:3], device="cuda")
        if op == "paged_decode":
            return mb.mosaic_bsa_paged_decode(pp, q, kp, vp, a["table"], a["k_len"], q_len=a["q_len"], o=out[0], lse=out[1])
        return mb.mosaic_bsa_prefix_decode(pp, q, kp, vp, a["prefix"], P, a["table"], a["k_len"], q_len=a["q_len"], o=out[0], lse=out[1])

    order.check(words, stale, lambda x: x, call)


def step_of(rp, fr, new, pools, table, prefix, P, k_len, **kw):
    """One step of a batch: the new tokens into the cache, then attention"""
    q, k, v = new
    qr = mb.mosaic_bsa_paged_append(rp, k, v, *pools, table, k_len, freqs=fr, start=P, q=q, **kw)
    a = mb.mosaic_bsa_paged_decode(mb.PagedParams(), qr, *pools, table, k_len, **kw)
    b = mb.mosaic_bsa_prefix_decode(mb.PagedParams(), qr, *pools, prefix, P, table, k_len, **kw)
    return (qr,) + a + b


def batch(seed, B=5, H=8, Hkv=2, d=128, page=16, P=500):
    q, kp, vp, table, prefix = with_prefix(B, H, Hkv, 1, d, page, 5, P, seed=seed)
    g = torch.Generator().manual_seed(seed)
    k, v = (torch.randn((B, Hkv, 1, d), generator=g).bfloat16().cuda() for _ in range(2))
    rp = mb.RotaryParams(d=d)
    return rp, mb.rotary_freqs(rp), (q, k, v), (kp, vp), table, prefix, P


def test_a_captured_step_is_replayed_as_the_cache_grows():
    """Lengths and new tokens change in place between replays; an eager twin on its own pools gives the same bits."""
    x = batch(11)
    rp, fr, new, pools, table, prefix, P = x
    twin = tuple(p.clone() for p in pools)
    k_len = lens([1, 17, 16, 40, 70])
    for p in (step_of(rp, fr, new, tuple(p.clone() for p in pools), table, prefix, P, k_len),):  # (whatever the first call sets up)
        torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        out = step_of(rp, fr, new, pools, table, prefix, P, k_len)
    for n in range(8):
        for t in new:
            t.copy_(torch.randn(t.shape, generator=torch.Generator().manual_seed(n)).bfloat16())
        g.replay()
        want = step_of(rp, fr, new, twin, table, prefix, P, k_len)
        assert all(torch.equal(a, b) for a, b in zip(out, want)) and all(torch.equal(a, b) for a, b in zip(pools, twin))
        k_len += 1


def test_two_captured_graphs_in_turn():
    """Each has a workspace of its own, although one was freed before the other was captured."""
    xs = [batch(21), batch(22, B=3, H=12, Hkv=3, d=64, P=1300)]
    ls = [lens([3, 20, 33, 64, 80]), lens([5, 50, 79])]
    want = [step_of(*x[:3], tuple(p.clone() for p in x[3]), *x[4:], k) for x, k in zip(xs, ls)]
    graphs, outs = [], []
    for x, k in zip(xs, ls):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            outs.append(step_of(*x[:3], x[3], *x[4:], k))
        graphs.append(g)
    for i in (0, 1, 1, 0, 0, 1):
        for o in outs[i]:
            o.zero_()
        graphs[i].replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(outs[i], want[i]))


def test_calls_of_two_threads_at_once():
    xs = [batch(31), batch(32, B=40, H=12, Hkv=3, d=64, P=1300)]
    ls = [lens([3, 20, 33, 64, 80]), lens([1 + 2 * i for i in range(40)])]
    want = [step_of(*x[:3], tuple(p.clone() for p in x[3]), *x[4:], k) for x, k in zip(xs, ls)]
    torch.cuda.synchronize()
    got, on = [None, None], [torch.cuda.Stream(), torch.cuda.Stream()]

    def work(i):
        for _ in range(20):
            with torch.cuda.stream(on[i]):
                got[i] = step_of(*xs[i][:3], xs[i][3], *xs[i][4:], ls[i])
        on[i].synchronize()

    threads = [threading.Thread(target=work, args=(i,)) for i in (0, 1)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    for w, g in zip(want, got):
        assert all(torch.equal(a, b) for a, b in zip(w, g))


def test_two_calls_on_two_streams_over_the_same_pools():
    q, kp, vp, table = make(6, 8, 2, 1, 128, 64, 40, seed=5)
    k_len = lens([2560, 1, 700, 1300, 64, 65])
    want = mb.mosaic_bsa_paged_decode(mb.PagedParams(), q, kp, vp, table, k_len)
    torch.cuda.synchronize()
    side = [torch.cuda.Stream() for _ in range(3)]
    got = []
    for _ in range(10):
        for s in side:
            got.append(mb.mosaic_bsa_paged_decode(mb.PagedParams(), q, kp, vp, table, k_len, stream=s))
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for g in got for a, b in zip(g, want))
