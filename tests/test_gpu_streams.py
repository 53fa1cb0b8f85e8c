"""Calls on a stream that the caller names: the tensors that a call makes come from that stream's memory.

The caching allocator hands a freed block to the next allocation of the same stream at once, although work queued there may still read or
write it; only the order of that stream makes it safe.  So a call that runs on another stream may not take its memory from the current
one, and the caller, who goes on with the results on the current stream, may not lose them to a later call when it frees them."""
import pytest
import torch

from paper_2604_16429_b200 import binding as mb

pytestmark = pytest.mark.gpu


def owner(t):
    """The stream whose memory `t` lies in."""
    at = t.data_ptr()
    for seg in torch.cuda.memory_snapshot():
        if seg["address"] <= at < seg["address"] + seg["total_size"]:
            return seg["stream"]
    raise AssertionError("not the allocator's")


def sequence_calls(B=1, H=4, Hkv=2, N=1024, d=64):
    """name -> a call that makes all its outputs, its own workspace too"""
    g = torch.Generator().manual_seed(1)
    q, k, v, d_o = (torch.randn((B, h, N, d), generator=g).bfloat16().cuda() for h in (H, Hkv, Hkv, H))
    rp, wp = mb.RotaryParams(d=d, half=True), mb.WindowParams(window=100, sinks=4)
    pos, fr, w = torch.arange(N, device="cuda"), mb.rotary_freqs(rp), torch.ones(d, device="cuda")
    o, lse = mb.mosaic_bsa_window_fwd(wp, q, k, v)
    return {
        "rotary": lambda **kw: mb.mosaic_bsa_rotary(rp, q, k, pos, fr, **kw),
        "qk_norm": lambda **kw: mb.mosaic_bsa_qk_norm(rp, q, k, w, w, pos, fr, **kw),
        "qk_norm_bwd": lambda **kw: mb.mosaic_bsa_qk_norm_bwd(rp, q, k, w, w, pos, fr, d_o, k, **kw),
        "window_fwd": lambda **kw: mb.mosaic_bsa_window_fwd(wp, q, k, v, **kw),
        "window_bwd": lambda **kw: mb.mosaic_bsa_window_bwd(wp, q, k, v, o, lse, d_o, **kw),
        "window_decode": lambda **kw: mb.mosaic_bsa_window_decode(wp, q[:, :, -1:], k, v, **kw),
    }


def block_calls(B=1, H=2, d=64):
    p = mb.Params(B=B, H=H, nlat=32, nlon=64, bh=8, bw=8, topk=4)
    g = torch.Generator().manual_seed(2)
    q, k, v, d_o = (torch.randn((B, H, p.N, d), generator=g).bfloat16().cuda() for _ in range(4))
    gates = torch.rand((B, H, p.N, 3), generator=g).cuda()
    pos = torch.rand((p.N, 2), generator=g).cuda()
    idx = mb.mosaic_bsa_select(p, q, k)
    mb.mosaic_bsa_select_static(p, q, k)
    o, lse = mb.mosaic_bsa_fwd(p, q, k, v, idx)
    return {
        "select": lambda **kw: mb.mosaic_bsa_select(p, q, k, **kw),
        "select_static": lambda **kw: mb.mosaic_bsa_select_static(p, q, k, **kw),
        "fwd": lambda **kw: mb.mosaic_bsa_fwd(p, q, k, v, idx, **kw),
        "bwd": lambda **kw: mb.mosaic_bsa_bwd(p, q, k, v, o, lse, d_o, idx, **kw),
        "fwd_branches": lambda **kw: mb.mosaic_bsa_fwd_branches(p, q, k, v, idx, gates, **kw),
        "bwd_branches": lambda **kw: mb.mosaic_bsa_bwd_branches(p, q, k, v, idx, gates, d_o, **kw),
        "rope": lambda **kw: mb.mosaic_bsa_rope(p, q, k, pos, **kw),
    }


BLOCK = ("select", "select_static", "fwd", "bwd", "fwd_branches", "bwd_branches", "rope")
SEQUENCE = ("rotary", "qk_norm", "qk_norm_bwd", "window_fwd", "window_bwd", "window_decode")


def made_by(call, **kw):
    """The results, and what the call took from the allocator: (stream, bytes) of each block."""
    torch.cuda.synchronize()
    torch.cuda.memory._record_memory_history(context=None, clear_history=True)
    try:
        out = call(**kw)
        trace = torch.cuda.memory._snapshot()["device_traces"][torch.cuda.current_device()]
    finally:
        torch.cuda.memory._record_memory_history(enabled=None)
    torch.cuda.synchronize()
    out = (out,) if torch.is_tensor(out) else out
    return out, [(e["stream"], e["size"]) for e in trace if e["action"] == "alloc"]


def check_memory_of_the_stream(call):
    want, here = made_by(call)
    side = torch.cuda.Stream()
    got, there = made_by(call, stream=side)
    assert all(torch.equal(a, b) for a, b in zip(want, got))
    assert all(owner(t) == side.cuda_stream for t in got)
    # the workspace too: as many blocks as on the current stream, every one of them the side stream's
    assert [n for _, n in there] == [n for _, n in here] and here
    assert all(s == side.cuda_stream for s, _ in there) and all(s == torch.cuda.current_stream().cuda_stream for s, _ in here)


def check_queued_work_is_left_alone(call):
    """A copy queued on the current stream reads blocks that have been freed since; a call on another stream, with nothing to order the
    two, makes outputs of those sizes."""
    want = call()
    want = (want,) if torch.is_tensor(want) else want
    side = torch.cuda.Stream()
    call(stream=side)  # (whatever the first call on a stream sets up)
    freed = [torch.full_like(t, 3) for t in want for _ in range(3)]
    kept = [torch.empty_like(t) for t in freed]
    torch.cuda.synchronize()
    torch.cuda._sleep(40_000_000)  # some 20 ms, so that the copies are still to come
    for a, b in zip(kept, freed):
        a.copy_(b)
    del freed, b
    got = call(stream=side)
    torch.cuda.synchronize()
    assert all((t == 3).all() for t in kept)
    assert all(torch.equal(a, b) for a, b in zip(want, got if isinstance(got, tuple) else (got,)))


def check_results_last_as_long_as_the_caller_needs_them(call):
    """Results copied on the current stream and freed; a call on their stream at once may not have their memory yet."""
    side = torch.cuda.Stream()
    want = call()
    want = [t.clone() for t in ((want,) if torch.is_tensor(want) else want)]
    got = call(stream=side)
    got = [got] if torch.is_tensor(got) else list(got)
    kept = [torch.empty_like(t) for t in got]
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda._sleep(40_000_000)
    for a, b in zip(kept, got):
        a.copy_(b)
    with torch.cuda.stream(side):  # what takes the freed blocks, if they are to be had, and writes them
        del got, b
        others = [torch.full_like(t, 5) for t in kept for _ in range(3)]
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(want, kept)) and len(others) == 3 * len(kept)


def check_captured_on_a_forked_stream(call):
    """A capture that forks to the named stream and joins it: what the call makes lives in the graph's memory."""
    want = call()
    want = [t.clone() for t in ((want,) if torch.is_tensor(want) else want)]
    side, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    call(stream=side)
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        side.wait_stream(torch.cuda.current_stream())
        out = call(stream=side)
        torch.cuda.current_stream().wait_stream(side)
    out = (out,) if torch.is_tensor(out) else out
    others = [torch.full_like(t, 5) for t in want for _ in range(3)]
    for _ in range(2):
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(want, out))
        for t in out:
            t.zero_()
    assert all((t == 5).all() for t in others)


@pytest.mark.parametrize("name", SEQUENCE)
def test_sequence_operators_captured_on_a_forked_stream(name):
    check_captured_on_a_forked_stream(sequence_calls()[name])


@pytest.mark.parametrize("name", SEQUENCE)
def test_sequence_operators_take_the_memory_of_their_stream(name):
    check_memory_of_the_stream(sequence_calls()[name])


@pytest.mark.parametrize("name", SEQUENCE)
def test_sequence_operators_leave_queued_work_alone(name):
    check_queued_work_is_left_alone(sequence_calls()[name])


@pytest.mark.parametrize("name", SEQUENCE)
def test_results_of_sequence_operators_last(name):
    check_results_last_as_long_as_the_caller_needs_them(sequence_calls()[name])


@pytest.mark.parametrize("name", BLOCK)
def test_block_sparse_calls_take_the_memory_of_their_stream(name):
    check_memory_of_the_stream(block_calls()[name])


@pytest.mark.parametrize("name", BLOCK)
def test_block_sparse_calls_leave_queued_work_alone(name):
    check_queued_work_is_left_alone(block_calls()[name])


@pytest.mark.parametrize("name", BLOCK)
def test_results_of_block_sparse_calls_last(name):
    check_results_last_as_long_as_the_caller_needs_them(block_calls()[name])


@pytest.mark.parametrize("name", BLOCK)
def test_block_sparse_calls_captured_on_a_forked_stream(name):
    check_captured_on_a_forked_stream(block_calls()[name])
