"""Where a call on a stream of the caller's takes its memory from (no GPU needed: the allocator and the streams are stand-ins)."""
import ast
import contextlib
import inspect

import pytest
import torch

from paper_2604_16429_b200 import binding as mb

SEQUENCE = ("mosaic_bsa_rotary", "mosaic_bsa_qk_norm", "mosaic_bsa_qk_norm_bwd", "mosaic_bsa_window_fwd", "mosaic_bsa_window_bwd",
            "mosaic_bsa_window_decode", "_window_ws")
BLOCK = ("mosaic_bsa_select", "mosaic_bsa_select_static", "mosaic_bsa_fwd", "mosaic_bsa_fwd_branches", "mosaic_bsa_bwd",
         "mosaic_bsa_bwd_branches", "mosaic_bsa_rope")


class FakeTensor:
    device = "cuda:0"

    def __init__(self, made_on):
        self.made_on, self.recorded = made_on, []

    def record_stream(self, s):
        self.recorded.append(s)


@pytest.fixture
def streams(monkeypatch):
    """torch.cuda's idea of the current stream, by name"""
    now = ["current"]

    @contextlib.contextmanager
    def on(s):
        now.append(s)
        yield
        now.pop()

    monkeypatch.setattr(torch.cuda, "stream", on)
    monkeypatch.setattr(torch.cuda, "current_stream", lambda device=None: now[-1])
    return now


def test_a_call_takes_its_memory_on_its_stream(streams):
    make = lambda: FakeTensor(streams[-1])  # noqa: E731
    t = mb._on("side", make)
    assert t.made_on == "side" and t.recorded == []  # a workspace: freed and used on one stream
    t = mb._new("side", make)
    assert t.made_on == "side" and t.recorded == ["current"]  # a result: the caller goes on with it
    for f in (mb._on, mb._new):
        t = f(None, make)
        assert t.made_on == "current" and t.recorded == []
    assert streams == ["current"]


def test_the_allocations_of_the_sequence_operators(streams, monkeypatch):
    for f in ("empty", "empty_like", "empty_strided"):
        monkeypatch.setattr(torch, f, lambda *a, **kw: FakeTensor(streams[-1]))
    q = FakeTensor("current")
    q.shape = (2, 3, 4, 64)
    for stream, where in ((None, "current"), ("side", "side")):
        for t in (mb._like(q, stream), mb._floats(64, 0, stream), mb._rows_like(q, stream)):
            assert t.made_on == where and t.recorded == (["current"] if stream else [])
        t = mb._scratch(256, "entry point", 0, None, stream)
        assert t.made_on == where and t.recorded == []


@pytest.mark.parametrize("name", SEQUENCE + BLOCK)
def test_no_call_allocates_past_its_stream(name):
    """The entry points leave it to the functions above to call torch's allocation functions."""
    tree = ast.parse(inspect.getsource(getattr(mb, name)))
    for call in (n for n in ast.walk(tree) if isinstance(n, ast.Call)):
        what = ast.unparse(call.func)
        assert what not in ("torch.empty", "torch.empty_like", "torch.empty_strided", "alloc_workspace"), ast.unparse(call)
