"""What the kernel right ahead on the stream writes last is what a call reads: lengths, positions, frequencies, inputs.

Kernels start before the one ahead of them has finished and wait there; nothing may be read before that wait.  The kernel ahead is a
rotation of many tokens whose passing channels hold the words that the next call reads; those of the last token are written last."""
import pytest
import torch

from paper_2604_16429_b200 import binding as mb
from tests.test_gpu_window import lens, make

pytestmark = pytest.mark.gpu


class Writer:
    """Writes up to 56 32-bit words by a rotation that takes some 100 us."""

    def __init__(self, words):
        self.rp = mb.RotaryParams(d=64, rot_dim=2)
        self.x = torch.randn(1, 8, 60000, 64, device="cuda")
        self.y, self.k = torch.zeros_like(self.x), torch.zeros(1, 8, 60000, 64, device="cuda")
        self.x.view(torch.int32)[0, 7, -1, 8:8 + words.numel()] = words
        self.at = self.y.view(torch.int32)[0, 7, -1, 8:8 + words.numel()]
        self.pos, self.fr = torch.arange(60000, device="cuda"), mb.rotary_freqs(self.rp)

    def go(self, stale):
        """`stale` stands there until the rotation, queued behind it, is done."""
        self.at.copy_(stale)
        torch.cuda.synchronize()
        mb.mosaic_bsa_rotary(self.rp, self.x, self.k, self.pos, self.fr, q_out=self.y, k_out=self.k)


def check(words, stale, view, call):
    w = Writer(words)
    want = call(view(words.clone()))
    for _ in range(5):
        w.go(stale)
        got = call(view(w.at))
        torch.cuda.synchronize()
        assert torch.equal(w.at, words)
        for a, b in zip(got, want):
            assert torch.equal(a, b)


@pytest.mark.parametrize("what", ["q_len", "k_len"])
@pytest.mark.parametrize("op", ["fwd", "bwd", "decode"])
def test_lengths(op, what):
    if op == "decode" and what == "q_len":
        return  # it has none
    wp = mb.WindowParams(window=100, sinks=4)
    q, k, v, d_o = make(4, 4, 2, 300, 300, 64, seed=1)
    full, short = lens([300, 290, 280, 299]), lens([1, 0, 2, 1])
    o, lse = mb.mosaic_bsa_window_fwd(wp, q, k, v)

    def call(n):
        kw = {what: n}
        if op == "decode":
            return mb.mosaic_bsa_window_decode(wp, q[:, :, :1], k, v, **kw)
        if op == "fwd":
            out = torch.zeros_like(q), torch.zeros_like(lse)
            return mb.mosaic_bsa_window_fwd(wp, q, k, v, o=out[0], lse=out[1], **kw)
        out = [torch.zeros_like(x) for x in (q, k, v)]
        return mb.mosaic_bsa_window_bwd(wp, q, k, v, o, lse, d_o, dq=out[0], dk=out[1], dv=out[2], **kw)

    check(full, short, lambda x: x, call)


@pytest.mark.parametrize("op", ["rotary", "qk_norm", "qk_norm_bwd"])
@pytest.mark.parametrize("what", ["freqs", "pos"])
def test_frequencies_and_positions(op, what):
    q, k, _, _ = make(1, 4, 2, 20, 20, 32, seed=2)
    rp = mb.RotaryParams(d=32)
    weights = torch.ones(32, device="cuda")
    values = {"freqs": 2.0 ** -torch.arange(16, dtype=torch.float64), "pos": torch.arange(20) * 3}
    values = {n: x.cuda() for n, x in values.items()}
    words = values[what].view(torch.int32)

    def call(x):
        kw = {**values, what: x}
        if op == "rotary":
            return mb.mosaic_bsa_rotary(rp, q, k, kw["pos"], kw["freqs"])
        if op == "qk_norm":
            return mb.mosaic_bsa_qk_norm(rp, q, k, weights, weights, kw["pos"], kw["freqs"])
        return mb.mosaic_bsa_qk_norm_bwd(rp, q, k, weights, weights, kw["pos"], kw["freqs"], q, k)

    check(words, torch.zeros_like(words), lambda x: x.view(values[what].dtype), call)
