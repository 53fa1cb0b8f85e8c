"""A head's results of the sliding-window attention are the same bits wherever the head stands in its group, and alone."""
import pytest
import torch

from paper_2604_16429_b200 import binding as mb
from tests.test_gpu_window import lens, make

pytestmark = pytest.mark.gpu

CASES = [  # query heads of a group, d, Nq, Nk, window, sinks, q_len, k_len
    (3, 64, 400, 400, 100, 0, None, None),
    (5, 64, 700, 700, 33, 7, None, None),
    (3, 128, 520, 520, 129, 100, None, None),
    (5, 128, 300, 300, 64, 128, None, None),
    (3, 64, 900, 900, 1, 1, None, None),
    (7, 128, 333, 333, 1000, 5, None, None),
    (3, 64, 300, 900, 150, 3, [300, 17, 129], [900, 500, 129]),
    (5, 128, 300, 900, 97, 70, [299, 300, 200], [901 - 7, 300, 150]),
    (2, 64, 300, 900, 200, 40, [300, 290, 1], [777, 333, 500]),
]


@pytest.mark.parametrize("case", CASES, ids=str)
@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
def test_the_place_in_a_group_does_not_matter(case, dtype):
    G, d, Nq, Nk, window, sinks, q_len, k_len = case
    B = len(q_len) if q_len else 2
    wp = mb.WindowParams(window=window, sinks=sinks)
    q, k, v, d_o = make(B, 2 * G, 2, Nq, Nk, d, dtype, seed=Nk + window)
    kw = dict(q_len=lens(q_len), k_len=lens(k_len))

    def both(q, k, v, d_o):
        o, lse = torch.zeros_like(q), torch.zeros(q.shape[:3], device="cuda")  # (rows behind a sequence stay as they are)
        mb.mosaic_bsa_window_fwd(wp, q, k, v, o=o, lse=lse, **kw)
        dq = torch.zeros_like(q)
        mb.mosaic_bsa_window_bwd(wp, q, k, v, o, lse, d_o, dq=dq, **kw)
        return o, lse, dq

    # different heads: each alone with its key head
    want = both(q, k, v, d_o)
    for h in range(2 * G):
        one = both(q[:, h:h + 1], k[:, h // G:h // G + 1], v[:, h // G:h // G + 1], d_o[:, h:h + 1])
        for name, a, b in zip(("o", "lse", "dq"), one, want):
            assert torch.equal(a, b[:, h:h + 1]), f"{name} of head {h}"
    # equal heads
    same = both(q[:, :1].expand(q.shape), k[:, :1].expand(k.shape), v[:, :1].expand(v.shape), d_o[:, :1].expand(d_o.shape))
    for name, a in zip(("o", "lse", "dq"), same):
        assert torch.equal(a, a[:, :1].expand(a.shape)), name
