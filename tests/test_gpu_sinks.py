"""The sinks' gradients, both of them, are as exact as results rounded once: the second products of P and of dS are there."""
import pytest
import torch

from paper_2604_16429_b200 import binding as mb
from tests import sinks_case as C

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
def test_the_sinks_gradients_round_once(d, dtype):
    window, (q, k, v, d_o) = C.inputs(d, dtype, "cuda")
    wp = mb.WindowParams(window=window, sinks=C.SINKS)
    o, lse = mb.mosaic_bsa_window_fwd(wp, q, k, v)
    assert (o[:, :, C.SINKS:, 0] == 0).all()
    _, dk, dv = mb.mosaic_bsa_window_bwd(wp, q, k, v, o, lse, d_o)
    for name, got, want in zip(("dk", "dv"), (dk, dv), C.gradients(window, q, k, v, d_o)):
        off, tol = (got[:, :, :C.SINKS].double() - want).abs(), C.tolerance(window, q, want)
        assert (off <= tol).all(), f"{name}: off by {float((off / want.abs()).max()):.3g} of it, {float((tol / want.abs()).max()):.3g} allowed"
