"""The tests' inputs for the sinks' gradients tell a backward that rounds P or dS once from one that does not (no GPU needed)."""
import pytest
import torch

from tests import sinks_case as C
from tests import window_ref as ref


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
def test_one_rounding_is_beyond_the_tolerance(d, dtype):
    window, x = C.inputs(d, dtype)
    dk, dv = C.gradients(window, *x)
    for once, want, got in (("P", dv, C.gradients(window, *x, once=("P",))[1]), ("dS", dk, C.gradients(window, *x, once=("dS",))[0])):
        off, tol = (got - want).abs(), C.tolerance(window, x[0], want)
        assert (off > tol).float().mean() > 0.25, once  # (the result's own rounding makes up for it in some)
    dk1, dv1 = C.gradients(window, *x, once=("result",))
    assert ((dk1 - dk).abs() <= C.tolerance(window, x[0], dk)).all() and ((dv1 - dv).abs() <= C.tolerance(window, x[0], dv)).all()


def test_the_gradients_are_the_definition_s():
    window, x = C.inputs(64, torch.bfloat16)
    want = ref.attention(*x[:3], window, C.SINKS, 0.0, None, None, x[3])
    dk, dv = C.gradients(window, *x)
    # 64-bit sums of 3000 terms in two orders
    assert (dk - want["dk"][:, :, :C.SINKS]).abs().max() <= 1e-11 * float(dk.abs().max())
    assert (dv - want["dv"][:, :, :C.SINKS]).abs().max() <= 1e-11 * float(dv.abs().max())
