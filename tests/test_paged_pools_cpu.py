"""Pools of pages whose rows overlap are refused, by what their strides say; slices and any order of the axes are not (no GPU needed)."""
import pytest
import torch

from tests.test_paged_cpu import append, built, decode, params, view  # noqa: F401 (built: the library's)

PAGES, HKV, PAGE, D = 100, 2, 16, 64
LATER = dict(table=258)  # a misaligned table, which is looked at behind the pools: no call here ever reaches a launch
TAKEN = -4               # and what it gives


def strides(shape, order, cut=lambda x: x):
    """Strides of [pages, Hkv, page] in elements: `shape` lies in memory as `order` says, of which `cut` takes a part"""
    x = torch.empty([shape[i] for i in order], device="meta").permute([order.index(i) for i in range(len(shape))])
    x = cut(x)
    assert x.shape == (PAGES, HKV, PAGE, D), x.shape
    return dict(zip(("sb", "sh", "sn"), x.stride()))


GOOD = [
    strides((PAGES, HKV, PAGE, D), (0, 1, 2, 3)),
    strides((PAGES, HKV, PAGE, D), (0, 2, 1, 3)),
    strides((PAGES, HKV, PAGE, D), (2, 1, 0, 3)),
    strides((PAGES, HKV, PAGE, D), (1, 0, 2, 3)),
    strides((PAGES, HKV, PAGE, 3 * D), (0, 1, 2, 3), lambda x: x[..., D:2 * D]),        # keys and values side by side
    strides((PAGES, 2 * HKV + 1, PAGE, D), (0, 1, 2, 3), lambda x: x[:, 1:2 * HKV:2]),  # every other head
    strides((PAGES, 2 * HKV - 1, PAGE, D), (0, 2, 1, 3), lambda x: x[:, ::2]),
    strides((2 * PAGES - 1, HKV, PAGE, D), (1, 0, 2, 3), lambda x: x[::2]),
    strides((PAGES, HKV, 2 * PAGE - 1, D), (0, 1, 2, 3), lambda x: x[:, :, ::2]),
]
BAD = [
    dict(sn=8), dict(sn=D - 8),                     # slots that begin inside the one before
    dict(sn=D, sh=8), dict(sn=D, sh=D),             # heads inside a slot, or in the same one
    dict(sn=HKV * D, sh=D - 8),
    dict(sn=D, sh=PAGE * D - 8),                    # heads that begin inside the last slot of the one before
    dict(sn=D, sh=PAGE * D, sb=PAGE * D),           # pages in one another
    dict(sn=D, sh=PAGE * D, sb=HKV * PAGE * D - 8),
    dict(sn=D, sh=PAGE * D, sb=D),
    dict(sn=1 << 30, sh=1 << 31, sb=1 << 32),
]


@pytest.mark.parametrize("st", GOOD, ids=str)
def test_other_layouts_are_taken(st):
    for at in ("k_pages", "v_pages"):
        assert append(**{at: view(**st)}, **LATER) == TAKEN and decode(**{at: view(**st)}, **LATER) == TAKEN


@pytest.mark.parametrize("st", BAD, ids=str)
def test_rows_that_overlap_are_refused(st):
    for at in ("k_pages", "v_pages"):
        assert append(**{at: view(**st)}, **LATER) == -2 and decode(**{at: view(**st)}, **LATER) == -2, at


def test_an_axis_of_one_has_no_stride_to_look_at():
    assert append(params(Hkv=1, H=4), k_pages=view(sn=D, sh=8, sb=PAGE * D), **LATER) == TAKEN
    assert append(params(pages=1), k_pages=view(sn=D, sh=PAGE * D, sb=8), **LATER) == TAKEN
    assert append(params(Hkv=1, H=4, pages=1), k_pages=view(sn=D, sh=0, sb=0), **LATER) == TAKEN


def test_extents_that_no_memory_holds_do_not_overflow():
    far = (1 << 37) - 8
    assert append(params(Hkv=1, H=4, pages=(1 << 31) - 1, page=1 << 10, width=1), k_pages=view(sn=far, sh=0, sb=far), **LATER) == -2
    assert append(params(Hkv=30000, H=30000, pages=(1 << 31) - 1), k_pages=view(sn=far, sh=far, sb=far), **LATER) == -2
