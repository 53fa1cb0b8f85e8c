"""Calls that are too large for the list of items are refused before anything is launched, and have no workspace (no GPU needed)."""
import pytest

from paper_2604_16429_b200 import binding as mb
from tests.test_paged_cpu import built, params, view  # noqa: F401 (built: the library's)

# members, query and key heads, new tokens, head dimension, page, width: items that weigh 2^31 and more in all
TOO_MANY = [dict(B=1 << 8, H=4, Hkv=2, Nq=1, d=128, page=1 << 10, width=1 << 20), dict(B=1 << 20, H=16, Hkv=16, Nq=1, d=64, page=512, width=16),
            dict(B=1 << 10, H=64, Hkv=1, Nq=16, d=128, page=1 << 15, width=1 << 10)]
NO_ROOM = 1 << 10  # bytes of workspace: a call that is not too large is refused for that, so none here is ever launched


def decode(p):
    g = view(sb=1 << 36, sh=1 << 31, sn=128)
    return mb.lib().mosaic_bsa_paged_decode(p, g, g, g, 256, 256, None, g, 256, 256, NO_ROOM, None)


def prefix(p):
    g = view(sb=1 << 36, sh=1 << 31, sn=128)
    return mb.lib().mosaic_bsa_prefix_decode(p, g, g, g, 256, 256, 256, None, g, 256, 256, NO_ROOM, None)


@pytest.mark.parametrize("kw", TOO_MANY, ids=str)
def test_too_many_items(kw):
    p = {"pages": 1 << 20, **kw}
    assert decode(params(**p)) == -2 and prefix(params(**p, prefix_len=1000)) == -2
    assert mb.lib().mosaic_bsa_paged_workspace_bytes(params(**p)) == 0 and mb.lib().mosaic_bsa_paged_workspace_bytes(params(**p, prefix_len=9)) == 0


@pytest.mark.parametrize("kw", TOO_MANY, ids=str)
def test_a_window_makes_them_few(kw):
    p = {"pages": 1 << 20, **kw, "window": 100}
    if kw["B"] < 1 << 20:
        assert decode(params(**p)) == -3 and mb.lib().mosaic_bsa_paged_workspace_bytes(params(**p)) > NO_ROOM


def test_the_last_that_is_taken():
    """2^20 heads of 170 and 171 chunks of 512 keys, each of weight 12."""
    p = dict(B=1 << 18, H=4, Hkv=4, Nq=1, d=64, page=512, pages=1 << 20)
    assert decode(params(**p, width=170)) == -3 and prefix(params(**p, width=170, prefix_len=1000)) == -3
    assert decode(params(**p, width=171)) == -2 and prefix(params(**p, width=171, prefix_len=1000)) == -2
