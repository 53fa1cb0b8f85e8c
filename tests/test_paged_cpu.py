"""Refusals and workspace sizes of the paged cache's calls (no GPU needed)."""
import ctypes

import pytest

from paper_2604_16429_b200 import binding as mb
from paper_2604_16429_b200 import build as mbuild

BASE = dict(table_stride=32, start=0, B=2, H=4, Hkv=2, Nq=3, d=64, page=16, pages=100, width=32, window=0, sinks=0, prefix_len=0, rot_dim=64,
            scale=0.0, amplitude=0.0, flags=0)


@pytest.fixture(scope="module", autouse=True)
def built():
    mbuild.build()


def params(**kw):
    v = {**BASE, **kw}
    return ctypes.byref(mb._PagedParams(*(v[k] for k, _ in mb._PagedParams._fields_)))


def view(ptr=256, sb=1 << 20, sh=1 << 16, sn=64):
    return ctypes.byref(mb._View(ptr, sb, sh, sn))


def append(p=None, k=None, v=None, k_pages=None, v_pages=None, table=256, k_len=256, q_len=None, freqs=256, q=None, q_out=None):
    g = view()
    return mb.lib().mosaic_bsa_paged_append(p or params(), k or g, v or g, k_pages or g, v_pages or g, table, k_len, q_len, freqs, q, q_out, None)


ANY = [(dict(B=0), -1), (dict(Hkv=0), -1), (dict(Nq=0), -1), (dict(pages=0), -1), (dict(width=0), -1), (dict(page=0), -1),
       (dict(page=-16), -1), (dict(table_stride=-1), -1), (dict(flags=1), -1), (dict(flags=4), -1), (dict(flags=64), -1), (dict(d=32), -2),
       (dict(d=256), -2), (dict(page=8), -2), (dict(page=24), -2), (dict(page=1 << 20, width=1 << 11), -2), (dict(page=1 << 21, width=1), -2), (dict(table_stride=1 << 41), -2)]


@pytest.mark.parametrize("kw,code", ANY + [
    (dict(rot_dim=-2), -1), (dict(rot_dim=3), -1), (dict(rot_dim=66), -1), (dict(rot_dim=24, flags=8), -2), (dict(flags=16), -1),
    (dict(amplitude=-1.0), -1), (dict(amplitude=float("nan")), -1), (dict(amplitude=float("inf")), -1), (dict(start=1 << 53), -2),
    (dict(start=-(1 << 53)), -2), (dict(B=1 << 20, Nq=1 << 11), -2), (dict(Hkv=1 << 16), -2)])
def test_bad_params_of_append_are_refused(kw, code):
    assert append(params(**kw)) == code


POOLS = [(view(0), -1), (view(256 + 8), -4), (view(sn=68), -4), (view(sh=4), -4), (view(sb=-64), -1), (view(sb=1 << 40), -2),
         (view(sn=0), -2), (view(sh=0), -2), (view(sb=0), -2)]


def test_bad_tensors_of_append_are_refused():
    for x, code in POOLS:
        for at in ("k_pages", "v_pages"):
            assert append(**{at: x}) == code, at
    for x, code in POOLS[:6]:
        for at in ("k", "v"):
            assert append(**{at: x}) == code, at
        assert append(q=x, q_out=view()) == code and append(q=view(), q_out=x) == code
    assert append(q=view()) == -1 and append(q_out=view()) == -1 and append(params(H=0), q=view(), q_out=view()) == -1
    assert append(table=None) == -1 and append(k_len=None) == -1 and append(freqs=None) == -1
    assert append(table=258) == -4 and append(k_len=257) == -4 and append(q_len=254) == -4 and append(freqs=252) == -4
    assert mb.lib().mosaic_bsa_paged_append(None, view(), view(), view(), view(), 256, 256, None, 256, None, None, None) == -1
    assert mb.lib().mosaic_bsa_paged_append(params(), None, view(), view(), view(), 256, 256, None, 256, None, None, None) == -1


def decode(p=None, q=None, k_pages=None, v_pages=None, o=None, table=256, k_len=256, q_len=None, lse=256, ws=256, n=1 << 40):
    g = view()
    return mb.lib().mosaic_bsa_paged_decode(p or params(), q or g, k_pages or g, v_pages or g, table, k_len, q_len, o or g, lse, ws, n, None)


@pytest.mark.parametrize("kw,code", ANY + [
    (dict(H=3), -1), (dict(H=0), -1), (dict(window=-1), -1), (dict(sinks=-1), -1), (dict(sinks=129), -2), (dict(prefix_len=1), -1),
    (dict(prefix_len=-1), -1), (dict(Nq=17), -2), (dict(scale=float("nan")), -1), (dict(scale=float("inf")), -1), (dict(flags=8), -1),
    (dict(B=1 << 23), -2), (dict(B=1, H=1 << 20, Hkv=1), -2)])
def test_bad_params_of_decode_are_refused(kw, code):
    assert decode(params(**kw)) == code
    if kw.get("prefix_len", 0) <= 0:  # (with one it is the size for a call behind a prefix)
        assert mb.lib().mosaic_bsa_paged_workspace_bytes(params(**kw)) == 0


def test_bad_tensors_of_decode_are_refused():
    for x, code in POOLS:
        for at in ("k_pages", "v_pages"):
            assert decode(**{at: x}) == code, at
    for x, code in POOLS[:6]:
        for at in ("q", "o"):
            assert decode(**{at: x}) == code, at
    assert decode(table=None) == -1 and decode(k_len=None) == -1 and decode(lse=None) == -1 and decode(ws=None) == -1
    assert decode(table=258) == -4 and decode(k_len=257) == -4 and decode(q_len=254) == -4 and decode(lse=258) == -4 and decode(ws=272) == -4
    assert decode(n=255) == -3 and decode(params(width=33), n=256) == -3


def test_workspaces():
    ws = mb.lib().mosaic_bsa_paged_workspace_bytes
    rows = 2 * 4 * 3
    assert ws(None) == 0 and ws(params()) == 256  # 512 tokens at most: one part, which is the result
    part = lambda n: 256 + n * rows * 64 * 4 + -(-n * rows * 8 // 256) * 256  # noqa: E731
    assert ws(params(width=33)) == part(2) and ws(params(width=320)) == part(10)
    assert ws(params(width=320, window=1)) == part(2) and ws(params(width=320, window=512)) == part(3)   # 514 keys end to end: three chunks
    assert ws(params(width=320, window=512, sinks=1)) == part(4) and ws(params(width=33, window=512, sinks=1)) == part(2)


def prefix(p=None, table=256, prefix_table=256, k_len=256, lse=256, ws=256, n=1 << 40, q=None):
    g = view()
    return mb.lib().mosaic_bsa_prefix_decode(p or params(prefix_len=1000), q or g, g, g, prefix_table, table, k_len, None, g, lse, ws, n, None)


@pytest.mark.parametrize("kw,code", ANY + [
    (dict(H=3), -1), (dict(window=5), -1), (dict(sinks=1), -1), (dict(prefix_len=0), -1), (dict(prefix_len=-1), -1), (dict(Nq=17), -2),
    (dict(prefix_len=(1 << 30) + 1), -2), (dict(scale=float("nan")), -1), (dict(flags=32), -1)])
def test_bad_params_behind_a_prefix_are_refused(kw, code):
    kw = {"prefix_len": 1000, **kw}
    assert prefix(params(**kw)) == code
    if kw["prefix_len"]:
        assert mb.lib().mosaic_bsa_paged_workspace_bytes(params(**kw)) == 0


def test_bad_tensors_behind_a_prefix_are_refused():
    assert prefix(prefix_table=None) == -1 and prefix(prefix_table=258) == -4 and prefix(table=None) == -1 and prefix(k_len=None) == -1
    assert prefix(lse=None) == -1 and prefix(ws=None) == -1 and prefix(ws=272) == -4 and prefix(n=4096) == -3
    assert prefix(q=view(256 + 8)) == -4 and prefix(q=view(0)) == -1


def test_parts_of_a_prefix():
    """The workspace holds the prefix' parts in front of the members' own: at least one, no more than steps of 64 keys or twice the SMs."""
    ws = mb.lib().mosaic_bsa_paged_workspace_bytes
    for B, H, Hkv, Nq, d in ((1, 1, 1, 1, 64), (64, 16, 4, 1, 128), (256, 16, 4, 4, 128), (33, 24, 3, 16, 64)):
        for n in (1, 64, 65, 1000, 8191, 32768, 1 << 20, 1 << 30):
            kw = dict(B=B, H=H, Hkv=Hkv, Nq=Nq, d=d, prefix_len=n)
            rows = B * H * Nq
            parts = (ws(params(**kw)) - 256) // (rows * (d * 4 + 8))  # (a member's own 512 tokens are one part, kept if the join is apart)
            assert 1 <= parts <= min(-(-n // 64), 2 * 148 // Hkv + 2) + 1, (kw, parts)
    assert ws(params(prefix_len=64)) == 256 + 24 * 64 * 4 + 256 and ws(params(prefix_len=64, width=33)) == 256 + 3 * 24 * 64 * 4 + 3 * 256
