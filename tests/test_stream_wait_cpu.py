"""What a kernel reads through the read-only path it may read ahead of its wait for the stream, unless the address holds the wait's
result: the sources are looked through for lengths and tables read at addresses that do not (no GPU needed)."""
import os
import re

import pytest

from paper_2604_16429_b200 import build as mbuild

KERNELS = [("paged_append.cu", "append_kernel"), ("paged_decode.cu", "paged_join_kernel"), ("window_bwd.cu", "window_rows_kernel"),
           ("window_bwd.cu", "window_sinks_kernel")]


def body(source, kernel):
    text = re.sub(r"//[^\n]*", "", open(os.path.join(mbuild.CSRC, source)).read())
    at = text.index("{", text.index(kernel + "("))
    depth, end = 0, at
    while True:
        depth += {"{": 1, "}": -1}.get(text[end], 0)
        end += 1
        if depth == 0:
            return text[at:end]


def arguments(text, name):
    """Argument lists of the calls of `name`"""
    for m in re.finditer(re.escape(name) + r"\(", text):
        depth, end = 1, m.end()
        while depth:
            depth += {"(": 1, ")": -1}.get(text[end], 0)
            end += 1
        yield text[m.end():end - 1]


def names(text):
    """Names in an expression (not those of members)"""
    return set(re.findall(r"(?<![\w.:])[A-Za-z_]\w*", text))


def holders(text):
    """Names that the wait's result takes part in: `name = expression` and `name += expression`, one from another"""
    made = re.findall(r"\b(\w+) \+?= ((?:(?!, \w+ = )[^;])*)", text)
    found = {"await_stream"}
    while True:
        more = {n for n, e in made if found & names(e)} - found
        if not more:
            return found
        found |= more


@pytest.mark.parametrize("source,kernel", KERNELS)
def test_lengths_and_tables_are_read_behind_the_wait(source, kernel):
    text = body(source, kernel)
    held = holders(text)
    reads = list(arguments(text, "span_of")) + [x for x in arguments(text, "__ldg")]
    assert reads
    for x in reads:
        assert held & names(x), f"{kernel} reads {x} at an address that does not hold the wait's result"
