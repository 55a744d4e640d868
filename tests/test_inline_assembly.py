"""Inline assembly says what it writes: a register that a statement sets without naming it may hold a value of the compiler's."""
import os
import re

import pytest

from paper_2510_19482_amd import build

SOURCES = sorted(n for n in os.listdir(build.CSRC) if n.endswith((".hip", ".h")))


def statements(text):
    """The text between the brackets of each asm statement."""
    for found in re.finditer(r"\basm\b(?:\s+volatile)?\s*\(", text):
        depth, at, quoted = 1, found.end(), False
        while depth:
            c = text[at]
            if c == '"' and text[at - 1] != "\\":
                quoted = not quoted
            elif not quoted:
                depth += (c == "(") - (c == ")")
            at += 1
        yield text[found.end():at - 1]


@pytest.mark.parametrize("name", SOURCES)
def test_m0_is_named_where_it_is_written(name):
    for asm in statements(open(os.path.join(build.CSRC, name)).read()):
        if re.search(r"\bs_mov_b32 m0\b", asm):
            assert re.search(r'"m0"\s*(,|$)', asm.rsplit(":", 1)[1]), asm


def test_the_statements_are_found():
    every = [s for n in SOURCES for s in statements(open(os.path.join(build.CSRC, n)).read())]
    assert sum("s_mov_b32 m0" in s for s in every) >= 3 and sum("s_waitcnt" in s for s in every) >= 3
    assert list(statements('asm volatile("a (b" ::"v"(x) : "memory"); asm("" : "+v"(y));')) == ['"a (b" ::"v"(x) : "memory"', '"" : "+v"(y)']
