"""Inline assembly in the kernel sources: what it writes is declared."""
import os
import re

import pytest

from paper_2503_22796_amd import build


def _asm_statements(text):
    """Every asm statement's text, up to the end of its parentheses."""
    for m in re.finditer(r"\basm\s+volatile\s*\(", text):
        depth, at = 1, m.end()
        while depth:
            c = text[at]
            if c == '"':                          # a string: to its end
                at = re.compile(r'"(?:[^"\\]|\\.)*"').match(text, at).end()
                continue
            depth += (c == "(") - (c == ")")
            at += 1
        yield text[m.start():at]


@pytest.mark.parametrize("source", build.KERNEL_SOURCES)
def test_statements_that_write_m0_declare_it(source):
    with open(os.path.join(build.CSRC, source)) as f:
        text = f.read()
    for s in _asm_statements(text):
        if re.search(r"s_mov_b32 m0\b", s):
            assert '"m0"' in s.rsplit(":", 1)[1], s


def test_statements_are_found():
    text = 'x; asm volatile("a (\\" b" :: "v"(f(1)) : "memory"); asm volatile("s_mov_b32 m0, %0" :: "s"(y) : "m0");'
    assert list(_asm_statements(text)) == ['asm volatile("a (\\" b" :: "v"(f(1)) : "memory")', 'asm volatile("s_mov_b32 m0, %0" :: "s"(y) : "m0")']
