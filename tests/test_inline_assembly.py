"""Inline assembly names every register that it writes and the compiler can not see: an m0 that is set behind its back is lost to whatever it kept there."""
import glob
import os
import re

import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2601_21198_amd", "csrc")
SOURCES = sorted(glob.glob(os.path.join(CSRC, "*.hip")) + glob.glob(os.path.join(CSRC, "*.h")))


def statements(text):
    """(template, clobbers) of every asm statement"""
    for m in re.finditer(r"\basm\s*(?:volatile\s*)?\(", text):
        at, depth, parts, quoted = m.end(), 1, [""], False
        while depth:
            c = text[at]
            if c == '"' and text[at - 1] != "\\":
                quoted = not quoted
            if not quoted:
                depth += (c in "([") - (c in ")]")
            if c == ":" and depth == 1 and not quoted:
                parts.append("")
            elif depth:
                parts[-1] += c
            at += 1
        yield parts[0], re.findall(r'"(\w+)"', parts[3]) if len(parts) > 3 else []


def written(template):
    """special registers that the template's instructions have as their destination"""
    return {m.group(1) for m in re.finditer(r"\b(?:s|v)_\w+\s+(m0|vcc|exec|scc)\b", template)}


def test_the_parser_sees_what_it_should():
    found = list(statements('asm volatile("s_mov_b32 m0, %0\\n\\ts_nop 0" ::"s"(a[1]) : "memory"); asm("v_mov_b32 %0, 1" : "=v"(r));'))
    assert [c for _, c in found] == [["memory"], []] and [written(t) for t, _ in found] == [{"m0"}, set()]


@pytest.mark.parametrize("path", SOURCES, ids=os.path.basename)
def test_registers_that_are_written_are_named(path):
    for template, clobbers in statements(open(path).read()):
        assert written(template) <= set(clobbers), template
