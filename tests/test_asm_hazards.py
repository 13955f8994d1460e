"""What the compiler does not see in inline assembly: the registers that a statement writes have to stand in its clobber
list (or be outputs)."""
import glob
import os
import re

import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2504_06419_amd", "csrc")


def statements(text):
    """(assembly text, clobbers) of every asm statement."""
    for m in re.finditer(r"\basm\s+volatile\s*\(", text):
        depth, at, quoted = 1, m.end(), False
        while depth:
            c = text[at]
            if c == '"' and text[at - 1] != "\\":
                quoted = not quoted
            if not quoted:
                depth += (c == "(") - (c == ")")
            at += 1
        # the four parts stand between colons outside of quotes
        parts = re.split(r":(?=(?:[^\"]*\"[^\"]*\")*[^\"]*$)", text[m.end():at - 1])
        yield parts[0], parts[3] if len(parts) > 3 else ""


def fixed_register_writes(code):
    for line in re.findall(r'"([^"]*)"', code):
        for ins in re.split(r"\\n|\\t|;", line):
            m = re.match(r"\s*(?:s|v)_\w+\s+(m0|vcc|exec|scc|[sv]\d+|[sv]\[\d+:\d+\])\b", ins)
            if m:
                yield m.group(1)


def unnamed(text):
    return [(code, reg) for code, clobbers in statements(text) for reg in fixed_register_writes(code)
            if f'"{reg}"' not in clobbers]


@pytest.mark.parametrize("text,found", [
    ('asm volatile("s_mov_b32 m0, %1\\n\\ts_nop 0" ::"v"(a), "s"(f(b)) : "memory");', 1),
    ('asm volatile("s_mov_b32 m0, %1\\n\\ts_nop 0" ::"v"(a), "s"(f(b)) : "memory", "m0");', 0),
    ('asm volatile("s_nop 0\\n\\tv_mov_b32 v7, %0" ::"v"(a));', 1),
    ('asm volatile("" : "+v"(x));', 0), ('asm volatile("s_waitcnt vmcnt(%0)" ::"n"(N) : "memory");', 0)])
def test_reading_of_statements(text, found):
    assert len(unnamed(text)) == found


def test_sources():
    seen = 0
    for path in sorted(glob.glob(os.path.join(CSRC, "*"))):
        text = open(path).read()
        seen += sum(1 for _ in statements(text))
        assert not unnamed(text), os.path.basename(path)
    assert seen > 10
