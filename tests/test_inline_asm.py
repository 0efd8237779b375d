"""What inline assembly says of itself to the compiler."""
import glob
import os
import re

import pytest

from paper_2503_06545_amd import build


def asm_statements(text):
    """The arguments of every asm(...) of a source, line continuations taken out."""
    text = text.replace("\\\n", "\n")
    for m in re.finditer(r"\basm\s+volatile\s*\(|\basm\s*\(", text):
        depth, at, quoted = 1, m.end(), False
        while depth:
            c = text[at]
            if c == '"' and text[at - 1] != "\\":
                quoted = not quoted
            elif not quoted:
                depth += (c == "(") - (c == ")")
            at += 1
        yield text[m.end():at - 1]


def parts(statement):
    """(template, everything behind it)"""
    m = re.match(r'\s*(?:"(?:[^"\\]|\\.)*"\s*)+', statement)
    return m.group(0), statement[m.end():]


@pytest.mark.parametrize("path", sorted(glob.glob(os.path.join(build.CSRC, "*"))), ids=os.path.basename)
def test_registers_that_asm_writes_by_name_are_clobbers(path):
    """m0, the carry of scalar additions and vcc: written in a template, so the compiler has to be told."""
    if not path.endswith((".h", ".hip")):
        pytest.skip("no device code")
    for statement in asm_statements(open(path).read()):
        template, rest = parts(statement)
        for register, writes in (("m0", r"\bs_\w+\s+m0\b"), ("scc", r"\bs_(?:add|sub|addc|subb|and|or|lshl|lshr|cmp)\w*\s"), ("vcc", r"\bv_cmp\w*\s+vcc\b")):
            if re.search(writes, template.replace("\\n", "\n").replace("\\t", " ")):
                assert f'"{register}"' in rest, (os.path.basename(path), statement.strip())


def test_the_reader_finds_them():
    found = [parts(s) for s in asm_statements('asm volatile("s_mov_b32 m0, %0\\n" "x (%1)" ::"s"(f(a)) : "m0"); asm("y")')]
    assert [t.count("m0") for t, _ in found] == [1, 0] and '"m0"' in found[0][1] and found[1][1] == ""
    assert sum(t.count("s_add_u32 m0") for p in glob.glob(os.path.join(build.CSRC, "*.hip")) for t, _ in map(parts, asm_statements(open(p).read()))) == 2
