"""Inline PTX in the kernel sources: an output that is written before the last input has been read needs an early clobber
("=&r"), or the compiler may give both one register and the input is read too late."""
import glob
import os
import re

import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2603_24517_b200", "csrc")
OPERAND_MACROS = {"ATTN_R4": '"=r"', "ATTN_W4": '"r"'}  # four operands each


def asm_statements(source):
    """(line, body) of every asm(...) in a source text."""
    for m in re.finditer(r"\basm(?:\s+volatile)?\s*\(", source):
        at, depth, quoted = m.end(), 1, False
        while depth:
            c = source[at]
            if quoted:
                at += c == "\\"
                quoted = c != '"'
            elif c == '"':
                quoted = True
            else:
                depth += (c == "(") - (c == ")")
            at += 1
        yield source.count("\n", 0, m.start()) + 1, source[m.end():at - 1]


def late_reads(body):
    """Output operands without early clobber that are written by an instruction before one that reads an input."""
    text = re.match(r'\s*(?:"(?:[^"\\]|\\.)*"\s*)+', body)
    code = "".join(re.findall(r'"((?:[^"\\]|\\.)*)"', text.group(0)))
    for name, one in OPERAND_MACROS.items():
        body = re.sub(name + r"\([^)]*\)", ", ".join([one] * 4), body)
    rest = re.sub(r"//[^\n]*", "", body[re.match(r'\s*(?:"(?:[^"\\]|\\.)*"\s*)+', body).end():])
    constraints = re.findall(r'"([=+&a-zA-Z]+)"', rest)
    outputs = [c for c in constraints if c.startswith("=")]
    steps = [re.findall(r"(?<!%)%(\d+)", part) for part in code.replace("\\n", " ").replace("\\t", " ").split(";")]
    reads = [i for i, ops in enumerate(steps) if any(int(o) >= len(outputs) for o in ops)]
    bad = []
    for n, c in enumerate(outputs):
        written = [i for i, ops in enumerate(steps) if str(n) in ops]
        if written and reads and written[0] < reads[-1] and "&" not in c:
            bad.append(n)
    return bad


def test_the_rule_itself():
    assert late_reads('"mov.u32 %1, 0;\\n\\t" "ld.shared.u32 %0, [%2];" : "=r"(a), "=r"(b) : "r"(p)') == [1]
    assert late_reads('"mov.u32 %1, 0;\\n\\t" "ld.shared.u32 %0, [%2];" : "=r"(a), "=&r"(b) : "r"(p)') == []
    assert late_reads('"ld.shared.u32 %0, [%1];" : "=r"(a) : "r"(p) : "memory"') == []


@pytest.mark.parametrize("path", sorted(glob.glob(os.path.join(CSRC, "*.cu*"))), ids=os.path.basename)
def test_outputs_keep_clear_of_inputs(path):
    with open(path) as f:
        source = f.read()
    bad = [(line, late_reads(body)) for line, body in asm_statements(source)]
    assert [b for b in bad if b[1]] == []
