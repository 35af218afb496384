"""The sources' assembly statements name what they change: a fixed register that one writes, and
does not list as changed, may hold a value of the compiler's across it."""
import glob
import os
import re

import pytest

SOURCES = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))),
                       "paper_2608_15383_amd", "csrc")
# The first operand of an instruction other than a store, if it is a fixed register.
WRITES = re.compile(r"(?:^|\n)\s*(?!s_cmp|s_bitcmp|v_cmpx?_|s_waitcnt|s_nop|s_barrier|\w*store)\w+\s+"
                    r"(m0|vcc|exec|scc|[sva]\d+|[sva]\[\d+:\d+\])\b")


def statements(text):
    """(text of the instructions, the list of what is changed) of each assembly statement."""
    for start in re.finditer(r"\basm\b(?:\s+volatile)?\s*\(", text):
        depth, at, quoted = 1, start.end(), False
        parts, part = [], at
        while depth:
            c = text[at]
            if c == '"' and text[at - 1] != "\\":
                quoted = not quoted
            elif not quoted:
                depth += (c == "(") - (c == ")")
                if c == ":" and depth == 1 or depth == 0:
                    parts.append(text[part:at])
                    part = at + 1
            at += 1
        code = "".join(re.findall(r'"((?:[^"\\]|\\.)*)"', parts[0]))
        yield code.replace("\\n", "\n").replace("\\t", "\t"), parts[3] if len(parts) > 3 else ""


def unnamed(text):
    return [(code, r) for code, changed in statements(text) for r in WRITES.findall(code)
            if f'"{r}"' not in changed]


def test_finds_what_is_not_named():
    code = 'asm volatile("s_mov_b32 m0, %0\\n\\ts_nop 0\\n\\tcopy %1, off" ::"s"(f(to)), "v"(x) : "memory"'
    assert [r for _, r in unnamed(code + ");")] == ["m0"]
    assert unnamed(code + ', "m0");') == []
    assert unnamed('asm("" : "+v"(x)); asm volatile("" ::: "memory");') == []
    assert [r for _, r in unnamed('asm("v_mov_b32 v3, %0" :: "v"(x));')] == ["v3"]


@pytest.mark.parametrize("path", sorted(glob.glob(os.path.join(SOURCES, "*.h"))
                                        + glob.glob(os.path.join(SOURCES, "*.hip"))), ids=os.path.basename)
def test_assembly_names_the_registers_that_it_writes(path):
    assert unnamed(open(path).read()) == []
