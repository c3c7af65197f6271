"""What an inline assembly statement writes besides its operands is named: the compiler may keep M0, SCC, VCC or EXEC over it."""
import glob
import os
import re

import pytest

from paper_2508_08256_amd import build


def _statements(text):
    """(assembly text, clobbered names) of the asm statements of a source."""
    for m in re.finditer(r"\basm\s*(?:volatile\s*)?\(", text):
        depth, at = 1, m.end()
        while depth:  # parentheses in the strings are balanced (global check below)
            depth += {"(": 1, ")": -1}.get(text[at], 0)
            at += 1
        body = text[m.end():at - 1]
        code = re.match(r'\s*((?:"(?:[^"\\]|\\.)*"\s*)+)', body)
        yield "".join(re.findall(r'"((?:[^"\\]|\\.)*)"', code[1])), set(re.findall(r'"(\w+)"', body.rsplit(":", 1)[-1]))


def _unnamed(text):
    bad = []
    for code, named in _statements(text):
        for line in code.replace("\\t", " ").split("\\n"):
            written = re.match(r"\s*[sv]_\w+\s+(m0|vcc|exec)\b", line)
            if written and written[1] not in named:
                bad.append(line.strip())
    return bad


@pytest.mark.parametrize("path", sorted(glob.glob(os.path.join(build.CSRC, "*"))), ids=os.path.basename)
def test_registers_written_by_assembly_are_named(path):
    assert not _unnamed(open(path).read())


def test_the_check_itself():
    bad = 'asm volatile("s_mov_b32 m0, %0\\n\\ts_nop 0" ::"s"(f(x)) : "memory");'
    assert _unnamed(bad) == ["s_mov_b32 m0, %0"] and not _unnamed(bad.replace('"memory"', '"memory", "m0"'))
    assert not _unnamed('asm volatile("v_pk_min_f16 %0, %1, %2" : "=v"(d) : "v"(a), "v"(b));')
