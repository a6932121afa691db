"""Inline assembly tells the compiler of every register that it names."""
import glob
import os
import re

import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2602_23999_amd", "csrc")
REGISTER = re.compile(r"\b(m0|vcc|exec|scc|[sva]\d+|[sva]\[\d+:\d+\])\b")


def _statements(text):
    """(instructions, the rest) of every asm statement: the strings up to the first colon, and what stands behind them."""
    for m in re.finditer(r"\basm\s*(?:volatile\s*)?\(", text):
        depth, at, quoted = 1, m.end(), False
        while depth:
            ch = text[at]
            if ch == '"' and text[at - 1] != "\\":
                quoted = not quoted
            elif not quoted:
                depth += (ch == "(") - (ch == ")")
            at += 1
        body = text[m.end():at - 1]
        head = re.match(r'\s*(?:"(?:[^"\\]|\\.)*"\s*)+', body)
        yield body[:head.end()].replace("\\n", " ").replace("\\t", " "), body[head.end():]


def _undeclared(text):
    return [(name, code) for code, rest in _statements(text) for name in REGISTER.findall(code) if f'"{name}"' not in rest]


def _sources():
    return sorted(glob.glob(os.path.join(CSRC, "*.h")) + glob.glob(os.path.join(CSRC, "*.hip")))


@pytest.mark.parametrize("path", _sources(), ids=os.path.basename)
def test_named_registers_are_declared(path):
    assert _undeclared(open(path).read()) == []


@pytest.mark.parametrize("path", _sources(), ids=os.path.basename)
def test_loads_to_lds_take_their_address_as_an_operand(path):
    # (they read m0, which the instruction does not name)
    for code, rest in _statements(open(path).read()):
        if "load_lds" in code:
            assert '"{m0}"' in rest


def test_the_check_sees_what_is_missing():
    assert _undeclared(r'asm volatile("s_mov_b32 m0, %0\n\ts_nop 0" ::"s"(x) : "memory");') != []
    assert _undeclared(r'asm volatile("s_mov_b32 m0, %0\n\ts_nop 0" ::"s"(x) : "memory", "m0");') == []
    assert _undeclared(r'asm("v_add_u32 %0, %1, v12" : "=v"(d) : "v"(f(x)));') != []
