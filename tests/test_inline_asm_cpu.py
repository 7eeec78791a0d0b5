"""What inline assembly in the kernels' sources writes without a result operand has to be named as clobbered (CPU: reads the sources)."""
import glob
import os
import re

import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_1801_08058_amd", "csrc")


def _statements(text):
    """The text of every asm statement, up to the parenthesis that closes it (strings skipped)."""
    for m in re.finditer(r"\basm\s+volatile\s*\(", text):
        depth, i, quoted = 1, m.end(), False
        while depth:
            c = text[i]
            if quoted:
                i += c == "\\"
                quoted = c != '"'
            elif c == '"':
                quoted = True
            else:
                depth += (c == "(") - (c == ")")
            i += 1
        yield text[m.end():i - 1]


def _code(statement):
    return "".join(re.findall(r'"((?:[^"\\]|\\.)*)"', re.split(r":", re.sub(r'"(?:[^"\\]|\\.)*"', lambda s: s.group().replace(":", "\0"), statement), maxsplit=1)[0]))


def test_the_reader_finds_statements():
    found = list(_statements('x; asm volatile("s_nop 1\\n\\ts_mov_b32 m0, %0" ::"s"(f(a)) : "m0"); asm volatile("" ::: "memory");'))
    assert len(found) == 2 and "m0, %0" in _code(found[0]) and found[0].rstrip().endswith('"m0"') and _code(found[1]) == ""


@pytest.mark.parametrize("path", sorted(glob.glob(os.path.join(CSRC, "*.h*"))), ids=os.path.basename)
def test_m0_is_named_where_it_is_written(path):
    with open(path) as f:
        text = f.read()
    for s in _statements(text):
        if re.search(r"\bs_\w+\s+m0\b", _code(s)):
            assert '"m0"' in s, s
