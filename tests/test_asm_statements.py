"""What the kernels' sources write out as instructions (CPU).

The compiler puts the pauses that this hardware needs between dependent
instructions only where it knows both: before an instruction of an asm
statement it puts none.  So asm statements hold waits, barriers and copies into
LDS (with the pauses that those need among them) and nothing that computes."""
import glob
import os
import re

import pytest

import paper_2510_23346_amd as bd

CSRC = os.path.join(os.path.dirname(os.path.abspath(bd.__file__)), "csrc")


def _statements():
    """(file, instructions, the whole statement) of every asm statement."""
    out = []
    for path in sorted(glob.glob(os.path.join(CSRC, "*.h")) + glob.glob(os.path.join(CSRC, "*.hip"))):
        text = re.sub(r"//[^\n]*", "", open(path).read())
        for m in re.finditer(r"\basm\s*(?:volatile\s*)?\(", text):
            depth, at = 1, m.end()
            while depth:
                depth += {"(": 1, ")": -1}.get(text[at], 0)
                at += 1
            whole = text[m.start():at]
            code = re.match(r'\s*((?:"(?:[^"\\]|\\.)*"\s*)*)', text[m.end():at])[1]
            code = "".join(re.findall(r'"((?:[^"\\]|\\.)*)"', code)).replace("\\n", "\n").replace("\\t", " ")
            out.append((os.path.basename(path), [x.strip() for x in code.split("\n") if x.strip()], whole))
    return out


def test_there_are_statements():
    assert sum(1 for s in _statements() if s[1]) >= 6


@pytest.mark.parametrize("file,code", [(f, "; ".join(c)) for f, c, _ in _statements() if c])
def test_asm_statements_compute_nothing(file, code):
    for x in code.split("; "):
        assert re.match(r"(s_waitcnt|s_barrier|s_nop|s_mov_b32 m0|buffer_load_dwordx4 .* lds$)", x), (file, x)


@pytest.mark.parametrize("file,code,whole", [(f, "; ".join(c), w) for f, c, w in _statements() if c])
def test_what_statements_write_is_named(file, code, whole):
    written = re.findall(r"s_mov_b32 (\w+),", code)
    clobbers = whole.rsplit(":", 1)[1] if whole.count(":") >= 3 else ""
    for r in written:
        assert f'"{r}"' in clobbers, (file, whole)
