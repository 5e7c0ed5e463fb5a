"""Assembly written in the kernels leaves the compiler's registers alone: a
register with a name of its own (M0, which holds the LDS address of a global ->
LDS copy) is an operand of the statement, so that the compiler knows of it, or
is saved first and restored last.  A reserved register cannot be declared as
overwritten, so there is no third way."""
import glob
import os
import re

import pytest

from paper_2603_04359_amd import build as b

SOURCES = sorted(glob.glob(os.path.join(b.CSRC, "*.hip")) + glob.glob(os.path.join(b.CSRC, "*.h")))


def _statements(text):
    """The instructions of every asm statement, one list each."""
    text = re.sub(r"//[^\n]*", "", text)
    for m in re.finditer(r"\basm\s*(?:volatile)?\s*\(((?:\s*\"(?:[^\"\\]|\\.)*\")+)", text):
        lines = "".join(re.findall(r"\"((?:[^\"\\]|\\.)*)\"", m.group(1)))
        yield [x.strip() for x in re.split(r"\\n|;", lines.replace("\\t", " ")) if x.strip()]


def _restored(ins):
    """M0 is written only between a save to an operand and its restoration."""
    if not any(re.match(r"\S+\s+m0\b", x) for x in ins):
        return True
    save = re.fullmatch(r"s_mov_b32\s+(%\d+),\s*m0", ins[0])
    return bool(save) and re.fullmatch(r"s_mov_b32\s+m0,\s*" + re.escape(save.group(1)), ins[-1]) is not None


def test_the_reader_sees_both_kinds():
    text = 'asm volatile("s_mov_b32 m0, %1\\n\\t" "s_nop 0" ::"s"(x)); // asm("s_mov_b32 m0, 0")\n' \
           'asm volatile(\n "s_mov_b32 %0, m0\\n\\t"\n "s_mov_b32 m0, %1\\n\\t"\n "s_mov_b32 m0, %0" : "=&s"(y));'
    got = list(_statements(text))
    assert got == [["s_mov_b32 m0, %1", "s_nop 0"],
                   ["s_mov_b32 %0, m0", "s_mov_b32 m0, %1", "s_mov_b32 m0, %0"]]
    assert [_restored(x) for x in got] == [False, True]


@pytest.mark.parametrize("path", SOURCES, ids=os.path.basename)
def test_m0_is_an_operand_or_restored(path):
    with open(path) as f:
        bad = [ins for ins in _statements(f.read()) if not _restored(ins)]
    assert not bad, bad
