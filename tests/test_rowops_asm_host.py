"""Inline assembly of the row operators' kernels.  A load whose result lands in a
register must be one that the compiler knows of: an inline one counts as done at once, so
that its register may be moved or given away while the data are on their way."""

import os
import re

import pytest

from test_host_sanitizers import ROOT

CSRC = os.path.join(ROOT, "paper_2606_19163_amd", "csrc")
SOURCES = ["lin8.hip", "kgrad.hip", "ldscopy.hpp", "rowvec.hpp", "keepvec.hpp", "bnorm.hip", "keep.hip"]


def inline_asm(text):
    """(instructions, whether it has outputs) of every asm statement."""
    text = re.sub(r"//[^\n]*", "", text)
    for m in re.finditer(r"\basm\s+volatile\s*\((.*?)\)\s*;", text, re.S):
        code = re.match(r'(\s*"[^"]*")+', m.group(1)).group(0)
        yield code, bool(re.search(r':\s*(\[\w+\]\s*)?"[=+]', m.group(1)[len(code):]))


@pytest.mark.parametrize("name", SOURCES)
def test_no_inline_load_into_a_register(name):
    with open(os.path.join(CSRC, name)) as f:
        for code, outputs in inline_asm(f.read()):
            load = re.search(r"\b(ds_read|ds_load|(global|buffer|flat|scratch|s)_load)\w*", code)
            if load and "_lds" not in load.group(0):
                assert not outputs, (name, code)


def test_what_the_search_finds():
    found = list(inline_asm('''
        asm volatile("ds_read_b128 %0, %1 offset:%2" : "=v"(v) : "v"(addr), "i"(OFF));
        asm volatile("s_nop 0\\n\\tglobal_load_lds_dwordx4 %0, off" ::"v"(p), "{m0}"(q) : "memory");
        asm volatile("" : "+v"(at));  // asm volatile("ds_read" : "=v"(x))
    '''))
    assert [out for _, out in found] == [True, False, True]
    assert "ds_read_b128" in found[0][0] and "global_load_lds" in found[1][0]
