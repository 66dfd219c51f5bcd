"""Rules of the device code that no result shows reliably, read off the sources.  No GPU."""
import glob
import os
import re

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
FILES = sorted(glob.glob(os.path.join(ROOT, "paper_2603_14371_amd", "**", "*.h*"), recursive=True))


def code_of(path):
    """Without comments."""
    text = open(path).read()
    return re.sub(r"//[^\n]*", "", re.sub(r"/\*.*?\*/", "", text, flags=re.S))


def asm_texts(code):
    """The instruction texts of inline assembly statements."""
    texts = []
    for m in re.finditer(r"\basm\b\s*(?:volatile\s*)?\(((?:\s*\"(?:[^\"\\]|\\.)*\")+)", code):
        parts = re.findall(r"\"((?:[^\"\\]|\\.)*)\"", m.group(1))
        texts.append("".join(parts).replace("\\t", " ").replace("\\n", "\n"))
    return texts


@pytest.mark.parametrize("path", FILES, ids=os.path.basename)
def test_inline_assembly_only_stores(path):
    """A reader of a matrix instruction's result has to keep a distance that the hardware does not enforce.  The compiler
    places the wait states for its own instructions and not for the text of inline assembly, which may therefore
    compute nothing: stores, whose data have passed through vector instructions, and wait states."""
    for text in asm_texts(code_of(path)):
        for line in filter(None, (x.strip() for x in text.split("\n"))):
            assert re.match(r"(global_store_\w+|s_nop)\b", line), line


def test_the_reader_of_inline_assembly_reads():
    code = 'asm("v_max3_f32 %0, %1, %2, %3" : "=v"(r));\nasm volatile("" : "+v"(x));\nasm volatile("a %0\\n\\t"\n "s_nop 1" ::"v"(d));'
    assert asm_texts(code) == ["v_max3_f32 %0, %1, %2, %3", "", "a %0\n s_nop 1"]


def conditional_exchanges(code):
    """Statements in which a lane exchange is computed only where something else is true: to the right of &&, || or ?."""
    return [s.strip() for s in re.split(r"[;{}]", code) if re.search(r"(&&|\|\||\?).*(__shfl\w*|ds_bpermute)\s*\(", s, re.S)]


@pytest.mark.parametrize("path", FILES, ids=os.path.basename)
def test_lanes_that_are_read_from_take_part(path):
    """A lane that is switched off gives nothing to one that reads from it."""
    assert not conditional_exchanges(code_of(path))


def test_the_reader_of_exchanges_reads():
    assert conditional_exchanges("x = __ballot(i + 1 < n &&\n __shfl(s, i + 1) == s + 1) & 0xffu;\ny = a ? __shfl(b, c) : 0;")
    assert not conditional_exchanges("const int y = __shfl(s, i + 1);\nx = __ballot(i + 1 < n && y == s + 1); if (a && b) { c = __shfl(d, e); }")
