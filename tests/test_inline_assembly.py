"""Assembly text in the kernels holds no instructions: the compiler inserts the
wait states that a matrix instruction's result needs before a vector instruction
reads it for the instructions it knows, and none for a statement's text. (Empty
statements, which only tie values to registers, are fine.)"""

import glob
import os
import re

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
ASM = re.compile(r'\b(?:__asm__|__asm|asm)\b(?:\s+(?:__volatile__|volatile))*\s*\(\s*((?:"(?:[^"\\]|\\.)*"\s*)+)')


def _texts(source):
    source = re.sub(r"//[^\n]*|/\*.*?\*/", "", source, flags=re.S)
    return ["".join(re.findall(r'"((?:[^"\\]|\\.)*)"', m)) for m in ASM.findall(source)]


def test_the_search_finds_statements():
    got = _texts('asm volatile("" : "+v"(x)); asm("v_a %0"\n "v_b" : "=v"(r)); // asm("v_c")')
    assert got == ["", "v_a %0v_b"]


def test_no_instructions_in_assembly_text():
    files = sorted(glob.glob(os.path.join(ROOT, "paper_2609_08131_amd", "csrc", "*")))
    assert files
    found = {}
    for path in files:
        if path.endswith((".hip", ".hpp")):
            with open(path) as f:
                found[os.path.basename(path)] = [t for t in _texts(f.read()) if t.strip()]
    assert {k: v for k, v in found.items() if v} == {}
