"""Inline assembly in the kernels waits, or does nothing: the compiler does not know how long an instruction in a string takes, nor how long after a matrix
instruction its result may be read, so that whatever computes has to be an instruction that the compiler chose."""
import os
import re

import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2404_04541_amd", "csrc")
SOURCES = sorted(f for f in os.listdir(CSRC) if f.endswith((".hip", ".hpp")))


@pytest.mark.parametrize("name", SOURCES)
def test_inline_assembly_does_not_compute(name):
    text = re.sub(r"//[^\n]*|/\*.*?\*/", "", open(os.path.join(CSRC, name)).read(), flags=re.S)
    for code in re.findall(r"\b(?:asm|__asm__)\s*(?:volatile|__volatile__)?\s*\(\s*((?:\"[^\"]*\"\s*)*)", text):
        lines = [line.strip() for part in re.findall(r"\"([^\"]*)\"", code) for line in re.split(r"\\n|;", part)]
        assert all(not line or line.startswith("s_waitcnt") for line in lines), (name, lines)
