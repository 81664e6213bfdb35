"""What the compiler cannot see in the sources of the kernels, looked up in their text."""
import glob
import os
import re

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2302_06646_amd", "csrc")


def _asm_statements(text):
    """Every asm statement, up to the parenthesis that closes it."""
    for m in re.finditer(r"\basm\b(?:\s+volatile)?\s*\(", text):
        depth, at, quoted = 1, m.end(), False
        while depth:
            c = text[at]
            if c == '"' and text[at - 1] != "\\":
                quoted = not quoted
            elif not quoted:
                depth += (c == "(") - (c == ")")
            at += 1
        yield text[m.start():at]


def test_assembly_that_writes_m0_names_it():
    seen = 0
    for path in glob.glob(os.path.join(CSRC, "*.h*")):
        for statement in _asm_statements(open(path).read()):
            if re.search(r"\bs_mov_b32\s+m0\b", statement):
                seen += 1
                assert re.search(r':[^:]*"m0"[^:]*\)$', statement), (os.path.basename(path), statement)
    assert seen
