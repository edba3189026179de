"""What the kernels' inline assembly writes is declared: the compiler may keep values of its
own in m0.  Reads the sources; no GPU."""
import glob
import os
import re

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_1903_06681_amd", "csrc")


def statements():
    """(file, text) of every asm statement, up to its closing parenthesis."""
    for path in sorted(glob.glob(os.path.join(CSRC, "*"))):
        text = open(path).read()
        for m in re.finditer(r"\basm\b(?:\s+volatile)?\s*\(", text):
            depth, i, quoted = 1, m.end(), False
            while depth:
                c = text[i]
                if c == '"' and text[i - 1] != "\\":
                    quoted = not quoted
                elif not quoted:
                    depth += (c == "(") - (c == ")")
                i += 1
            yield os.path.basename(path), text[m.start():i]


def test_assembly_that_writes_m0_says_so():
    found = [(f, s) for f, s in statements() if re.search(r"\bs_mov_b32 m0\b", s)]
    assert found
    for f, s in found:
        assert re.search(r':[^:]*"m0"[^:]*\)$', s), f"{f}: {s}"
