"""CPU: what a statement of inline assembly writes, its operands and clobbers name."""
import glob
import os
import re

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2408_01331_amd", "csrc")


def statements():
    for path in sorted(glob.glob(os.path.join(CSRC, "*"))):
        text = open(path).read()
        for m in re.finditer(r"\basm\b[^(;]*\(", text):
            depth, end, quoted = 1, m.end(), False
            while depth:
                c = text[end]
                if c == '"':
                    quoted = not quoted
                elif not quoted:
                    depth += (c == "(") - (c == ")")
                end += 1
            yield os.path.basename(path), text[m.end():end - 1]


def test_m0_is_named():
    """m0 is a register like others to the compiler: a statement that writes it says so among its clobbers."""
    seen = 0
    for path, body in statements():
        if re.search(r"\bs_\w+ m0\b", body):
            seen += 1
            assert re.search(r':[^:]*"m0"[^:]*$', body), f"{path}: {body}"
    assert seen
