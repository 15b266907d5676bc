"""What the compiler has to be told about instructions written by hand."""
import glob
import os
import re

from paper_2412_03213_amd.build import CSRC


def asm_blocks():
    for path in sorted(glob.glob(os.path.join(CSRC, "*.h*"))):
        with open(path) as f:
            text = f.read()
        for at in re.finditer(r"\basm\s+volatile\s*\(", text):
            depth, i, quoted = 1, at.end(), False
            while depth:
                c = text[i]
                if c == '"' and text[i - 1] != "\\":
                    quoted = not quoted
                depth += 0 if quoted else (c == "(") - (c == ")")
                i += 1
            yield os.path.basename(path), text[at.end():i - 1]


def test_loads_to_lds_get_their_address_through_the_compiler():
    """The address is an operand in m0: a block that writes the register itself changes it behind the compiler's back."""
    loads = 0
    for path, block in asm_blocks():
        code, operands = (re.split(r'"\s*:', block, maxsplit=1) + [""])[:2]
        assert not re.search(r"\bm0\b", code), (path, block)
        if "_load_lds_" in code:
            loads += 1
            assert '"{m0}"(' in operands and '"memory"' in operands, (path, block)
    assert loads
