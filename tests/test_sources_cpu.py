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


def test_blocks_that_write_m0_say_so():
    found = 0
    for path, block in asm_blocks():
        code = block.split('"::')[0]
        if re.search(r"\bm0\b", code):
            found += 1
            clobbers = block.rsplit(":", 1)[1]
            assert '"m0"' in clobbers and '"memory"' in clobbers, (path, block)
    assert found
