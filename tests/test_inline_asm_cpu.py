"""Inline assembly of the kernels' sources: no statement sets a register that the
compiler is not told of.  m0 cannot be named as overwritten, so it is an operand."""
import glob
import os
import re

from paper_1904_05347_amd import build


def test_m0_is_an_operand():
    seen = 0
    for path in sorted(glob.glob(os.path.join(build.CSRC, "*.h*"))):
        with open(path) as fh:
            text = fh.read()
        for statement in re.findall(r"\basm\s*(?:volatile)?\s*\((.*?)\);", text, re.S):
            code = statement.split(":")[0]
            assert not re.search(r"\bm0\b", code), (os.path.basename(path), statement)
            if re.search(r"\blds\b", code):   # a copy from memory to LDS reads it
                assert '"{m0}"' in statement, (os.path.basename(path), statement)
                seen += 1
    assert seen >= 1
