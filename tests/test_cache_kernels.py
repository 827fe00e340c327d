"""What the kernels of the 8-bit cache count on: that the compiler sees every instruction."""
import glob
import os
import re

CSRC = os.path.join(os.path.dirname(os.path.abspath(__file__)), "..", "paper_2506_14107_amd", "csrc")


def test_no_instruction_hides_from_the_compiler():
    """A vector instruction that reads a matrix instruction's result has to stand 8 or 12 wait states behind it,
    which the compiler sees to for its own instructions and not for those of inline assembly: such statements pin
    values to registers and hold no instruction."""
    held = []
    for path in sorted(glob.glob(os.path.join(CSRC, "*"))):
        with open(path) as f:
            text = re.sub(r"//[^\n]*", "", f.read())
        held += [(os.path.basename(path), m.group(1)) for m in re.finditer(r"\basm\b(?:\s+volatile)?\s*\(\s*((?:\"[^\"]*\"\s*)+)", text)
                 if m.group(1).replace('"', "").strip()]
    assert not held
