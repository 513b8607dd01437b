"""What the HIP sources hold, read as text on the host."""
import os
import re

import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2012_03837_amd", "csrc")
FILES = sorted(f for f in os.listdir(CSRC) if f.endswith((".hip", ".h")))


@pytest.mark.parametrize("name", FILES)
def test_inline_asm_computes_nothing(name):
    """Between a matrix instruction and a vector instruction that reads its result there are wait states, which the compiler puts in for its own instructions
    only: a vector instruction in inline asm may read registers that are not written yet."""
    with open(os.path.join(CSRC, name)) as f:
        text = re.sub(r"//[^\n]*", "", f.read())
    for code in re.findall(r'\basm\s*(?:volatile)?\s*\(\s*((?:"[^"]*"\s*)+)', text):
        assert not re.search(r"\bv_", code), code
