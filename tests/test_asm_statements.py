"""asm statements of the device code.  The compiler does not look into them: a vector instruction in one may read a matrix
instruction's result before it is there."""
from __future__ import annotations

import glob
import os
import re

import pytest

from paper_2412_19829_amd import build


@pytest.mark.parametrize("path", sorted(glob.glob(os.path.join(build.CSRC, "*.h*"))), ids=os.path.basename)
def test_asm_statements_hold_no_vector_arithmetic(path):
    with open(path) as f:
        text = re.sub(r"//[^\n]*", "", f.read())
    for statement in re.findall(r"\basm\b(?:\s+volatile)?\s*\((.*?)\);", text, re.S):
        strings = " ".join(re.findall(r'"((?:[^"\\]|\\.)*)"', statement))
        assert not re.search(r"\bv_[a-z]", strings), statement
