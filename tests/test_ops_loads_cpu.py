"""No-GPU check of the operators' sources: no read-only loads (which may be moved in front of the wait for the kernel before)."""
import os
import re

import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2605_08134_b200", "csrc")
SOURCES = ["rope.cu", "linear.cu", "linear.h", "linear_tc.cu", "gemm_f32.cu", "attn_packed.h", "attn_packed.cu", "attn_packed_tc.cuh",
           "attn_packed_tc.cu", "attn_packed_tiles.cu"]


@pytest.mark.parametrize("name", SOURCES)
def test_no_read_only_loads_of_operands(name):
    with open(os.path.join(CSRC, name)) as f:
        code = re.sub(r"//[^\n]*", "", f.read())
    assert not re.search(r"\b__ldg\s*\(|ld\.global\.nc|const\s[^,;(){}]*\*\s*__restrict__", code)
