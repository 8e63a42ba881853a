"""What the compiler reports of the attention kernels of few rows: no scratch memory, whose loads and stores stand between those of keys
and values and wait for them (on the CPU, from the build's own reports)."""
import os
import re

import pytest

from paper_2601_12698_amd import build
from test_host_sanitizers import BUILD


@pytest.mark.parametrize("dtype", [0, 1])
@pytest.mark.parametrize("fmt", [0, 1])
@pytest.mark.parametrize("padded", [64, 128, 256])
def test_few_rows_take_no_scratch_memory(dtype, fmt, padded):
    path = os.path.join(BUILD, f"prefixattn_d{dtype}_f{fmt}_h{padded}.remarks")
    if not os.path.exists(path):
        pytest.skip("the library is not built here")
    with open(path) as f:
        kernels = build.parse_remarks(f.read())
    seen = set()
    for name, r in kernels.items():
        m = re.search(r"attn_kernelILi\dELi\dELi\d+ELi(\d)ELi(\d)E", name)
        prefix, suffix = int(m[1]), int(m[2])
        if suffix in (0, 4):                                   # few rows, four or eight waves
            seen.add((prefix, suffix))
            assert r["scratch"] == 0, (name, r)
    assert {(0, 0), (4, 4), (2, 0)} <= seen
