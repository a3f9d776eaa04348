"""The norm's kernels keep a row and the weights in registers: those with one and with two octets a thread, which is all rows of up to 16384 values in either direction
(two forward from 512 columns on already, where there are many rows), must not spill.  Compiles for gfx950 (no GPU needed) and reads the compiler's remarks."""
import os
import re

import pytest

from test_group_resources import kernels, number
from test_kernel_resources import HIPCC, resource_remarks


@pytest.mark.skipif(not os.path.exists(HIPCC), reason="hipcc not installed")
def test_norm_of_rows_up_to_16384_values_does_not_spill():
    text = resource_remarks("skim_norm.hip").stdout
    octets = []
    for name in ("rms_norm_kernel", "rms_norm_back_kernel"):
        for m in kernels(text, name):
            r = int(re.search(name + r"I[tf]Li(\d)ELb[01]E", m.group(0)).group(1))
            octets.append(r)
            if r <= 2:
                assert number(m.group(0), "ScratchSize [bytes/lane]") == 0, m.group(0)[:120]
    assert sorted(octets) == [1] * 8 + [2] * 8 + [4] * 8
