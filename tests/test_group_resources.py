"""The products with 4-bit weights on tiles keep 128 accumulators, two operand sets and two blocks of codes in 256 registers: a spill inside their
loops waits behind every copy in flight.  Compiles for gfx950 (no GPU needed) and reads the compiler's resource remarks."""
import os
import re

import pytest

from test_kernel_resources import HIPCC, resource_remarks


def kernels(text, name):
    return list(re.finditer(r"Function Name: \S*\d" + name + r"\S*.*?LDS Size", text, re.S))


def number(text, what):
    return int(re.search(re.escape(what) + r": (\d+)", text).group(1))


@pytest.mark.skipif(not os.path.exists(HIPCC), reason="hipcc not installed")
def test_products_on_tiles_do_not_spill():
    r = resource_remarks("skim_group_mm.hip")
    found = kernels(r.stdout, "group_wide_kernel")
    assert len(found) == 10          # three forward ones and the gradient's with one and two groups of wavefronts, that also with 64 tokens a tile
    for m in found:
        assert number(m.group(0), "ScratchSize [bytes/lane]") == 0, m.group(0)[:120]
        assert number(m.group(0), "Occupancy [waves/SIMD]") == 2
    few = kernels(r.stdout, "group_few_kernel")
    assert len(few) == 2 * 2 * 3 * 3 * 2
    for m in few:
        assert number(m.group(0), "ScratchSize [bytes/lane]") == 0, m.group(0)[:120]


@pytest.mark.skipif(not os.path.exists(HIPCC), reason="hipcc not installed")
def test_quantiser_and_norm_keep_their_rows_in_registers():
    for m in kernels(resource_remarks("skim_group.hip").stdout, "group_quantize_kernel"):
        assert number(m.group(0), "ScratchSize [bytes/lane]") == 0
    r = resource_remarks("skim_norm.hip")
    found = kernels(r.stdout, "rms_norm_kernel") + kernels(r.stdout, "rms_norm_back_kernel")
    assert len(found) == 24
    for m in found:                  # up to 8192 columns (one octet a thread)
        if "Li1ELb" in m.group(0)[:200]:
            assert number(m.group(0), "ScratchSize [bytes/lane]") == 0, m.group(0)[:120]
