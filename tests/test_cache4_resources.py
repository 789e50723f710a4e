"""Registers and shared memory of the kernels of rotated appends and caches of 4
bits (code object metadata, no GPU)."""
import os
import re

import pytest

from paper_2608_02134_amd import binding as B

from .code_objects import kernels


@pytest.fixture(scope="module")
def built():
    if not os.path.exists(B.LIB_PATH):
        pytest.fail("libgmc.so is not built; run __graft_entry__.build()")
    return kernels(B.LIB_PATH)


def _find(built, pattern, count):
    found = {n: k for n, k in built.items() if re.search(pattern, n)}
    assert len(found) == count, sorted(found)
    return found


def test_appends_and_decode_spill_nothing(built):
    """Two types, into pages (two kinds of pairs) and 4 bits (none too), few and
    many tokens; every head dimension of decode, and the short ones in one block."""
    for found in (_find(built, r"rotary_append(_few)?_kernel", 2 * 2 * (2 + 3)), _find(built, r"cache4_read_kernel", 2),
                  _find(built, r"decode4_kernel", 2 * (8 + 4))):
        assert {n: k[".private_segment_fixed_size"] for n, k in found.items() if k[".private_segment_fixed_size"]} == {}


def test_prefill_spills_in_fp32_from_224_on_alone(built):
    found = _find(built, r"prefill4_kernel", 2 * 8)
    spilt = {n: k[".private_segment_fixed_size"] for n, k in found.items() if k[".private_segment_fixed_size"]}
    assert all(re.search(r"prefill4_kernelIfLi(224|256)", n) and size <= 256 for n, size in spilt.items()), spilt


def test_blocks_find_the_room_that_the_splits_count_on(built):
    """Three decode blocks to a CU with heads of up to 128 in bf16, two of prefill."""
    for n, k in _find(built, r"decode4_kernelItLi(32|64|96|128)ELi4E", 4).items():
        assert k[".vgpr_count"] <= 168 and 3 * k[".group_segment_fixed_size"] <= 160 * 1024, n
    for n, k in _find(built, r"prefill4_kernelItLi(32|64|96|128)E", 4).items():
        assert k[".vgpr_count"] <= 256 and 2 * k[".group_segment_fixed_size"] <= 160 * 1024, n
