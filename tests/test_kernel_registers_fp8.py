"""The tiles of the products in 8 bits keep their sums in registers, none of them in scratch memory."""
import os
import re


def test_no_tile_spills_its_registers():
    from paper_2604_03298_amd import enec
    if not os.path.exists(enec.LIB_PATH):
        from paper_2604_03298_amd import build
        build.build()
    with open(enec.LIB_PATH, "rb") as f:
        data = f.read()
    # the kernels' metadata, written by the compiler: a map per kernel, keys in alphabetical order
    found = re.findall(rb"\.private_segment_fixed_size([\x00-\x7f]|\xcc.|\xcd..).{0,500}?\.symbol.{1,3}?(_ZN4enec6lowbit15fp8_tile_kernel\w+)\.kd.{0,200}?\.vgpr_spill_count(\xcc?.)", data, re.S)
    assert len(found) == 11                                # seven tiles, four of them for exact products too
    assert {name.decode(): (scratch, spilled) for scratch, name, spilled in found if scratch != b"\0" or spilled != b"\0"} == {}
