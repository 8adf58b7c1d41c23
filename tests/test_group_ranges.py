"""The ranges that the kernels on group-scaled rows may read, from their sources: zero points are bytes at any address, and
a descriptor filled up to whole words from an address that is not on 4 bytes would admit up to three bytes behind the
array, which may lie in a page that is not there."""
import glob
import os
import re

import paper_1809_10572_amd as samd

CSRC = os.path.join(os.path.dirname(samd.LIB_PATH), "csrc")


def test_zero_points_are_read_by_exact_ranges():
    found = 0
    for path in glob.glob(os.path.join(CSRC, "group_*.h*")):
        with open(path) as f:
            text = f.read()
        for maker in re.findall(r"= (\w+)\([^;]*?\.zero \+", text):
            found += 1
            assert maker == "byte_buffer_of", path
    assert found == 4   # the vector, narrow and tiled products and the input gradient
    with open(os.path.join(CSRC, "group_device.hpp")) as f:
        body = re.search(r"byte_buffer_of\(const uint8_t \*p.*?\n}\n", f.read(), re.S)[0]
    assert "+ 3" not in body and "min(bytes," in body
