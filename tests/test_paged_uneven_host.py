"""What the page kernels rely on, by their sources: alignment of what is read 16 bytes at a time."""
import os
import re

import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2405_14256_b200", "csrc")


def source(name):
    with open(os.path.join(CSRC, name)) as f:
        return re.sub(r"//[^\n]*", "", f.read())


@pytest.mark.parametrize("name", ["zc_paged_decode.cu", "zc_paged_chunk.cu", "zc_paged_own.cu", "zc_paged_weights.cu", "zc_page_evict.cu"])
def test_shared_memory_of_bulk_accesses_is_declared_aligned(name):
    """Copies and accesses of 16 bytes: the dynamic shared memory says so itself, whatever static variables lie before it."""
    found = re.findall(r"extern __shared__ ([^;]*);", source(name))
    assert found
    for what in found:
        align = re.search(r"__align__\((\d+)\)", what)
        assert (align and int(align.group(1)) >= 16) or what.startswith("uint4 "), what
