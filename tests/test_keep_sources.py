"""A rule of the sources, no GPU: lengths and grants are words in the caller's memory that anyone can write; the kernels that move tokens bound
them to what a row can hold before they become addresses."""

import re

import pytest

from test_cluster_sources import bodies, code_of

RAW = {name: r"v\.(?:lens|granted)\[|v\.lens\s*\+" for name in ("path_kernel", "evict_pick_kernel", "evict_move_kernel", "evict_finish_kernel")}


@pytest.mark.parametrize("kernel", sorted(RAW))
def test_lengths_and_grants_are_bounded(kernel):
    (body,) = [b for is_kernel, name, b in bodies(code_of("csd_keep.cuh")) if is_kernel and name == kernel]
    assert not re.search(RAW[kernel], body)
    for read in re.finditer(r"[^;]*v\.granted\s*\+[^;]*;", body):
        assert re.search(r"min\(max\(.*, 0\), len\)", read.group())


def test_counts_that_are_read_four_at_a_time_are_aligned():
    """Shared memory follows the alignment of what is declared: words alone would promise four bytes."""
    code = code_of("csd_keep.cuh")
    (from_, to) = re.search(r"struct PickShared \{(.*?)\};", code, re.S).span(1)
    read = re.search(r"const unsigned int \*const count = blocks == 1 \? s\.(\w+) : s\.(\w+);.*?reinterpret_cast<const uint4 \*>\(count", code, re.S)
    for name in read.groups():
        assert re.search(rf"__align__\(16\) unsigned int {name}\[kBins\];", code[from_:to])
