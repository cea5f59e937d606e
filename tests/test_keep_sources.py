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
