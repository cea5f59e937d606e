"""Host side of the decode-pass operators: what is refused before anything is launched, and rules of the sources.  No GPU."""

import os
import re

import pytest

from paper_2604_13634_b200 import build

CSRC = os.path.join(os.path.dirname(os.path.abspath(build.__file__)), "csrc")


@pytest.fixture(scope="module", autouse=True)
def _built():
    build.build()


@pytest.mark.parametrize("name", ["csd_attention.cuh", "csd_rope.cuh", "csd_pages.cuh"])
def test_only_constants_are_loaded_as_read_only(name):
    """Kernels that start beside their predecessor must not load what it writes as data that nobody writes."""
    with open(os.path.join(CSRC, name)) as f:
        code = re.sub(r"//[^\n]*", "", f.read())
    loads = re.findall(r"__ldg\(([^)]*)\)|(ld_stream16|\.nc\b)", code)
    assert [a for a, _ in loads] == (["t.steps + pair"] if name == "csd_rope.cuh" else [])
