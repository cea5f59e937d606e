"""Host side of the decode-pass operators: what is refused before anything is launched, and rules of the sources.  No GPU."""

import os
import re
from ctypes import byref

import pytest
import torch

from paper_2604_13634_b200 import binding, build, decode

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


INVALID_ARG, UNSUPPORTED = 1, 4
SOMEWHERE = 1 << 20                                                  # an aligned address that nothing may follow


@pytest.mark.parametrize("B,S", [(1, 2 ** 31 - 1), (2 ** 31 - 1, 1), (1, 2 ** 31 - 256)])
def test_token_counts_whose_last_block_passes_31_bits_are_refused(B, S):
    """Blocks of several tokens count up to a block's tokens beyond the last: 85 to a block (three units of one head) make
    25264515 blocks of 2^31 - 1 tokens, whose last index is 2^31 + 126."""
    assert -(-(2 ** 31 - 1) // 85) * 85 - 1 > 2 ** 31 - 1
    plan = decode.RopeStruct(SOMEWHERE, 2, 0, 1.0)
    rc = decode._lib().csd_rope(SOMEWHERE, SOMEWHERE, binding.CSD_F32, B, S, 1, 6, 6 * S, 6, 6, 6 * S, 6, 6, SOMEWHERE, S, 1, byref(plan), 0, None)
    assert rc == UNSUPPORTED


class _Stream:
    def __init__(self, device_index):
        self.device_index, self.cuda_stream = device_index, 5


def test_addresses_of_another_device_are_refused(monkeypatch):
    monkeypatch.setattr(decode, "_current_device", lambda: 0)
    assert decode._stream_ptr(_Stream(0), 0) == 5
    for stream, device in ((_Stream(1), 0), (_Stream(1), 1), (None, 1)):
        with pytest.raises(binding.CsdError, match="device"):
            decode._stream_ptr(stream, device)
    x, pos, plan = torch.zeros(1, 3, 2, 64), torch.zeros(1, 3, dtype=torch.int32), decode.RopePlan(64, device="cpu")
    with pytest.raises(binding.CsdError, match="device"):
        decode.csd_rope(x, pos, plan)
    plan._device = 0
    with pytest.raises(binding.CsdError, match="device"):
        decode.csd_rope(x, pos, plan)


def test_more_layers_than_the_page_copies_can_have_are_refused_before_the_bookkeeping():
    """The copies' grid has a row for every layer's keys and values, at most 65535 of them."""
    c = decode.CacheStruct(SOMEWHERE, SOMEWHERE, binding.CSD_BF16, 32768, 4, 8, 1, 8, 4 * 64, 64, 64, 8, 1, 4, SOMEWHERE, SOMEWHERE)
    for call in (lambda L: L.csd_cache_extend(byref(c), 1, None, None), lambda L: L.csd_cache_compact(byref(c), None), lambda L: L.csd_cache_rebuild(byref(c), None)):
        assert call(decode._lib()) == UNSUPPORTED


def test_half_a_pool_is_refused():
    half = torch.zeros(1, 4, 1, 16, 64, dtype=torch.bfloat16)
    for kw in (dict(k=half), dict(v=half)):
        with pytest.raises(binding.CsdError, match="both"):
            decode.PagedCache(1, 4, 16, 1, 1, 64, torch.bfloat16, 64, **kw)


@pytest.mark.parametrize("H", [2 ** 31 - 1, 2 ** 31 - 3])
def test_head_counts_that_pass_31_bits_in_groups_are_refused(H):
    """Heads are taken four at a time, and the count is rounded up: three more than 2^31 - 1 - 3 wrap."""
    plan = decode.RopeStruct(SOMEWHERE, 2, 0, 1.0)
    L = decode._lib()
    assert L.csd_rope(SOMEWHERE, SOMEWHERE, binding.CSD_F32, 1, 1, H, 6, 6 * H, 6 * H, 6, 6 * H, 6 * H, 6, SOMEWHERE, 1, 1, byref(plan), 0, None) == UNSUPPORTED
    c = decode.CacheStruct(SOMEWHERE, SOMEWHERE, binding.CSD_BF16, 1, 4, 8, 1, 8, 4 * 64, 64, 64, 8, 1, 4, SOMEWHERE, SOMEWHERE)
    three = (8, 8, 8)
    assert L.csd_rope_append(SOMEWHERE, *three, H, SOMEWHERE, *three, SOMEWHERE, *three, SOMEWHERE, 1, byref(c), 0, None, None, None) == UNSUPPORTED


def test_blocks_that_give_up_stay_until_their_copies_have_landed():
    """Each kernel with bounded waits sees at its end whether one ran out, and lingers before its memory goes to another block."""
    with open(os.path.join(CSRC, "csd_attention.cuh")) as f:
        kernels = re.split(r"__global__", re.sub(r"//[^\n]*", "", f.read()))[1:]
    waiting = [k for k in kernels if "mbar_wait(" in k]
    assert len(waiting) == 2
    for k in waiting:
        end = k[k.rindex("if (*give_up)"):]
        assert "CSD_CACHE_INTERNAL" in end and "ptx::linger();" in end
        assert "tmem_alloc" not in k or end.index("ptx::linger();") < end.index("tmem_dealloc")
