"""Edges of the decode-pass operators: arguments that have to be refused, and places where a result could go wrong silently."""

import pytest
import torch

from paper_2604_13634_b200 import AttentionBuffers, CsdError, PagedCache, RopePlan, csd_attention, csd_rope, csd_rope_append, decode

pytestmark = pytest.mark.gpu


def test_a_plan_in_host_memory_or_another_current_device_is_refused(monkeypatch):
    x, pos = torch.randn(1, 3, 2, 64, device="cuda"), torch.zeros(1, 3, dtype=torch.int32, device="cuda")
    with pytest.raises(CsdError, match="device"):
        csd_rope(x, pos, RopePlan(64, device="cpu"))
    cache = PagedCache(1, 4, 16, 1, 2, 64, torch.bfloat16, 64)
    q = torch.zeros(1, 1, 2, 64, dtype=torch.bfloat16, device="cuda")
    with pytest.raises(CsdError, match="device"):
        csd_rope_append(q, q, q, cache, 0, RopePlan(64, device="cpu"))
    buf, plan = AttentionBuffers(cache, 1, 2), RopePlan(64)
    monkeypatch.setattr(decode, "_current_device", lambda: 1)
    for call in (lambda: csd_rope(x, pos, plan), lambda: csd_rope_append(q, q, q, cache, 0, None), lambda: csd_attention(q, cache, 0, buf),
                 lambda: decode.csd_cache_extend(cache, 1), lambda: decode.csd_cache_compact(cache)):
        with pytest.raises(CsdError, match="device"):
            call()
