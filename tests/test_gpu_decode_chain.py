"""The decode-pass operators one behind the other on a stream: every call reads what the call before has just written."""

import pytest
import torch

from paper_2604_13634_b200 import (AttentionBuffers, Ocm, PagedCache, RopePlan, StepBuffers, csd_attention, csd_cache_commit, csd_cache_compact,
                                   csd_cache_extend, csd_cache_fork, csd_cache_truncate, csd_rope_append, csd_step)

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("q_heads", [4, 16])                        # 12 query rows to a key head, and 48
def test_what_a_call_reads_was_written_just_before(q_heads):
    """Lengths, tables, grants, parents and accepted counts come from the call before, without a wait of the host: the same bits as
    with one after every call."""
    rows, K, T, D, steps = 32, 5, 6, 64, 120
    gen = torch.Generator(device="cuda").manual_seed(7)
    rand = lambda *shape: torch.randn(shape, generator=gen, device="cuda").to(torch.bfloat16)  # noqa: E731
    logits = torch.randn(4, rows, K + 1, rows, generator=gen, device="cuda").to(torch.bfloat16)   # as many tokens as rows: next_token names a row
    draft = logits.float().argmax(-1)[:, :, :K].int().contiguous()
    draft[torch.rand(draft.shape, generator=gen, device="cuda") < 0.3] = 1
    qkv = rand(4, rows, T, q_heads + 4, D)
    plan = RopePlan(D)

    def go(waits):
        cache = PagedCache(rows, 40 * rows, 8, 1, 2, D, torch.bfloat16, 300)
        buf, step, ocm = AttentionBuffers(cache, T, q_heads), StepBuffers(rows, K, rows, torch.bfloat16), Ocm(4096, lam=3)
        wait = torch.cuda.synchronize if waits else lambda: None
        out, seen = torch.zeros(rows, T, q_heads, D, device="cuda"), torch.zeros(rows, device="cuda", dtype=torch.int64)
        for s in range(steps):
            q, k, v = qkv[s % 4].split([q_heads, 2, 2], dim=2)
            csd_cache_extend(cache, T)
            wait()
            q = csd_rope_append(q, k, v, cache, 0, plan, n_new=cache.granted)
            wait()
            csd_attention(q, cache, 0, buf, n_new=cache.granted)
            wait()
            csd_step(logits[s % 4], draft[s % 4], ocm, 0.3, step)
            wait()
            csd_cache_commit(cache, step.accept_len)
            wait()
            csd_cache_fork(cache, step.next_token)                   # every row continues some row, many of them the same
            wait()
            csd_cache_extend(cache, 1, n_new=step.accept_len)
            wait()
            csd_cache_commit(cache, cache.granted)                   # all of them stay
            wait()
            if s % 3 == 2:
                csd_cache_compact(cache)
                wait()
            csd_cache_truncate(cache, cache.lens if s % 10 else step.accept_len)
            wait()
            out += buf.out.float()
            seen += cache.lens * (s + 1) + cache.table.sum(1)
        torch.cuda.synchronize()
        assert cache.stats()["flags"] == 0
        ocm.close()
        return out, seen, cache.meta.clone(), cache.k.clone(), cache.v.clone()

    want = go(True)
    assert torch.isfinite(want[0]).all() and len(set(want[1].tolist())) > 1
    for _ in range(5):
        for a, b in zip(go(False), want):
            assert torch.equal(a, b)
