"""The tree pass, its cache and the budget as they are used together: the example, and the calls one behind the other on a stream."""

import os
import sys

import pytest
import torch

from paper_2604_13634_b200 import (AttentionBuffers, EvictBuffers, Ocm, PagedCache, RopePlan, TreeBuffers, TreePlan, csd_attention_mass,
                                   csd_attention_tree, csd_cache_commit_path, csd_cache_evict, csd_cache_extend, csd_rope_append, csd_tree_plan,
                                   csd_verify_tree)

pytestmark = pytest.mark.gpu

sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))


@pytest.mark.parametrize("rows,nodes,steps,prompt", [(1, 1, 5, 3), (8, 12, 20, 100), (3, 40, 10, 57), (2, 64, 4, 130)])
def test_decoding_with_trees_equals_decoding_without_a_cache(rows, nodes, steps, prompt):
    """The tolerance of the chain's example: bf16 states of root mean square 1 after two layers, twelve roundings of 2^-9 on either side."""
    import decode_with_tree as example
    target = example.Target()
    sequences, hidden, kept, d = example.decode(target, rows, nodes, steps, prompt)
    assert example.check(target, sequences, hidden, kept, d.cache) < 0.02
    assert all(len(s) >= prompt - 1 + steps for s in sequences)
    d.ocm.close()


def test_decoding_within_a_budget():
    import decode_with_tree as example
    target = example.Target()
    sequences, hidden, kept, d = example.decode(target, 4, 12, 30, 100, budget=64)
    lens = d.cache.lens.tolist()
    assert all(64 <= n < 64 + 16 for n in lens) and torch.isfinite(hidden.float()).all()
    assert [n + int(o) for n, o in zip(lens, d.offset)] == [len(s) for s in sequences]
    pages = d.cache.stats()["pages"]
    assert pages == sum(-(-n // 16) for n in lens)
    d.ocm.close()


@pytest.mark.parametrize("q_heads", [2, 16])                        # 9 query rows to a key head, and 72
def test_what_a_call_reads_was_written_just_before(q_heads):
    """Nothing waits for the host between the calls: the same bits as with a wait after every call."""
    rows, T, D, V, steps = 24, 9, 64, 3001, 60
    gen = torch.Generator(device="cuda").manual_seed(7)
    qkv = torch.randn(4, rows, T, q_heads + 4, D, generator=gen, device="cuda").to(torch.bfloat16)
    logits = torch.randn(4, rows, T, V, generator=gen, device="cuda").to(torch.bfloat16)
    parents = torch.tensor([[-1] + [int(torch.randint(max(0, t - 3), t, (1,), generator=gen, device="cuda")) for t in range(1, T)] for _ in range(rows)],
                           dtype=torch.int32, device="cuda")
    tokens = torch.randint(0, V, (4, rows, T), generator=gen, device="cuda", dtype=torch.int32)
    for s in range(4):                                                # most nodes' tokens are what the target says after their parents
        said = logits[s].float().argmax(-1).gather(1, parents.clamp(min=0).long()).int()
        tokens[s] = torch.where(torch.rand(rows, T, generator=gen, device="cuda") < 0.7, said, tokens[s])
    rope = RopePlan(D)

    def go(waits):
        cache = PagedCache(rows, 16 * rows, 16, 2, 2, D, torch.bfloat16, 200)
        plan, buf, out, ocm = TreePlan(cache, T), AttentionBuffers(cache, T, q_heads, tree=True), TreeBuffers(rows, T), Ocm(4096, lam=2)
        mass, evict = torch.zeros(rows, cache.max_pages * 16, device="cuda"), EvictBuffers(cache, 100)
        offset = torch.zeros(rows, dtype=torch.int32, device="cuda")
        wait = torch.cuda.synchronize if waits else lambda: None
        total, seen = torch.zeros(rows, T, q_heads, D, device="cuda"), torch.zeros(rows, device="cuda", dtype=torch.int64)
        for s in range(steps):
            q, k, v = qkv[s % 4].split([q_heads, 2, 2], dim=2)
            csd_cache_extend(cache, T)
            wait()
            csd_tree_plan(parents, cache, plan, n_new=cache.granted, offset=offset)
            wait()
            for layer in range(2):
                turned = csd_rope_append(q, k, v, cache, layer, rope, n_new=cache.granted, positions=plan.positions)
                wait()
                csd_attention_tree(turned, cache, layer, buf, plan.masks, n_new=cache.granted)
                wait()
                csd_attention_mass(turned, buf.lse, cache, layer, mass, n_new=cache.granted, masks=plan.masks, fresh=layer == 0)
                wait()
                total += buf.out.float()
            csd_verify_tree(logits[s % 4], tokens[s % 4], parents, ocm, 0.3, out, n_nodes=cache.granted)
            wait()
            ocm.update(out.rej_draft, out.rej_target)
            wait()
            csd_cache_commit_path(cache, out.accept_len, out.path, mass)
            wait()
            csd_cache_evict(cache, mass, 100 if s % 5 else 80, evict, sinks=4, recent=20)
            wait()
            offset += evict.evicted
            seen += cache.lens * (s + 1) + cache.table.sum(1) + out.path.sum(1) + evict.kept.sum(1)
        torch.cuda.synchronize()
        assert cache.stats()["flags"] == 0 and ocm.stats()["flags"] == 0
        assert int(offset.sum()) > 0 and ocm.stats()["matches"] > 0
        ocm.close()
        return total, seen, mass.clone(), cache.meta.clone(), cache.k.clone(), cache.v.clone()

    want = go(True)
    assert torch.isfinite(want[0]).all() and len(set(want[1].tolist())) > 1
    for _ in range(4):
        for a, b in zip(go(False), want):
            assert torch.equal(a, b)


class Step:
    """One step of the tree pass over a cache of its own: everything a call needs, so that two of them share nothing."""

    def __init__(self, seed, rows=6, T=12, heads=24, D=128, V=2000):
        gen = torch.Generator(device="cuda").manual_seed(seed)
        self.cache, self.layers = PagedCache(rows, 20 * rows, 16, 2, 2, D, torch.bfloat16, 300), 2
        self.qkv = torch.randn(rows, T, heads + 4, D, generator=gen, device="cuda").to(torch.bfloat16)
        self.heads, self.rope = heads, RopePlan(D)
        self.logits = torch.randn(rows, T, V, generator=gen, device="cuda").to(torch.bfloat16)
        self.parents = torch.tensor([-1, 0, 0, 1, 1, 2, 3, 3, 4, 6, 8, 9][:T], dtype=torch.int32, device="cuda")
        self.tokens = self.logits.float().argmax(-1)[:, self.parents.clamp(min=0).long()].int().contiguous()      # every child matches
        self.plan, self.buf, self.out = TreePlan(self.cache, T), AttentionBuffers(self.cache, T, heads, tree=True), TreeBuffers(rows, T)
        self.ocm, self.evict = Ocm(256, lam=2), EvictBuffers(self.cache, 70)
        self.mass = torch.zeros(rows, self.cache.max_pages * 16, device="cuda")
        self.offset = torch.zeros(rows, dtype=torch.int32, device="cuda")
        torch.cuda.synchronize()

    def __call__(self):
        c = self.cache
        q, k, v = self.qkv.split([self.heads, 2, 2], dim=2)
        csd_cache_extend(c, self.plan.T)
        csd_tree_plan(self.parents, c, self.plan, n_new=c.granted, offset=self.offset)
        for layer in range(self.layers):
            turned = csd_rope_append(q, k, v, c, layer, self.rope, n_new=c.granted, positions=self.plan.positions)
            csd_attention_tree(turned, c, layer, self.buf, self.plan.masks, n_new=c.granted)
            csd_attention_mass(turned, self.buf.lse, c, layer, self.mass, n_new=c.granted, masks=self.plan.masks, fresh=layer == 0)
        csd_verify_tree(self.logits, self.tokens, self.parents, self.ocm, 0.3, self.out, n_nodes=c.granted)
        csd_cache_commit_path(c, self.out.accept_len, self.out.path, self.mass)
        csd_cache_evict(c, self.mass, 70, self.evict, sinks=2, recent=16)
        self.offset += self.evict.evicted

    def state(self):
        torch.cuda.synchronize()
        assert self.cache.stats()["flags"] == 0
        return [x.clone() for x in (self.cache.meta, self.cache.k, self.cache.v, self.mass, self.offset, self.buf.out, self.buf.lse, self.out.path)]


def test_a_step_captured_and_replayed():
    eager, played = Step(1), Step(1)
    for _ in range(2):                                               # what is asked of the device once is asked outside the capture
        eager()
        played()
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        played()
    for _ in range(30):
        eager()
        graph.replay()
    for a, b in zip(eager.state(), played.state()):
        assert torch.equal(a, b)
    assert int(eager.offset.sum()) > 0 and int(eager.cache.lens.max()) <= 70
    eager.ocm.close()
    played.ocm.close()


def test_two_passes_at_once():
    """Two caches, each on a stream of its own, at the same time: what each gives alone.  (36, 48, 144 and 864 query rows to a key head: every kernel.)"""
    for heads in ((6, 8), (24, 144)):
        alone = []
        for i, h in enumerate(heads):
            s = Step(3 + i, heads=h)
            for _ in range(25):
                s()
            alone.append(s.state())
            s.ocm.close()
        both, streams = [Step(3 + i, heads=h) for i, h in enumerate(heads)], [torch.cuda.Stream() for _ in heads]
        for _ in range(25):
            for s, stream in zip(both, streams):
                with torch.cuda.stream(stream):
                    s()
        torch.cuda.synchronize()
        for s, want in zip(both, alone):
            for a, b in zip(s.state(), want):
                assert torch.equal(a, b)
            s.ocm.close()
