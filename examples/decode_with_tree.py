"""Speculative decoding with trees of drafted tokens, over a paged cache that is kept to a budget.

The target and its weights are decode_with_cache.py's.  Every step drafts a tree of `nodes` tokens per row (each node's children are the
tokens that last followed its token, the latest first), and then

    csd_cache_extend       room for all nodes
    csd_tree_plan          who sees whom, and at which position
    per layer              projections; csd_rope_append at positions; csd_attention_tree; with a budget csd_attention_mass
    csd_verify_tree        the path through the tree, from the LM head's logits; Ocm.update with what diverged
    csd_cache_commit_path  keep the path, free the rest
    csd_cache_evict        with a budget: rows that are `slack` tokens over it lose those that got the least attention

with nothing read back to the host between.  `--check` (without a budget) recomputes the hidden states of each row's whole sequence
without a cache.

    python examples/decode_with_tree.py --rows 8 --steps 40 --check
    python examples/decode_with_tree.py --rows 8 --steps 40 --budget 96
"""

import argparse
import os
import sys

import torch

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
for place in (ROOT, os.path.join(ROOT, "examples")):
    if place not in sys.path:
        sys.path.insert(0, place)

import paper_2604_13634_b200 as csd  # noqa: E402
from decode_with_cache import Target, check  # noqa: E402


def tree_of(nodes):
    """Parents of a tree of `nodes` nodes: the first child of every node goes on, every second node has another child."""
    parents, order = [-1], [0]
    while len(parents) < nodes:
        at = order.pop(0)
        for _ in range(1 + (at % 2 == 0)):
            if len(parents) < nodes:
                order.append(len(parents))
                parents.append(at)
    return parents


class TreeDecoder:
    def __init__(self, target: Target, rows, nodes, cache, budget=None, sinks=4, recent=32, slack=16):
        dev = target.embedding.device
        self.target, self.rows, self.nodes, self.cache = target, rows, nodes, cache
        self.budget, self.sinks, self.recent, self.slack = budget, sinks, recent, slack
        self.parents_host = parents = tree_of(nodes)
        self.parents = torch.tensor(parents, dtype=torch.int32, device=dev)
        self.rank = [sum(p == parents[t] for p in parents[:t]) for t in range(nodes)]      # which child of its parent a node is
        self.plan, self.buffers = csd.TreePlan(cache, nodes), csd.AttentionBuffers(cache, nodes, target.q_heads, tree=True)
        self.out, self.ocm = csd.TreeBuffers(rows, nodes, device=dev), csd.Ocm(4096, lam=6)
        self.offset = torch.zeros(rows, dtype=torch.int32, device=dev)                      # what positions are ahead of places
        self.mass = None
        if budget is not None:
            self.mass = torch.zeros(rows, cache.max_pages * cache.page_size, device=dev)
            self.evict = csd.EvictBuffers(cache, budget + slack)

    def hidden(self, tokens, n_new):
        """tokens [rows, T], of which the cache has granted the first n_new[row], as nodes that self.plan describes -> [rows, T, H]."""
        t, (rows, T) = self.target, tokens.shape
        x = t.embedding[tokens.long()]
        for layer in range(t.layers):
            qkv = (t.normed(x) @ t.qkv[layer].T).view(rows, T, -1, t.D)
            q, k, v = qkv.split([t.q_heads, t.kv_heads, t.kv_heads], dim=2)
            q = csd.csd_rope_append(q, k, v, self.cache, layer, t.rope, n_new=n_new, positions=self.plan.positions)
            seen = csd.csd_attention_tree(q, self.cache, layer, self.buffers, self.plan.masks, n_new=n_new)
            if self.budget is not None:
                csd.csd_attention_mass(q, self.buffers.lse, self.cache, layer, self.mass, n_new=n_new, masks=self.plan.masks, fresh=layer == 0)
            x = x + seen.view(rows, T, -1) @ t.out[layer].T
        return t.normed(x)

    def step(self, last, followers):
        """One step from the rows' last tokens; followers [V, 2]: the tokens that last followed a token.  Returns the drafted tokens [rows,
        nodes] and their hidden states; self.out says which were accepted."""
        tokens = [last]
        for t in range(1, self.nodes):
            tokens.append(followers[tokens[self.parents_host[t]].long(), min(self.rank[t], 1)])
        tokens = torch.stack(tokens, dim=1)
        csd.csd_cache_extend(self.cache, self.nodes)
        csd.csd_tree_plan(self.parents, self.cache, self.plan, n_new=self.cache.granted, offset=self.offset)
        hidden = self.hidden(tokens, self.cache.granted)
        csd.csd_verify_tree(hidden @ self.target.head.T, tokens, self.parents, self.ocm, 0.3, self.out)
        self.ocm.update(self.out.rej_draft, self.out.rej_target)
        csd.csd_cache_commit_path(self.cache, self.out.accept_len, self.out.path, self.mass)
        if self.budget is not None:
            # rows `slack` over the budget go down to it, the others stay as they are
            keep = torch.where(self.cache.lens >= self.budget + self.slack, self.budget, self.budget + self.slack).to(torch.int32)
            csd.csd_cache_evict(self.cache, self.mass, keep, self.evict, sinks=self.sinks, recent=self.recent)
            self.offset += self.evict.evicted
        return tokens, hidden


def decode(target: Target, rows=8, nodes=12, steps=40, prompt_len=100, page_size=16, budget=None, seed=1):
    """Returns (sequences: one list of tokens per row, the last step's hidden states of the kept nodes, how many, decoder)."""
    dev = target.embedding.device
    gen = torch.Generator(device=dev).manual_seed(seed)
    longest = prompt_len + (steps + 2) * nodes
    cache = csd.PagedCache(rows, rows * -(-longest // page_size), page_size, target.layers, target.kv_heads, target.D, torch.bfloat16, longest)
    d = TreeDecoder(target, rows, nodes, cache, budget)
    # the prompt, all but its last token, as chains of `nodes` tokens: every row its own copy (a budget moves tokens within pages)
    prompt = torch.randint(0, target.V, (prompt_len,), generator=gen, device=dev, dtype=torch.int32)
    for at in range(0, prompt_len - 1, nodes):
        part = prompt[at:min(at + nodes, prompt_len - 1)]
        n_new = torch.full((rows,), part.numel(), dtype=torch.int32, device=dev)
        tokens = torch.zeros(rows, nodes, dtype=torch.int32, device=dev)
        tokens[:, :part.numel()] = part
        csd.csd_cache_extend(cache, nodes, n_new)
        csd.csd_tree_plan(None, cache, d.plan, n_new=cache.granted)
        d.hidden(tokens, cache.granted)
    last = torch.randint(0, target.V, (rows,), generator=gen, device=dev, dtype=torch.int32)
    followers = torch.stack([torch.arange(target.V, device=dev, dtype=torch.int32).roll(-k) for k in (1, 2)], dim=1)
    said = []                                                    # per step: tokens along the path [rows, nodes], how many
    for _ in range(steps):
        tokens, hidden = d.step(last, followers)
        path = d.out.path.long().clamp(min=0)
        said.append((tokens.gather(1, path), d.out.accept_len + 1))
        emitted = tokens.gather(1, path.gather(1, d.out.accept_len[:, None].long()))[:, 0].long()
        last = d.out.next_token.clone()
        followers[emitted] = torch.stack([last, torch.where(followers[emitted, 0] == last, followers[emitted, 1], followers[emitted, 0])], dim=1)
    if cache.stats()["flags"]:
        raise RuntimeError(f"cache flags {cache.stats()['flags']:#x}")
    sequences = [prompt[:-1].tolist() for _ in range(rows)]
    for tokens, kept in said:
        for r, (row, n) in enumerate(zip(tokens.tolist(), kept.tolist())):
            sequences[r] += row[:n]
    hidden = hidden.gather(1, path[..., None].expand(-1, -1, target.H))
    return sequences, hidden, said[-1][1], d


def main():
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--rows", type=int, default=8)
    ap.add_argument("--nodes", type=int, default=12)
    ap.add_argument("--steps", type=int, default=40)
    ap.add_argument("--prompt", type=int, default=100)
    ap.add_argument("--budget", type=int)
    ap.add_argument("--check", action="store_true")
    a = ap.parse_args()
    target = Target()
    sequences, hidden, kept, d = decode(target, a.rows, a.nodes, a.steps, a.prompt, budget=a.budget)
    st, made = d.cache.stats(), sum(len(s) for s in sequences) - a.rows * (a.prompt - 1)
    print(f"{made} tokens in {a.steps} steps of {a.rows} rows; cache: {st['tokens']} tokens in {st['pages']} pages; {int(d.offset.sum())} evicted")
    if a.check and a.budget is None:
        print(f"hidden states against a computation without cache: rms difference {check(target, sequences, hidden, kept, d.cache):.4f}")
    d.ocm.close()


if __name__ == "__main__":
    main()
