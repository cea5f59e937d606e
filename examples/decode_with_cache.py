"""Speculative decoding of several rows with a paged cache: the target pass around the verification step.

A small random target (embedding, two attention layers, LM head) decodes `rows` continuations of one prompt.  The prompt goes into
the cache once, in pieces, and every row shares its pages (csd_cache_fork).  Each step then

    csd_cache_extend     room for the last token and the K drafted ones
    per layer            projections; csd_rope_append; csd_attention; output projection
    csd_step_lmhead      verification straight from the hidden states
    csd_cache_commit     keep the last token and the accepted drafts, free the rest

with nothing read back to the host between.  The tokens that a pass stores and attends to are those that the extension granted
(cache.granted, on the device): one that finds no room grants none and leaves a flag, and the pass then touches no page.  The drafts
come from a table of the last successor of every token, which stands in for a draft model.  `--check` recomputes the hidden states of a row's whole sequence without a cache.

    python examples/decode_with_cache.py --rows 8 --steps 40 --check
"""

import argparse
import os
import sys

import torch

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
if ROOT not in sys.path:
    sys.path.insert(0, ROOT)

import paper_2604_13634_b200 as csd  # noqa: E402


class Target:
    """Weights of a small decoder: H hidden, q_heads query heads on kv_heads key heads of D, V tokens."""

    def __init__(self, H=512, layers=2, q_heads=8, kv_heads=2, D=64, V=2048, seed=0, device="cuda"):
        gen = torch.Generator(device=device).manual_seed(seed)
        make = lambda *shape: (torch.randn(shape, generator=gen, device=device) * shape[-1] ** -0.5).to(torch.bfloat16)  # noqa: E731
        self.H, self.layers, self.q_heads, self.kv_heads, self.D, self.V = H, layers, q_heads, kv_heads, D, V
        self.embedding = torch.randn((V, H), generator=gen, device=device).to(torch.bfloat16)
        self.qkv = [make((q_heads + 2 * kv_heads) * D, H) for _ in range(layers)]
        self.out = [make(H, q_heads * D) for _ in range(layers)]
        self.head = make(V, H)
        self.rope = csd.RopePlan(D, layout="half", scaling="parts", factor=4.0, original_len=1024, device=device)

    @staticmethod
    def normed(x):
        y = x.float()
        return (y * torch.rsqrt(y.square().mean(-1, keepdim=True) + 1e-6)).to(x.dtype)

    def hidden(self, tokens, cache, buffers):
        """tokens [rows, T]: new tokens of every row, of which the last extension of the cache granted the first cache.granted[row]
        -> [rows, T, H].  After an extension that found no room that is none of them: nothing is stored, nothing attended to."""
        rows, T = tokens.shape
        x = self.embedding[tokens.long()]
        for layer in range(self.layers):
            qkv = (self.normed(x) @ self.qkv[layer].T).view(rows, T, -1, self.D)
            q, k, v = qkv.split([self.q_heads, self.kv_heads, self.kv_heads], dim=2)
            q = csd.csd_rope_append(q, k, v, cache, layer, self.rope, n_new=cache.granted)
            seen = csd.csd_attention(q, cache, layer, buffers, n_new=cache.granted)
            x = x + seen.view(rows, T, -1) @ self.out[layer].T
        return self.normed(x)

    def hidden_from_scratch(self, tokens):
        """The same for one whole sequence [n], without a cache and without the library's kernels."""
        n = tokens.numel()
        x = self.embedding[tokens.long()]
        turn = torch.arange(n, device=x.device)[:, None] * (self.rope.steps.double() / 2.0 ** 64 * 2 * torch.pi)
        c, s = turn.cos()[:, None].float(), turn.sin()[:, None].float()
        seen_by = torch.ones(n, n, dtype=torch.bool, device=x.device).tril()
        for layer in range(self.layers):
            qkv = (self.normed(x) @ self.qkv[layer].T).view(n, -1, self.D)
            q, k, v = qkv.float().split([self.q_heads, self.kv_heads, self.kv_heads], dim=1)

            def turned(y):
                a, b = y.chunk(2, dim=-1)
                return torch.cat([a * c - b * s, b * c + a * s], dim=-1).to(x.dtype).float()
            q, k = turned(q), turned(k).repeat_interleave(self.q_heads // self.kv_heads, dim=1)
            v = v.repeat_interleave(self.q_heads // self.kv_heads, dim=1)
            w = (torch.einsum("ihd,jhd->hij", q, k) * self.D ** -0.5).masked_fill(~seen_by, float("-inf")).softmax(-1)
            seen = torch.einsum("hij,jhd->ihd", w, v).to(x.dtype)
            x = x + seen.reshape(n, -1) @ self.out[layer].T
        return self.normed(x)


def decode(target: Target, rows=8, K=4, steps=40, prompt_len=100, page_size=16, seed=1):
    """Returns (sequences: one list of tokens per row, the target's hidden states of the last step's kept tokens, cache)."""
    dev = target.embedding.device
    gen = torch.Generator(device=dev).manual_seed(seed)
    longest = prompt_len + steps * (K + 1) + K + 1
    cache = csd.PagedCache(rows, rows * -(-longest // page_size), page_size, target.layers, target.kv_heads, target.D, torch.bfloat16, longest)
    only_first = torch.zeros(rows, dtype=torch.int32, device=dev)

    # the prompt, all but its last token, into row 0, a piece at a time; the other rows then continue row 0
    prompt = torch.randint(0, target.V, (prompt_len,), generator=gen, device=dev, dtype=torch.int32)
    piece = csd.CSD_MAX_K + 1
    buffers = csd.AttentionBuffers(cache, piece, target.q_heads)
    for at in range(0, prompt_len - 1, piece):
        part = prompt[at:min(at + piece, prompt_len - 1)]
        only_first[0] = part.numel()
        tokens = torch.zeros(rows, piece, dtype=torch.int32, device=dev)
        tokens[0, :part.numel()] = part
        csd.csd_cache_extend(cache, piece, only_first)
        target.hidden(tokens, cache, buffers)
    csd.csd_cache_fork(cache, torch.zeros(rows, dtype=torch.int32, device=dev))

    # rows begin with different tokens, or all would say the same
    last = torch.randint(0, target.V, (rows,), generator=gen, device=dev, dtype=torch.int32)
    successor = torch.arange(target.V, device=dev, dtype=torch.int32).roll(-1)
    ocm = csd.Ocm(4096, lam=6)
    buf = csd.LmheadBuffers(rows, K, target.H, target.V)
    buffers = csd.AttentionBuffers(cache, K + 1, target.q_heads)
    said = []                                                    # per step: tokens [rows, K + 1], how many were kept
    for _ in range(steps):
        tokens = [last]
        for _ in range(K):
            tokens.append(successor[tokens[-1].long()])
        tokens = torch.stack(tokens, dim=1)
        draft = tokens[:, 1:].contiguous()
        csd.csd_cache_extend(cache, K + 1)
        hidden = target.hidden(tokens, cache, buffers)
        csd.csd_step_lmhead(hidden, target.head, draft, ocm, 0.3, buf)
        csd.csd_cache_commit(cache, buf.accept_len)
        said.append((tokens, buf.accept_len + 1))
        emitted = tokens.gather(1, buf.accept_len[:, None].long())[:, 0]
        last = buf.next_token.clone()
        successor[emitted.long()] = last
    if cache.stats()["flags"]:                                    # an extension found no room, or worse
        raise RuntimeError(f"cache flags {cache.stats()['flags']:#x}")
    sequences = [prompt[:-1].tolist() for _ in range(rows)]
    for tokens, kept in said:
        for r, (row, n) in enumerate(zip(tokens.tolist(), kept.tolist())):
            sequences[r] += row[:n]
    ocm.close()
    return sequences, hidden, said[-1][1], cache


def check(target, sequences, hidden, kept, cache):
    """Largest difference, in units of the states' root mean square of 1, between the last step's hidden states and a computation
    from scratch; the cache's lengths have to be the sequences'."""
    assert cache.lens.tolist() == [len(s) for s in sequences] and cache.stats()["flags"] == 0
    worst = 0.0
    for r, s in enumerate(sequences):
        n = int(kept[r])
        want = target.hidden_from_scratch(torch.tensor(s, device=hidden.device))[-n:]
        worst = max(worst, float((hidden[r, :n].float() - want.float()).square().mean().sqrt()))
    return worst


def main():
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--rows", type=int, default=8)
    ap.add_argument("--drafts", type=int, default=4)
    ap.add_argument("--steps", type=int, default=40)
    ap.add_argument("--prompt", type=int, default=100)
    ap.add_argument("--check", action="store_true")
    a = ap.parse_args()
    target = Target()
    sequences, hidden, kept, cache = decode(target, a.rows, a.drafts, a.steps, a.prompt)
    st = cache.stats()
    made = sum(len(s) for s in sequences) - a.rows * (a.prompt - 1)
    print(f"{made} tokens in {a.steps} steps of {a.rows} rows; cache: {st['tokens']} tokens in {st['pages']} pages, {st['shared']} of them shared")
    if a.check:
        print(f"hidden states against a computation without cache: rms difference {check(target, sequences, hidden, kept, cache):.4f}")


if __name__ == "__main__":
    main()
