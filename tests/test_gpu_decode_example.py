"""The example that runs the decode-pass operators together with the verification step, and the operators at sizes where a
block works on many tiles of many units."""

import math
import os
import sys

import pytest
import torch

from paper_2604_13634_b200 import AttentionBuffers, PagedCache, csd_attention

pytestmark = pytest.mark.gpu

sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))


@pytest.mark.parametrize("rows,K,steps,prompt", [(1, 1, 5, 2), (8, 4, 30, 100), (5, 8, 20, 257)])
def test_decoding_with_the_cache_equals_decoding_without(rows, K, steps, prompt):
    """bf16 states of root mean square 1 after two layers: a rounding is at most 2^-9 of a value, and each layer makes about
    six of them on either side; 0.02 is five times the sum of twelve of random sign."""
    import decode_with_cache as example
    target = example.Target()
    sequences, hidden, kept, cache = example.decode(target, rows, K, steps, prompt)
    assert example.check(target, sequences, hidden, kept, cache) < 0.02
    assert all(len(s) >= prompt - 1 + steps for s in sequences)
    st = cache.stats()
    shared = (prompt - 1) // 16 if rows > 1 else 0                 # whole pages of the prompt
    assert st["shared"] == shared and st["pages"] == shared + sum(-(-n // 16) - shared for n in cache.lens.tolist())


def attention64(q, cache, news, scale):
    """The definition in float64 on the GPU, row by row; and the error bounds' pieces as in test_gpu_decode."""
    B, T, Hq, D = q.shape
    group, page = Hq // cache.kv_heads, cache.page_size
    out = torch.zeros(q.shape, dtype=torch.float64, device="cuda")
    reach, lse, size = torch.zeros_like(out), torch.full(q.shape[:3], -math.inf, dtype=torch.float64, device="cuda"), torch.zeros(q.shape[:3], dtype=torch.float64, device="cuda")
    for b, n in enumerate(cache.lens.tolist()):
        if n == 0:
            continue                                               # nothing to see: zeros and -inf
        ids = cache.table[b, :-(-n // page)].long()
        k, v = (x[0, ids].double().transpose(0, 1).reshape(cache.kv_heads, -1, D)[:, :n].repeat_interleave(group, 0) for x in (cache.k, cache.v))
        last = n - news[b] + torch.arange(T, device="cuda")
        last = torch.where(torch.arange(T, device="cuda") < news[b], last, -1)
        x = torch.einsum("thd,hjd->thj", q[b].double(), k) * scale
        x = x.masked_fill(torch.arange(n, device="cuda") > last[:, None, None], -math.inf)
        w = torch.where(last[:, None, None] >= 0, x, torch.zeros_like(x)).softmax(-1) * (last >= 0)[:, None, None]
        out[b], reach[b] = torch.einsum("thj,hjd->thd", w, v), torch.einsum("thj,hjd->thd", w, v.abs())
        lse[b] = x.logsumexp(-1)
        size[b] = torch.einsum("thd,hjd->thj", q[b].double().abs(), k.abs()).amax(-1) * abs(scale)
    return out, lse, reach, size


@pytest.mark.parametrize("dtype,page,Hq,Hkv,D,T,lens,ragged,token_major", [
    (torch.bfloat16, 16, 40, 8, 128, 6, [int(300 * i) for i in range(24)], True, False),      # 30 query rows, two blocks per SM
    (torch.bfloat16, 64, 32, 8, 128, 9, [500 + 90 * i for i in range(40)], False, True),       # 36
    (torch.float16, 16, 64, 8, 64, 9, [0, 12000, 7, 3001, 640, 64, 9999], True, False),         # 72
    (torch.bfloat16, 32, 17, 1, 128, 1, [20000, 1, 3000], False, False),                        # 17: the first of the kernel
    (torch.bfloat16, 16, 48, 4, 128, 9, [2500 + i for i in range(20)], True, False),            # 108: one set of query rows fits
    (torch.float16, 128, 32, 2, 96, 17, [5000, 40, 2111], True, True),                          # 272: three row tiles
    (torch.bfloat16, 8, 64, 4, 256, 5, [4000, 100, 0, 1777], False, False),                      # 80 rows of 256 elements, one block per SM
    (torch.bfloat16, 64, 24, 3, 192, 4, [3000, 1000, 90], True, False),                          # 32 rows of 192
    (torch.bfloat16, 16, 8, 8, 128, 1, [17 * i for i in range(300)], False, False),               # one row a head, thousands of units
    (torch.float16, 32, 16, 16, 64, 1, [int(110 * i) for i in range(30)], False, True),           # 64 elements: wide tiles
    (torch.bfloat16, 16, 4, 2, 256, 4, [6000, 1, 2, 300, 0, 77], True, False)])                   # 256 elements, 8 rows
def test_attention_with_many_tiles_to_a_block(dtype, page, Hq, Hkv, D, T, lens, ragged, token_major):
    gen, rows = torch.Generator(device="cuda").manual_seed(7), len(lens)
    need = sum(-(-n // page) for n in lens)
    cache = PagedCache(rows, need + 1, page, 1, Hkv, D, dtype, max(lens), token_major=token_major)
    for pool in (cache.k, cache.v):
        pool.copy_(torch.randn(pool.shape, generator=gen, device="cuda"))
    ids = torch.randperm(need, generator=gen, device="cuda").int()
    table, at = torch.full((rows, cache.max_pages), -1, dtype=torch.int32, device="cuda"), 0
    for r, n in enumerate(lens):
        m = -(-n // page)
        table[r, :m] = ids[at:at + m]
        at += m
    cache.load(table, torch.tensor(lens, dtype=torch.int32, device="cuda"))
    news = [min(n, 1 + r % T) for r, n in enumerate(lens)] if ragged else [T] * rows
    n_new = torch.tensor(news, dtype=torch.int32, device="cuda") if ragged else None
    q = (torch.randn((rows, T, Hq, D), generator=gen, device="cuda") * 2).to(dtype)
    buf = AttentionBuffers(cache, T, Hq)
    csd_attention(q, cache, 0, buf, n_new=n_new)
    out, lse, reach, size = attention64(q, cache, news, D ** -0.5)
    u = 2.0 ** -8 if dtype == torch.bfloat16 else 2.0 ** -11
    n = cache.lens.double()[:, None, None]
    e = 2 * (D + 8) * 2.0 ** -24 * size
    bound = (u + 2 * e + 2.0 ** -20 + n * 2.0 ** -24)[..., None] * reach + u * out.abs() + 2.0 ** -24
    assert ((buf.out.double() - out).abs() <= bound).all()
    seen = torch.isfinite(lse)
    assert torch.equal(seen, torch.isfinite(buf.lse)) and not buf.out[~seen].any()
    assert ((buf.lse.double() - lse).abs() <= e + 2.0 ** -20 + n * 2.0 ** -24 + 2.0 ** -22 * lse.abs())[seen].all()
    first, first_lse = buf.out.clone(), buf.lse.clone()
    for _ in range(25):                                            # a race would show sooner or later as other bits
        csd_attention(q, cache, 0, buf, n_new=n_new)
        assert torch.equal(buf.out, first) and torch.equal(buf.lse, first_lse)
    assert cache.stats()["flags"] == 0
