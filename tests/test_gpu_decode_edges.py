"""Edges of the decode-pass operators: arguments that have to be refused, and places where a result could go wrong silently."""

import math
import os
import sys

import numpy as np
import pytest
import torch

from oracle import decode_oracle as O
from paper_2604_13634_b200 import (AttentionBuffers, CsdError, PagedCache, RopePlan, csd_attention, csd_cache_commit, csd_cache_extend, csd_cache_fork,
                                   csd_rope, csd_rope_append, decode)

pytestmark = pytest.mark.gpu

HERE = os.path.dirname(os.path.abspath(__file__))
sys.path.insert(0, HERE)
from test_gpu_decode import ULP, check_attention, f64, filled_cache, rand  # noqa: E402


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
                 lambda: csd_cache_extend(cache, 1), lambda: decode.csd_cache_compact(cache)):
        with pytest.raises(CsdError, match="device"):
            call()


@pytest.mark.parametrize("poison", [math.nan, math.inf])
@pytest.mark.parametrize("dtype,Hq,Hkv,D,T,page", [(torch.bfloat16, 4, 2, 64, 3, 16), (torch.float16, 16, 2, 256, 2, 64), (torch.bfloat16, 8, 1, 128, 9, 16),
                                                   (torch.float16, 24, 1, 64, 1, 32), (torch.bfloat16, 20, 2, 256, 4, 128)])
def test_a_pass_over_the_first_of_many_new_tokens(poison, dtype, Hq, Hkv, D, T, page):
    """n_new > T: token t lies at lens - n_new + t, and sees neither the places after it nor what they hold (nothing is written there yet)."""
    lens, news = [400, 130, 64, 20, 700, 65], [300, T + 1, 64, 25, T, 2 ** 31 - 1]
    cache, gen = filled_cache(50, lens, page, Hkv, D, dtype, False)
    for b, n in enumerate(lens):
        for at in range(max(0, n - news[b] + T), n):
            page_id = int(cache.table[b, at // page])
            cache.k[0, page_id, :, at % page] = poison
            cache.v[0, page_id, :, at % page] = poison
    q = rand(gen, len(lens), T, Hq, D, dtype=dtype, scale=2.0)
    buf = AttentionBuffers(cache, T, Hq)
    csd_attention(q, cache, 0, buf, n_new=torch.tensor(news, dtype=torch.int32, device="cuda"))
    check_attention(buf, q, cache, lens, news, 1 / math.sqrt(D))
    assert cache.stats()["flags"] == 0


def test_a_prompt_in_pieces_after_one_extension():
    """Room for the whole prompt once, then pieces of T tokens with n_new = what is left: each token sees what it would see alone."""
    n, T, Hq, Hkv, D = 150, 33, 8, 2, 64
    caches = [PagedCache(2, 24, 16, 1, Hkv, D, torch.bfloat16, 192) for _ in range(2)]
    gen = torch.Generator(device="cuda").manual_seed(8)
    qkv = rand(gen, 2, 5 * T, Hq + 2 * Hkv, D)
    plan = RopePlan(D)
    outs = []
    for whole, cache in zip((True, False), caches):
        cache.k.fill_(math.nan), cache.v.fill_(math.nan)
        buf, got = AttentionBuffers(cache, T, Hq), []
        if whole:
            csd_cache_extend(cache, n)
        for at in range(0, n, T):
            left = torch.full((2,), n - at if whole else min(T, n - at), dtype=torch.int32, device="cuda")
            if not whole:
                csd_cache_extend(cache, T, left)
            q, k, v = qkv[:, at:at + T].split([Hq, Hkv, Hkv], dim=2)
            q = csd_rope_append(q, k, v, cache, 0, plan, n_new=left)
            got.append(csd_attention(q, cache, 0, buf, n_new=left).clone())
        outs.append(torch.cat(got, dim=1))
        assert cache.stats()["flags"] == 0 and cache.lens.tolist() == [n, n]
    assert torch.isfinite(outs[0].float()).all() and not outs[0][:, n:].any()
    for a, b in zip(caches[0].table[0].tolist(), caches[1].table[0].tolist()):
        assert a < 0 or torch.equal(caches[0].k[0, a].nan_to_num(), caches[1].k[0, b].nan_to_num())
    # the splits differ with the lengths, so the sums' order does: two roundings of bf16
    assert (outs[0] - outs[1]).abs().max() <= 2 * 2.0 ** -8 * qkv[..., Hq + Hkv:, :].abs().max()


@pytest.mark.parametrize("extreme,kept", [(2 ** 31 - 1, 5), (-2 ** 31, 0)])
def test_commit_takes_any_accepted_count(extreme, kept):
    cache = PagedCache(3, 12, 8, 1, 1, 64, torch.bfloat16, 64)
    csd_cache_extend(cache, 20)
    csd_cache_commit(cache, torch.full((3,), 19, dtype=torch.int32, device="cuda"))
    csd_cache_extend(cache, 5)
    csd_cache_commit(cache, torch.tensor([extreme, 1, extreme], dtype=torch.int32, device="cuda"))
    assert cache.lens.tolist() == [20 + kept, 22, 20 + kept]


def test_a_pool_of_one_head_keeps_its_token_stride():
    for shape, halves in (((2, 4, 1, 16, 128), 4), ((2, 4, 1, 32, 64), 3)):
        kv = torch.zeros(shape, dtype=torch.bfloat16, device="cuda")
        k, v = kv.split(64, dim=4) if halves == 4 else (kv[:, :, :, 0::2], kv[:, :, :, 1::2])
        with pytest.raises(CsdError):
            PagedCache(1, 4, 16, 2, 1, 64, torch.bfloat16, 64, k=k, v=v)
    for shape in ((2, 4, 1, 16, 64), (2, 4, 16, 1, 64)):
        k, v = (torch.zeros(shape, dtype=torch.bfloat16, device="cuda").view(2, 4, 1, 16, 64) for _ in range(2))
        cache = PagedCache(1, 4, 16, 2, 1, 64, torch.bfloat16, 64, k=k, v=v)
        csd_cache_extend(cache, 3)
        new = torch.arange(3, device="cuda").view(1, 3, 1, 1).expand(1, 3, 1, 64).to(torch.bfloat16)
        csd_rope_append(new, new, new, cache, 1, None)
        assert torch.equal(cache.k[1, 0, 0, :3], new[0, :, 0]) and torch.equal(cache.v[1, 0, 0, :3], new[0, :, 0])


def test_a_refused_extension_leaves_every_page_as_it_was():
    sys.path.insert(0, os.path.join(os.path.dirname(HERE), "examples"))
    import decode_with_cache as example
    target = example.Target()
    cache = PagedCache(3, 3, 16, target.layers, target.kv_heads, target.D, torch.bfloat16, 64)
    buffers = AttentionBuffers(cache, 5, target.q_heads)
    tokens = torch.arange(15, dtype=torch.int32, device="cuda").view(3, 5)
    n = torch.tensor([5, 0, 0], dtype=torch.int32, device="cuda")
    for _ in range(4):
        csd_cache_extend(cache, 5, n)
        target.hidden(tokens, cache, buffers)
    csd_cache_fork(cache, torch.zeros(3, dtype=torch.int32, device="cuda"))
    assert cache.lens.tolist() == [20] * 3 and cache.stats() == dict(flags=0, pages=2, shared=2, tokens=60)
    k, v, table = cache.k.clone(), cache.v.clone(), cache.table.clone()
    csd_cache_extend(cache, 5)                                        # two copies of the shared last page are wanted, one page is free
    target.hidden(tokens, cache, buffers)
    csd_cache_commit(cache, torch.full((3,), 2, dtype=torch.int32, device="cuda"))
    assert torch.equal(cache.k, k) and torch.equal(cache.v, v) and torch.equal(cache.table, table)
    assert cache.lens.tolist() == [20] * 3 and cache.stats()["flags"] == decode.CACHE_FULL


def test_load_of_a_narrower_table_keeps_nothing_of_the_one_before():
    cache = PagedCache(2, 20, 8, 1, 1, 64, torch.bfloat16, 64)
    table = torch.arange(16, dtype=torch.int32).view(2, 8)
    cache.load(table, torch.tensor([64, 64], dtype=torch.int32))
    cache.load(table[:, :2].contiguous(), torch.tensor([40, 16], dtype=torch.int32))
    assert cache.stats()["flags"] == decode.CACHE_BAD_PAGE and (cache.table[:, 2:] == -1).all()
    assert cache.refs.tolist() == [1, 1] + [0] * 6 + [1, 1] + [0] * 10


def test_buffers_of_another_type_are_refused():
    caches = [PagedCache(1, 4, 16, 1, 2, 64, dtype, 64) for dtype in (torch.bfloat16, torch.float16)]
    buf = AttentionBuffers(caches[0], 1, 2)
    with pytest.raises(AssertionError):
        csd_attention(torch.zeros(1, 1, 2, 64, dtype=torch.float16, device="cuda"), caches[1], 0, buf)


def test_results_belong_to_the_stream_that_writes_them():
    s = torch.cuda.Stream()
    x, pos, plan = torch.randn(1, 500, 8, 64, device="cuda"), torch.zeros(1, 500, dtype=torch.int32, device="cuda"), RopePlan(64)
    cache = PagedCache(1, 64, 16, 1, 8, 64, torch.bfloat16, 1024)
    q = torch.zeros(1, 300, 8, 64, dtype=torch.bfloat16, device="cuda")
    csd_cache_extend(cache, 300)
    torch.cuda.synchronize()
    for call in (lambda: csd_rope(x, pos, plan, stream=s), lambda: csd_rope_append(q, q, q, cache, 0, plan, stream=s)):
        y = call()
        torch.cuda.synchronize()
        at, like = y.data_ptr(), (y.shape, y.dtype)
        del y
        again = torch.empty(like[0], dtype=like[1], device="cuda")
        assert again.data_ptr() != at


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_rope_has_a_gradient(dtype):
    gen = torch.Generator(device="cuda").manual_seed(3)
    x = torch.randn(2, 5, 3, 80, generator=gen, device="cuda").to(dtype).requires_grad_()
    g = torch.randn(2, 5, 3, 80, generator=gen, device="cuda").to(dtype)
    pos = torch.randint(0, 5000, (2, 5), generator=gen, device="cuda", dtype=torch.int32)
    plan = RopePlan(64, layout="interleaved", scaling="yarn", factor=4.0)
    y = csd_rope(x, pos, plan)
    assert y.requires_grad and torch.equal(y, csd_rope(x.detach(), pos, plan))
    (got,) = torch.autograd.grad(y, x, g)
    assert torch.equal(got, csd_rope(g, pos, plan, inverse=True))
    (got,) = torch.autograd.grad(csd_rope(x, pos, plan, inverse=True).sum(), x)      # a gradient without strides, of the turn back
    assert torch.equal(got, csd_rope(torch.ones_like(g), pos, plan))
    with pytest.raises(CsdError, match="gradient"):
        csd_rope(x, pos, plan, out=torch.empty_like(x))
    with torch.no_grad():
        assert not csd_rope(x, pos, plan, out=torch.empty_like(x)).requires_grad


@pytest.mark.parametrize("group,T,raised", [(2, 1, 14), (20, 1, 7), (3, 9, 7)])     # 2 query rows to a key head, 20 and 27
@pytest.mark.parametrize("at", [0, 70000, 131071])
def test_many_small_weights_in_float16(group, T, raised, at):
    """One place with most of the weight and 131071 with 2^-25.1 of it each, which a weight rounded to float16 as it is would drop.
    The rows share their pages; there are more of them than blocks, so that some are read by one block whole."""
    n, D, rows, heads = 131072, 64, 40, 8
    cache = PagedCache(rows, n // 64, 64, 1, heads, D, torch.float16, n)
    cache.load(torch.arange(n // 64, dtype=torch.int32, device="cuda").expand(rows, -1), torch.full((rows,), n, dtype=torch.int32, device="cuda"))
    cache.v.fill_(1.0)
    cache.k[0, at // 64, :, at % 64, 0] = 1.0
    cache.v[0, at // 64, :, at % 64] = 0.0
    q = torch.zeros(rows, T, heads * group, D, dtype=torch.float16, device="cuda")
    q[..., 0] = 16.0
    scale = 25.1 * math.log(2) / 16
    buf = AttentionBuffers(cache, T, heads * group)
    csd_attention(q, cache, 0, buf, scale=scale)
    k, v = (f64(x[0, :, 0]).reshape(1, n, D) for x in (cache.k, cache.v))
    out, lse, reach, size = O.attention(f64(q[0, :, :1]), k, v, T, scale)                # all heads hold the same
    e, u = 2 * (D + 8) * 2.0 ** -24 * size, ULP[torch.float16]
    # a weight is off by half of float16's smallest step at most, in units of the largest weight raised by `raised` powers of two
    bound = (u + (2 * e + 2.0 ** -20 + n * 2.0 ** -24)[..., None]) * reach + u * np.abs(out) + n * 2.0 ** -(25 + raised) + 2.0 ** -24
    err = np.abs(f64(buf.out) - out[None])
    assert (err <= bound[None]).all(), (float(err.max()), float(bound.min()), float(out.max()))
    assert np.abs(f64(buf.lse) - lse[None]).max() <= e.max() + 2.0 ** -20 + n * 2.0 ** -24 + 2.0 ** -22 * np.abs(lse).max()


@pytest.mark.parametrize("Hq", [2, 20])
@pytest.mark.parametrize("n", [1, 50, 300, 9000])
def test_scores_of_minus_infinity(Hq, n):
    D, page = 64, 16
    cache, gen = filled_cache(51, [n, n, n], page, 1, D, torch.bfloat16, False)
    q = rand(gen, 3, 1, Hq, D)
    q[..., 0] = q[..., 0].abs() + 0.5
    places = {0: range(n), 1: range(n // 2), 2: range(n - n // 2, n)}
    for b, r in places.items():
        at = torch.tensor(list(r), dtype=torch.long, device="cuda")
        cache.k[0, cache.table[b, at // page].long(), 0, at % page, 0] = -math.inf
    buf = AttentionBuffers(cache, 1, Hq)
    csd_attention(q, cache, 0, buf)
    assert not buf.out[0].any() and torch.isneginf(buf.lse[0]).all()
    for b in (1, 2):
        keep = [j for j in range(n) if j not in places[b]]
        k, v = (O.rows_of(f64(x[0]), cache.table[b].tolist(), n, page)[:, keep] for x in (cache.k, cache.v))
        out, lse, reach, size = O.attention(f64(q[b]), k, v, 1, D ** -0.5)
        e = 2 * (D + 8) * 2.0 ** -24 * size
        u = ULP[torch.bfloat16]
        assert (np.abs(f64(buf.out[b]) - out) <= (u + (2 * e + 2.0 ** -20 + n * 2.0 ** -24)[..., None]) * reach + u * np.abs(out)).all()
        assert np.abs(f64(buf.lse[b]) - lse).max() <= e.max() + 2.0 ** -20 + n * 2.0 ** -24 + 2.0 ** -22 * np.abs(lse).max()


@pytest.mark.parametrize("Hq", [2, 20])
def test_attention_over_the_most_rows(Hq):
    """4096 rows: the table of their tiles leaves the fewest stages for keys and values; rows of no tile, one, and several."""
    rows, page, D = 4096, 8, 64
    lens = [(i * 7) % 150 if i % 5 else 0 for i in range(rows - 1)] + [3000]
    cache, gen = filled_cache(52, lens, page, 1, D, torch.bfloat16, False)
    q = rand(gen, rows, 1, Hq, D, scale=2.0)
    buf = AttentionBuffers(cache, 1, Hq)
    csd_attention(q, cache, 0, buf)
    check_attention(buf, q, cache, lens, [1] * rows, 1 / math.sqrt(D), rows=list(range(0, rows, 61)) + [rows - 1])
    empty = torch.tensor([n == 0 for n in lens], device="cuda")
    assert not buf.out[empty].any() and torch.isneginf(buf.lse[empty]).all() and torch.isfinite(buf.lse[~empty]).all()
    first = buf.out.clone()
    for _ in range(5):
        csd_attention(q, cache, 0, buf)
        assert torch.equal(buf.out, first)
    assert cache.stats()["flags"] == 0


@pytest.mark.parametrize("dtype,token_major,layout,D,rot", [(torch.bfloat16, False, "half", 128, 128), (torch.float16, True, "interleaved", 80, 34)])
@pytest.mark.parametrize("T", [34, 300, 1001])
def test_rope_append_of_a_prompt(dtype, token_major, layout, D, rot, T):
    """Any number of new tokens: queries and keys as csd_rope turns them, values as they are, each at its place."""
    page, Hq, Hkv, lens = 16, 5, 2, [T, T + 700, T - 1, 40]
    cache, gen = filled_cache(53, lens, page, Hkv, D, dtype, token_major)
    news = [T, T, T - 1, 7]
    qkv = rand(gen, len(lens), T, Hq + 2 * Hkv, D, dtype=dtype)
    q, k, v = qkv.split([Hq, Hkv, Hkv], dim=2)
    plan = RopePlan(rot, layout=layout, scaling="parts", factor=8.0)
    pos = torch.tensor([n - m for n, m in zip(lens, news)], dtype=torch.int32, device="cuda")[:, None] + torch.arange(T, dtype=torch.int32, device="cuda")
    want_q, want_k = csd_rope(q, pos, plan), csd_rope(k, pos, plan)
    out = csd_rope_append(q, k, v, cache, 0, plan, n_new=torch.tensor(news, dtype=torch.int32, device="cuda"))
    for b, m in enumerate(news):
        assert torch.equal(out[b, :m], want_q[b, :m]) and not out[b, m:].any()
        at = pos[b, :m].long()
        pages = cache.table[b, at // page].long()
        assert torch.equal(cache.k[0, pages, :, at % page], want_k[b, :m]) and torch.equal(cache.v[0, pages, :, at % page], v[b, :m])
    assert cache.stats()["flags"] == 0
