"""csd_attention_mass against its 64-bit statement (oracle/tree_oracle.py).

Tolerance.  Scores: D products summed in float32, at most 2 (D + 8) 2^-24 sum_d |scale q k| off; the exponent's two products and its sum
round once each, relative to the sizes of score and lse (the constant scale log2(e) is rounded too): together at most
(2 (D + 8) + 8) 2^-24 S with S = max sum_d |scale q k| + |lse|.  A weight is off by the factor e^that, the exponential itself by 2^-21; a
place's sum of N weights by N 2^-24, and the addition to what was there by 2^-24 of the result.  Weights below 2^-126 may become 0.
"""

import numpy as np
import pytest
import torch

from oracle import decode_oracle as D
from oracle import tree_oracle as O
from paper_2604_13634_b200 import (AttentionBuffers, CsdError, PagedCache, TreePlan, csd_attention, csd_attention_mass, csd_attention_tree,
                                   csd_cache_extend, csd_tree_plan)
from test_gpu_tree import as_i64, f64, filled, gen_of, i32, rand, rows_of, some_parents

pytestmark = pytest.mark.gpu


def check(mass, before, q, lse, cache, table, lens, news, masks, scale, fresh):
    got, was = f64(mass), f64(before)
    T, Hq, dim = q.shape[1:]
    for b, n in enumerate(lens):
        k, _ = rows_of(cache, table, b, n)
        want, size = O.mass(f64(q[b]), k, f64(lse[b]), masks[b], news[b], scale, was[b], fresh)
        start = np.array(was[b, :n])
        if fresh and news[b] > 0:
            start[max(n - news[b], 0):] = 0.0
        given = want - start
        rel = 2 * (2 * (dim + 8) + 8) * 2.0 ** -24 * size + 2.0 ** -21 + T * Hq * 2.0 ** -24
        bound = rel * given + 2.0 ** -23 * np.abs(want) + T * Hq * 2.0 ** -125
        err = np.abs(got[b, :n] - want)
        assert (err <= bound).all(), (b, float((err - bound).max()), float(given.max()))
        assert np.array_equal(got[b, n:], was[b, n:]), b


def chain(T):
    return [2 ** (t + 1) - 1 for t in range(T)]


CASES = [  # rows' lengths, T, query heads, key heads, dim, page
    ([1], 1, 1, 1, 64, 16),
    ([700], 1, 32, 8, 128, 16),
    ([129, 128, 127, 0, 5], 1, 12, 3, 80, 8),
    ([40, 2500, 9], 9, 8, 2, 128, 64),
    ([64, 65, 300, 70], 64, 8, 1, 128, 256),                            # 512 query rows: four passes
    ([33, 600], 33, 6, 1, 256, 32),                                     # 198 of 64 at a time
    ([100] * 20, 2, 10, 5, 192, 16),
    (list(range(60)), 3, 4, 2, 72, 16),
    ([5000, 20, 4097], 16, 2, 2, 64, 128),
]


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("fresh", [False, True])
@pytest.mark.parametrize("lens,T,Hq,Hkv,dim,page", CASES)
def test_mass(dtype, fresh, lens, T, Hq, Hkv, dim, page):
    rng, gen = np.random.default_rng(dim + T), gen_of(T + page)
    cache, table = filled(T + dim, lens, page, Hkv, dim, dtype, token_major=dim in (64, 80), poison=float("nan"))
    news = [min(n, T if b % 2 == 0 else int(rng.integers(0, T + 1))) for b, n in enumerate(lens)]
    q = rand(gen, len(lens), T, Hq, dim, dtype=dtype)
    parents, plan = [some_parents(rng, T) for _ in lens], TreePlan(cache, T)
    csd_tree_plan(i32(parents), cache, plan, n_new=i32(news))
    buf = AttentionBuffers(cache, T, Hq, tree=True)
    csd_attention_tree(q, cache, 0, buf, plan.masks, n_new=i32(news))
    before = torch.rand(len(lens), cache.max_pages * page + 2, generator=gen, device="cuda")
    masks = [O.plan(parents[b], news[b], 0)[0] for b in range(len(lens))]
    mass = before.clone()
    assert csd_attention_mass(q, buf.lse, cache, 0, mass, n_new=i32(news), masks=plan.masks, fresh=fresh) is mass
    check(mass, before, q, buf.lse, cache, table, lens, news, masks, dim ** -0.5, fresh)
    # every token that sees something hands out a weight of 1 per head
    tokens = torch.tensor([sum(bool(O.sees(masks[b][t], news[b], n, t)) for t in range(T)) for b, n in enumerate(lens)], device="cuda")
    given = torch.zeros_like(before)
    csd_attention_mass(q, buf.lse, cache, 0, given, n_new=i32(news), masks=plan.masks)
    assert torch.allclose(given.double().sum(1), (tokens * Hq).double(), rtol=1e-3, atol=0)      # lse and scores: 2 (D + 8) 2^-24 S each, S <= 16
    again = before.clone()
    csd_attention_mass(q, buf.lse, cache, 0, again, n_new=i32(news), masks=plan.masks, fresh=fresh)
    assert torch.equal(again, mass) and cache.stats()["flags"] == 0


@pytest.mark.parametrize("T,Hq", [(1, 4), (9, 36), (33, 3)])
def test_chain(T, Hq):
    lens, gen = [T + 3, 1000, 0, T, 257], gen_of(T)
    cache, table = filled(T, lens, 16, 1, 128, torch.bfloat16, poison=float("inf"))
    q, buf = rand(gen, len(lens), T, Hq, 128), AttentionBuffers(cache, T, Hq)
    csd_attention(q, cache, 0, buf, scale=0.11)
    mass = torch.zeros(len(lens), cache.max_pages * 16, device="cuda")
    csd_attention_mass(q, buf.lse, cache, 0, mass, scale=0.11)
    check(mass, torch.zeros_like(mass), q, buf.lse, cache, table, lens, [T] * len(lens), [chain(T)] * len(lens), 0.11, False)


def test_tokens_that_add_nothing():
    """lse of minus infinity, tokens without a place, rows without new tokens; NaN in the queries of tokens that do not exist."""
    T, Hq, lens, news = 5, 4, [3, 300, 200, 4], [5, 3, 0, 70]
    cache, table = filled(9, lens, 16, 2, 64, torch.bfloat16)
    q = rand(gen_of(1), 4, T, Hq, 64)
    q[1, 3:] = float("nan")
    q[0, :2] = float("nan")                                              # places -2 and -1
    lse = torch.full((4, T, Hq), 1.5, device="cuda")
    lse[1, 1] = -float("inf")
    q[1, 1, 2] = float("nan")
    masks = [[31] * T, [7, 7, 4, 31, 31], [31] * T, [2 ** 64 - 1] * T]
    before = torch.rand(4, cache.max_pages * 16, device="cuda")
    for fresh in (False, True):
        mass = before.clone()
        csd_attention_mass(q, lse, cache, 0, mass, n_new=i32(news), masks=as_i64(masks), fresh=fresh)
        check(mass, before, torch.nan_to_num(q), lse, cache, table, lens, news, masks, 64 ** -0.5, fresh)
        assert torch.equal(mass[2], before[2])


def test_on_a_stream_in_a_graph_with_strides():
    """Queries that are slices of a projection, a mass with a stride of its own, another stream, a replayed graph: the same numbers."""
    lens, T = [500, 90], 4
    cache, _ = filled(3, lens, 16, 2, 128, torch.float16)
    wide = rand(gen_of(2), 2, T, 12, 128, dtype=torch.float16)
    q, lse = wide[:, :, 2:10], torch.full((2, T, 8), 3.0, device="cuda")
    want = torch.zeros(2, cache.max_pages * 16, device="cuda")
    csd_attention_mass(q.contiguous(), lse, cache, 0, want)
    mass = torch.zeros(2, cache.max_pages * 16 + 7, device="cuda")
    part, side, graph = mass[:, :cache.max_pages * 16], torch.cuda.Stream(), torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    csd_attention_mass(q, lse, cache, 0, part, stream=side)
    side.synchronize()
    assert torch.equal(part, want) and not mass[:, cache.max_pages * 16:].any()
    mass.zero_()
    with torch.cuda.graph(graph):
        csd_attention_mass(q, lse, cache, 0, part)
        csd_attention_mass(q, lse, cache, 0, part)
    graph.replay()
    torch.cuda.synchronize()
    assert torch.allclose(part, 2 * want, rtol=2.0 ** -23, atol=0)


def test_refusals():
    cache, _ = filled(1, [40, 40], 16, 2, 64, torch.bfloat16)
    q, lse, mass = rand(gen_of(1), 2, 3, 4, 64), torch.zeros(2, 3, 4, device="cuda"), torch.zeros(2, 48, device="cuda")
    for scale in (float("nan"), float("inf")):
        with pytest.raises(CsdError):
            csd_attention_mass(q, lse, cache, 0, mass, scale=scale)
    for layer in (-1, 1):
        with pytest.raises(CsdError):
            csd_attention_mass(q, lse, cache, layer, mass)
    with pytest.raises(CsdError):
        csd_attention_mass(rand(gen_of(1), 2, 65, 4, 64), torch.zeros(2, 65, 4, device="cuda"), cache, 0, mass)
    with pytest.raises(CsdError):
        csd_attention_mass(rand(gen_of(1), 2, 3, 3, 64), torch.zeros(2, 3, 3, device="cuda"), cache, 0, mass)
    with pytest.raises(CsdError):                                        # not 16 bytes aligned
        csd_attention_mass(rand(gen_of(1), 2, 3, 4, 72)[..., 4:68], lse, cache, 0, mass)
    for bad in (dict(lse=lse[:, :2]), dict(lse=lse.double()), dict(mass=mass[:, :40]), dict(q=q.half())):
        with pytest.raises(AssertionError):
            csd_attention_mass(**{**dict(q=q, lse=lse, cache=cache, layer=0, mass=mass), **bad})
    with pytest.raises(CsdError, match="device"):
        csd_attention_mass(q, lse.cpu(), cache, 0, mass)
