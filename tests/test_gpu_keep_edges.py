"""Bookkeeping that contradicts itself: lengths and grants written by hand.  The calls bound them; nothing outside the row is touched."""

import numpy as np
import pytest
import torch

from oracle import tree_oracle as O
from paper_2604_13634_b200 import EvictBuffers, PagedCache, csd_cache_commit_path, csd_cache_evict, csd_cache_extend

pytestmark = pytest.mark.gpu


def i32(x):
    return torch.tensor(np.asarray(x), dtype=torch.int32, device="cuda")


def contents(cache, b, n):
    at = torch.arange(n, device="cuda")
    pages = cache.table[b].long()[at // cache.page_size]
    return torch.stack([x[:, pages, :, at % cache.page_size] for x in (cache.k, cache.v)])          # [2, n, layers, heads, dim]


def filled(lens, seed=0):
    cache = PagedCache(len(lens), 40, 16, 2, 2, 64, torch.bfloat16, 96)
    csd_cache_extend(cache, 0, i32(lens))
    gen = torch.Generator(device="cuda").manual_seed(seed)
    for x in (cache.k, cache.v):
        x.copy_(torch.randn(x.shape, generator=gen, device="cuda"))
    return cache, torch.rand(len(lens), cache.max_pages * 16, generator=gen, device="cuda")


@pytest.mark.parametrize("grant", [9, 2 ** 31 - 1, -3, -2 ** 31])
def test_a_grant_above_the_length(grant):
    """Counts as the row's length (below zero: as none): the path is one of the row's tokens."""
    T, lens, path = 9, [40, 5, 33, 0], [0, 2, 3, 4, 6, 7, -1, -1, -1]
    cache, mass = filled(lens)
    before, weights, table, pools = [contents(cache, b, n) for b, n in enumerate(lens)], mass.clone(), cache.table.clone(), (cache.k.clone(), cache.v.clone())
    cache.granted.copy_(i32([0, grant, 0, grant]))
    csd_cache_commit_path(cache, i32([5] * 4), i32([path] * 4), mass=mass)
    torch.cuda.synchronize()
    g = min(max(grant, 0), 5)
    kept, _ = O.kept_of_path(g, 5, path)
    order = list(range(5 - g)) + [5 - g + i for i in kept]
    assert cache.lens.tolist() == [40, len(order), 33, 0] and cache.granted.tolist() == [0] * 4
    want, row = weights.clone(), torch.zeros(5, device="cuda")
    row[:len(order)] = weights[1, order]
    want[1, :5] = row
    assert torch.equal(mass, want)
    assert torch.equal(cache.table, table) and cache.stats()["flags"] & ~0x20 == 0
    for b, order_b in enumerate([list(range(40)), order, list(range(33)), []]):
        assert torch.equal(contents(cache, b, len(order_b)), before[b][:, order_b])
    mine = int(table[1, 0])
    others = [p for p in range(cache.n_pages) if p != mine]
    assert all(torch.equal(x[:, others], y[:, others]) for x, y in zip((cache.k, cache.v), pools))


@pytest.mark.parametrize("length", [97, 1000, 2 ** 31 - 1, -1])
def test_a_length_that_the_table_cannot_hold(length):
    """Counts as what the table holds (below zero: as nothing)."""
    cache, mass = filled([40, 96, 33])
    before, table, weights = contents(cache, 1, 96), cache.table.clone(), mass.clone()
    cache.lens[1] = length
    cache.granted.copy_(i32([0, 4, 0]))
    csd_cache_commit_path(cache, i32([1] * 3), i32([[0, 3, -1, -1]] * 3), mass=mass)
    torch.cuda.synchronize()
    now = 94 if length > 0 else 0
    assert cache.lens.tolist() == [40, now, 33] and torch.equal(cache.table, table)
    assert torch.equal(mass[[0, 2]], weights[[0, 2]])
    if now:
        order = list(range(93)) + [95]
        assert torch.equal(contents(cache, 1, 94), before[:, order])
        assert torch.equal(mass[1, :94], weights[1, order]) and not mass[1, 94:].any()


@pytest.mark.parametrize("length,keep", [(97, 50), (2 ** 31 - 1, 50), (1000, 96), (1000, 120), (-1, 50)])
def test_evicting_from_a_length_that_the_table_cannot_hold(length, keep):
    cache, mass = filled([40, 96, 33], seed=3)
    before, table, weights = contents(cache, 1, 96), cache.table.clone(), mass.clone()
    cache.lens[1] = length
    buf = EvictBuffers(cache, 120)
    csd_cache_evict(cache, mass, keep, buf, sinks=2, recent=10)
    torch.cuda.synchronize()
    n = 96 if length > 0 else 0
    where = O.evict(weights[1].tolist(), n, keep, 2, 10)
    assert cache.lens.tolist() == [40, len(where), 33] and buf.evicted.tolist() == [0, n - len(where), 0]
    assert buf.kept[1].tolist() == where + [-1] * (120 - len(where))
    want = weights.clone()
    if n:
        want[1] = 0.0
        want[1, :len(where)] = weights[1, where]
    assert torch.equal(mass, want) and torch.equal(contents(cache, 1, len(where)), before[:, where])
    held = -(-len(where) // 16) if n else 6
    assert torch.equal(cache.table[:, :held], table[:, :held]) and torch.equal(cache.table[[0, 2]], table[[0, 2]])
    assert cache.stats()["flags"] == 0
