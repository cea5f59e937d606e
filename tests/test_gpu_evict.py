"""csd_cache_evict against the rule taken one row and one place at a time (oracle/tree_oracle.py).  Choices, copies and bookkeeping: equal."""

import numpy as np
import pytest
import torch

from oracle import decode_oracle as D
from oracle import tree_oracle as O
from paper_2604_13634_b200 import CsdError, EvictBuffers, PagedCache, csd_cache_evict, csd_cache_extend, csd_cache_fork

pytestmark = pytest.mark.gpu

SHARED = 0x40


def i32(x):
    return torch.tensor(np.asarray(x), dtype=torch.int32, device="cuda")


def contents(cache, rows, lens):
    """Per row: keys and values of its tokens, [n, 2, layers, heads, dim]."""
    out = []
    for b in rows:
        at = torch.arange(lens[b], device="cuda")
        pages = cache.table[b].long()[at // cache.page_size]
        out.append(torch.stack([x[:, pages, :, at % cache.page_size] for x in (cache.k, cache.v)], dim=1))
    return out


def filled(seed, lens, page, layers, heads, dim, dtype=torch.bfloat16, token_major=False, places=None):
    rng = np.random.default_rng(seed)
    held = [-(-n // page) for n in lens]
    n_pages = sum(held) + 5
    cache = PagedCache(len(lens), n_pages, page, layers, heads, dim, dtype, places or max(1, max(held)) * page, token_major=token_major)
    table = np.full((len(lens), cache.max_pages), -1, dtype=np.int32)
    ids = rng.permutation(n_pages).tolist()
    for b, m in enumerate(held):
        table[b, :m], ids = ids[:m], ids[m:]
    gen = torch.Generator(device="cuda").manual_seed(seed)
    for x in (cache.k, cache.v):
        x.copy_(torch.randn(x.shape, generator=gen, device="cuda"))
    cache.load(torch.from_numpy(table).cuda(), i32(lens))
    return cache, table


def run_and_check(cache, table, lens, mass, keep, sinks, recent, width=None, keep_rows=None, stream=None):
    rows, page = len(lens), cache.page_size
    before, weights, whole = contents(cache, range(rows), lens), mass.cpu().numpy().copy(), (cache.k.clone(), cache.v.clone())
    buf = EvictBuffers(cache, keep if width is None else width)
    csd_cache_evict(cache, mass, keep if keep_rows is None else i32(keep_rows), buf, sinks=sinks, recent=recent, stream=stream)
    torch.cuda.synchronize()
    got_mass = mass.cpu().numpy()
    now, pages_written = [], set()
    for b, n in enumerate(lens):
        k = min(keep if keep_rows is None else keep_rows[b], buf.keep)
        where = O.evict(weights[b], n, k, sinks, recent)
        now.append(len(where))
        kept = buf.kept[b].tolist()
        assert kept == (where + [-1] * buf.keep)[:buf.keep], b
        assert int(buf.evicted[b]) == n - len(where), b
        want = weights[b].copy()
        want[:len(where)] = weights[b][where]
        want[len(where):n] = 0.0
        assert np.array_equal(got_mass[b], want, equal_nan=True), b
        pages_written |= {int(table[b, i // page]) for i, j in enumerate(where) if i != j}
    assert cache.lens.tolist() == now and cache.granted.tolist() == [0] * rows
    for b, got in enumerate(contents(cache, range(rows), now)):
        assert torch.equal(got, before[b][torch.tensor(O.evict(weights[b], lens[b], min(keep if keep_rows is None else keep_rows[b], buf.keep), sinks, recent),
                                                       dtype=torch.long, device="cuda")]), b
    books = D.Cache(rows, cache.n_pages, page, cache.max_pages)
    books.tables, books.lens = [[int(x) for x in table[b] if x >= 0] for b in range(rows)], list(lens)
    books.truncate(now)
    assert np.array_equal(cache.table.cpu().numpy(), books.table()) and cache.refs.tolist() == books.refs()
    untouched = torch.tensor([p not in pages_written for p in range(cache.n_pages)], device="cuda")
    assert all(torch.equal(x[:, untouched], y[:, untouched]) for x, y in zip((cache.k, cache.v), whole))
    return buf


def masses(seed, rows, places, kind="tail"):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    x = torch.randn(rows, places, generator=gen, device="cuda")
    if kind == "tail":
        return torch.exp(2 * x)
    if kind == "ties":
        return (x.abs() * 2).floor()
    if kind == "same":
        return torch.full_like(x, 0.25)
    x[:, ::7] = float("nan")                                          # "odd"
    x[:, 1::11] = float("inf")
    x[:, 2::13] = -float("inf")
    x[:, 3::5] = -0.0
    x[:, 4::5] = 0.0
    return x


@pytest.mark.parametrize("kind", ["tail", "ties", "same", "odd"])
@pytest.mark.parametrize("keep,sinks,recent", [(64, 4, 16), (100, 0, 0), (33, 40, 0), (33, 5, 50), (1, 0, 0), (0, 3, 3), (200, 199, 1), (97, 0, 90)])
def test_budgets(kind, keep, sinks, recent):
    lens = [0, 1, keep, keep + 1, 200, 201, 333, 1000, 47]
    cache, table = filled(keep, lens, 16, 2, 2, 64)
    mass = masses(keep, len(lens), cache.max_pages * 16, kind)
    run_and_check(cache, table, lens, mass, keep, sinks, recent)
    assert cache.stats()["flags"] == 0


@pytest.mark.parametrize("page,layers,heads,dim,dtype,token_major", [(8, 3, 2, 72, torch.float16, True), (256, 1, 1, 256, torch.bfloat16, False),
                                                                     (32, 2, 3, 8, torch.bfloat16, True), (64, 1, 4, 168, torch.float16, False)])
def test_layouts(page, layers, heads, dim, dtype, token_major):
    lens = [700, 64, 301, 1111]
    cache, table = filled(dim, lens, page, layers, heads, dim, dtype, token_major)
    run_and_check(cache, table, lens, masses(3, 4, cache.max_pages * page), 250, 4, 100)
    assert cache.stats()["flags"] == 0


@pytest.mark.parametrize("kind", ["tail", "ties", "same", "odd"])
def test_long_rows(kind):
    """Rows whose places eight blocks share, one among many that are short; budgets of their own."""
    lens = [40000, 300, 20011, 8193, 0]
    cache, table = filled(7, lens, 64, 1, 1, 64, places=40000)
    mass = masses(11, len(lens), cache.max_pages * 64 + 3, kind)[:, :cache.max_pages * 64]        # a stride of its own
    run_and_check(cache, table, lens, mass, 0, 16, 500, width=30000, keep_rows=[9000, 299, 20010, 50000, 7])
    assert cache.stats()["flags"] == 0


def test_shared_pages():
    """Rows that share a prompt: one whose moves would reach the shared pages stays as it is, one whose moves lie behind them does not."""
    cache = PagedCache(3, 60, 16, 2, 1, 64, torch.bfloat16, 320)
    csd_cache_extend(cache, 0, i32([100, 0, 50]))
    csd_cache_fork(cache, i32([0, 0, 2]))
    csd_cache_extend(cache, 100)                                       # rows 0 and 1 share 6 pages; the 7th was copied
    for x in (cache.k, cache.v):
        x.copy_(torch.randn(x.shape, device="cuda"))
    mass = torch.rand(3, cache.max_pages * 16, device="cuda")
    mass[1, :100] = 9.0                                                # nothing of the prompt leaves row 1
    before, lens = contents(cache, range(3), [200, 200, 150]), [200, 200, 150]
    buf = EvictBuffers(cache, 140)
    csd_cache_evict(cache, mass, 140, buf, sinks=2, recent=10)
    assert cache.stats()["flags"] == SHARED and cache.lens.tolist() == [200, 140, 140] and buf.evicted.tolist() == [0, 60, 10]
    assert buf.kept[0].tolist() == list(range(140))
    for b, got in enumerate(contents(cache, range(3), [200, 140, 140])):
        order = torch.arange(200, device="cuda") if b == 0 else buf.kept[b].long()
        assert torch.equal(got, before[b][order])
    shared = cache.refs.cpu()
    assert int((shared > 1).sum()) == 6 and lens == [200, 200, 150]


def test_again_and_in_a_graph():
    """Step after step in a captured graph, on a stream of its own: the cache grows by extensions and stays within its budget."""
    lens = [300, 310, 7]
    cache, table = filled(2, lens, 16, 1, 2, 64, places=600)
    mass, buf = masses(5, 3, cache.max_pages * 16), EvictBuffers(cache, 290)
    side, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph, stream=side):
        csd_cache_evict(cache, mass, 290, buf, sinks=4, recent=32)
    for step in range(4):
        n = cache.lens.tolist()
        before, weights = contents(cache, range(3), n), mass.cpu().numpy().copy()
        graph.replay()
        torch.cuda.synchronize()
        for b, got in enumerate(contents(cache, range(3), cache.lens.tolist())):
            where = O.evict(weights[b], n[b], 290, 4, 32)
            assert torch.equal(got, before[b][torch.tensor(where, dtype=torch.long, device="cuda")])
            assert np.array_equal(mass[b, :len(where)].cpu().numpy(), weights[b][where])
        csd_cache_extend(cache, 9)
        assert cache.granted.tolist() == [9] * 3
        mass[:, 280:320] = torch.rand(3, 40, device="cuda")
    assert cache.stats()["flags"] == 0


def test_pages_that_are_none():
    """A table with an id outside the pool: that token's move is skipped and flagged, everything else goes on."""
    cache, table = filled(4, [200], 16, 1, 1, 64)
    cache.table[0, 12] = 10 ** 6                                        # places 192 .. 199: recent ones
    mass, buf = masses(1, 1, cache.max_pages * 16), EvictBuffers(cache, 100)
    csd_cache_evict(cache, mass, 100, buf, recent=20)
    assert cache.stats()["flags"] == 4 and cache.lens.tolist() == [100]
    assert buf.kept[0].tolist()[80:] == list(range(180, 200))


def test_refusals():
    cache, _ = filled(1, [40, 40], 16, 1, 1, 64)
    mass, buf = torch.zeros(2, 48, device="cuda"), EvictBuffers(cache, 20)
    for kw in (dict(keep=21), dict(keep=-1), dict(keep=5, sinks=-1), dict(keep=5, recent=-1)):
        with pytest.raises(CsdError):
            csd_cache_evict(cache, mass, buf=buf, **kw)
    with pytest.raises(CsdError):
        EvictBuffers(cache, -1)
    for bad in (mass.double(), mass[:, :47], mass[:1], mass[:1].expand(2, 48), torch.zeros(2, 96, device="cuda")[:, ::2]):
        with pytest.raises(AssertionError):
            csd_cache_evict(cache, bad, 5, buf)
    with pytest.raises(CsdError, match="device"):
        csd_cache_evict(cache, mass.cpu(), 5, buf)
    other, _ = filled(1, [40, 40, 40], 16, 1, 1, 64)
    with pytest.raises(CsdError, match="another cache"):
        csd_cache_evict(other, torch.zeros(3, 48, device="cuda"), 5, buf)


def test_many_rows_and_layers():
    """More heads than the GPU has blocks for: a warp moves one of them; rows that lose nothing among those that do, an odd head size."""
    rng = np.random.default_rng(3)
    lens = [int(n) for n in rng.integers(30, 400, 40)]
    cache, table = filled(6, lens, 16, 8, 5, 24)
    run_and_check(cache, table, lens, masses(8, 40, cache.max_pages * 16, "ties"), 150, 4, 60)
    assert cache.stats()["flags"] == 0
