"""csd_cache_commit_path: contents and bookkeeping after a tree's path has been kept, against lists of tokens (oracle/decode_oracle.py's
cache, oracle/tree_oracle.py's path).  Copies and whole numbers: equal."""

import numpy as np
import pytest
import torch

from oracle import decode_oracle as D
from oracle import tree_oracle as O
from paper_2604_13634_b200 import CsdError, PagedCache, csd_cache_commit, csd_cache_commit_path, csd_cache_extend, csd_cache_fork, csd_rope_append

pytestmark = pytest.mark.gpu

BAD_PATH = 0x20


def i32(x):
    return torch.tensor(np.asarray(x), dtype=torch.int32, device="cuda")


class Twin:
    """A cache and what its rows should hold: per row a list of tokens, a token a pair of [layers, heads, dim] tensors."""

    def __init__(self, rows, n_pages, page, layers, heads, dim, max_len, dtype=torch.bfloat16, token_major=False):
        self.cache = PagedCache(rows, n_pages, page, layers, heads, dim, dtype, max_len, token_major=token_major)
        self.books = D.Cache(rows, n_pages, page, self.cache.max_pages)
        self.rows = [[] for _ in range(rows)]
        self.gen = torch.Generator(device="cuda").manual_seed(page * dim + rows)

    def extend(self, T, news=None):
        news = [T] * len(self.rows) if news is None else news
        csd_cache_extend(self.cache, T, i32(news))
        self.books.extend(news)
        c = self.cache
        made = torch.randn(c.layers, len(self.rows), T, 3 * c.kv_heads, c.head_dim, generator=self.gen, device="cuda").to(c.dtype)
        for layer in range(c.layers):
            q, k, v = made[layer].split([c.kv_heads] * 3, dim=2)
            csd_rope_append(q, k, v, c, layer, None, n_new=c.granted)
        h = c.kv_heads
        for b, n in enumerate(self.books.granted):
            self.rows[b] += [(made[:, b, t, h:2 * h], made[:, b, t, 2 * h:]) for t in range(n)]

    def keep(self, accept, path):
        csd_cache_commit_path(self.cache, i32(accept), i32(path))
        bad = False
        for b, g in enumerate(self.books.granted):
            kept, short = O.kept_of_path(g, int(accept[b]), list(path[b]))
            bad |= short
            base = len(self.rows[b]) - g
            self.rows[b] = self.rows[b][:base] + [self.rows[b][base + i] for i in kept]
        self.books.truncate([len(x) for x in self.rows])
        return bad

    def check(self):
        c = self.cache
        assert c.lens.tolist() == [len(x) for x in self.rows] == self.books.lens
        assert np.array_equal(c.table.cpu().numpy(), self.books.table()) and c.refs.tolist() == self.books.refs()
        assert c.granted.tolist() == self.books.granted
        for b, tokens in enumerate(self.rows):
            if tokens:
                at = torch.arange(len(tokens), device="cuda")
                pages = c.table[b].long()[at // c.page_size]
                for which, pool in enumerate((c.k, c.v)):
                    got = pool[:, pages, :, at % c.page_size]                 # [n, layers, heads, dim]
                    assert torch.equal(got, torch.stack([t[which] for t in tokens])), b


def some_path(rng, T, n):
    """n ascending nodes, the root first, -1 behind them."""
    chosen = [0] + sorted(rng.choice(np.arange(1, T), n - 1, replace=False).tolist())
    return chosen + [-1] * (T - n)


@pytest.mark.parametrize("page,layers,heads,dim,dtype,token_major", [(16, 3, 2, 64, torch.bfloat16, False), (8, 2, 3, 72, torch.float16, True),
                                                                     (64, 1, 1, 256, torch.bfloat16, True), (32, 5, 4, 8, torch.bfloat16, False)])
@pytest.mark.parametrize("T", [1, 2, 26, 64])
def test_paths(T, page, layers, heads, dim, dtype, token_major):
    rng, rows = np.random.default_rng(T + page), 5
    x = Twin(rows, 100, page, layers, heads, dim, 500, dtype, token_major)
    x.extend(3, [0, 1, 2, 3, 3])
    csd_cache_commit(x.cache, i32([9] * rows))
    x.books.commit([9] * rows)
    for step in range(3):
        x.extend(T, [T, T, max(0, T - 1), T, 0] if step else None)
        lengths = [int(rng.integers(1, T + 1)) for _ in range(rows)]
        accept = [n - 1 for n in lengths]
        accept[1] = [-1, 2 ** 31 - 1, 0][step]                                # nothing, everything there is, the root alone
        path = [some_path(rng, T, n) for n in lengths]
        path[1] = list(range(T))
        path[2] = [min(t, max(0, T - 2)) if t >= 0 else t for t in path[2]]
        bad = x.keep(accept, path)
        x.check()
        assert (x.cache.stats()["flags"] == BAD_PATH) == bad or step            # the flag is sticky
    assert (x.cache.stats()["flags"] & ~BAD_PATH) == 0


def test_paths_that_are_none():
    x = Twin(6, 40, 16, 2, 2, 64, 200)
    x.extend(8)
    paths = [[0, 3, 2, 5, -1, -1, -1, -1], [0, 1, 1, 2, -1, -1, -1, -1], [-1] * 8, [2, 4, 8, 9, -1, -1, -1, -1], [7] * 8, [0, 1, 2, 3, 4, 5, 6, 7]]
    assert x.keep([3, 3, 2, 3, 0, 7], paths)
    x.check()
    assert x.cache.lens.tolist() == [2, 2, 0, 2, 1, 8] and x.cache.stats()["flags"] == BAD_PATH
    x.keep([3] * 6, paths)                                                        # nothing has been granted since
    x.check()


def test_shared_pages_and_a_graph():
    """Rows that continue one prompt: the path moves within the copies that the extension made.  The same calls captured and replayed."""
    x = Twin(4, 60, 16, 2, 2, 64, 300)
    x.extend(21, [21, 0, 0, 0])
    csd_cache_fork(x.cache, i32([0, 0, 0, 0]))
    x.books.fork([0, 0, 0, 0])
    x.rows = [list(x.rows[0]) for _ in range(4)]
    rng = np.random.default_rng(0)
    path, accept = [some_path(rng, 9, n) for n in (9, 4, 1, 5)], [8, 3, 0, 4]
    x.extend(9)
    x.keep(accept, path)
    x.check()
    dev_accept, dev_path = i32(accept), i32(path)
    graph, side = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.graph(graph, stream=side):
        csd_cache_commit_path(x.cache, dev_accept, dev_path)
    for _ in range(2):
        x.extend(9)
        new = [some_path(rng, 9, n) for n in (2, 9, 3, 1)]
        lengths = [1, 8, 2, 0]
        dev_accept.copy_(i32(lengths))
        dev_path.copy_(i32(new))
        graph.replay()
        for b, g in enumerate(x.books.granted):
            kept, _ = O.kept_of_path(g, lengths[b], new[b])
            base = len(x.rows[b]) - g
            x.rows[b] = x.rows[b][:base] + [x.rows[b][base + i] for i in kept]
        x.books.truncate([len(t) for t in x.rows])
        x.check()


def test_refusals():
    cache = PagedCache(2, 8, 16, 1, 1, 64, torch.bfloat16, 64)
    with pytest.raises(CsdError):
        csd_cache_commit_path(cache, i32([0, 0]), i32(np.zeros((2, 65))))
    for accept, path in ((i32([0]), i32(np.zeros((2, 3)))), (i32([0, 0]), i32(np.zeros((3, 3)))), (i32([0, 0]), i32(np.zeros((2, 3))).long())):
        with pytest.raises(AssertionError):
            csd_cache_commit_path(cache, accept, path)


@pytest.mark.parametrize("T", [1, 9, 64])
def test_masses_move_with_their_tokens(T):
    """Kept tokens' masses at their new places, zeros where tokens were dropped, everything else as it was; a stride of its own."""
    rng, rows = np.random.default_rng(T), 4
    x = Twin(rows, 60, 16, 1, 1, 64, 200)
    x.extend(5, [5, 0, 3, 1])
    csd_cache_commit(x.cache, i32([9] * rows))
    x.books.commit([9] * rows)
    news = [T, T, max(0, T - 2), 0]
    x.extend(T, news)
    lengths = [int(rng.integers(1, T + 1)) for _ in range(rows)]
    path, accept = [some_path(rng, T, n) for n in lengths], [n - 1 for n in lengths]
    lens = x.cache.lens.tolist()
    mass = torch.rand(rows, x.cache.max_pages * 16 + 3, device="cuda")
    before = mass.cpu().numpy().copy()
    csd_cache_commit_path(x.cache, i32(accept), i32(path), mass[:, :x.cache.max_pages * 16])
    for b, (n, g) in enumerate(zip(lens, news)):
        kept, _ = O.kept_of_path(g, accept[b], path[b])
        want = before[b].copy()
        want[n - g:n] = 0.0
        want[n - g:n - g + len(kept)] = before[b][[n - g + i for i in kept]]
        assert np.array_equal(mass[b].cpu().numpy(), want), b
    with pytest.raises(AssertionError):
        csd_cache_commit_path(x.cache, i32(accept), i32(path), mass[:, :40])
