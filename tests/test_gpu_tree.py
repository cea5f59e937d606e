"""The tree form of the target pass on the GPU against its 64-bit statements (oracle/tree_oracle.py): masks and positions, storing at
positions, attention by masks.

Tolerances as for the chain (tests/test_gpu_decode.py): scores are D products summed in float32, at most 2 (D + 8) 2^-24 max_j sum_d
|scale q_d k_jd| =: e off; weights off by a factor 1 + 2 e + 2^-20 + n 2^-24, rounded to the cache's type (u: half a step, 2^-8 or 2^-11,
twice over for numerator and result's neighbourhood) and averaged over |v|; then u |out|.  lse: e + 2^-20 + n 2^-24 + 2^-22 |lse|.
"""

import numpy as np
import pytest
import torch

from oracle import decode_oracle as D
from oracle import tree_oracle as O
from paper_2604_13634_b200 import (AttentionBuffers, CsdError, PagedCache, RopePlan, TreePlan, csd_attention, csd_attention_tree, csd_cache_extend,
                                   csd_rope, csd_rope_append, csd_tree_plan)

pytestmark = pytest.mark.gpu

ULP = {torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}


def f64(t):
    return t.detach().cpu().to(torch.float64).numpy()


def gen_of(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def rand(gen, *shape, dtype=torch.bfloat16, scale=1.0):
    return (torch.randn(shape, generator=gen, device="cuda") * scale).to(dtype)


def i32(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def some_parents(rng, T):
    return [-1] + [int(rng.integers(max(0, t - 5), t)) for t in range(1, T)]


def as_i64(masks):
    return torch.tensor([[m - 2 ** 64 if m >= 2 ** 63 else m for m in row] for row in masks], dtype=torch.int64, device="cuda")


def filled(seed, lens, page, Hkv, dim, dtype, token_major=False, poison=None, layers=1):
    """A cache of these lengths over scattered pages; everything outside the rows' tokens is `poison`."""
    gen, rng = gen_of(seed), np.random.default_rng(seed)
    held = [-(-n // page) for n in lens]
    n_pages = sum(held) + 3
    shape = (layers, n_pages, page, Hkv, dim) if token_major else (layers, n_pages, Hkv, page, dim)
    k, v = rand(gen, *shape, dtype=dtype), rand(gen, *shape, dtype=dtype)
    if token_major:
        k, v = k.transpose(2, 3), v.transpose(2, 3)
    ids, table = rng.permutation(n_pages)[:sum(held)].tolist(), np.full((len(lens), max(1, max(held))), -1, dtype=np.int32)
    for b, m in enumerate(held):
        table[b, :m], ids = ids[:m], ids[m:]
    cache = PagedCache(len(lens), n_pages, page, layers, Hkv, dim, dtype, table.shape[1] * page, k=k, v=v)
    cache.load(torch.from_numpy(table).cuda(), i32(lens))
    if poison is not None:
        inside = torch.zeros(n_pages, page, dtype=torch.bool)
        for b, n in enumerate(lens):
            for j in range(n):
                inside[table[b, j // page], j % page] = True
        outside = ~inside.cuda()
        for x in (k, v):
            x.masked_fill_(outside[None, :, None, :, None], poison)
    return cache, table


def rows_of(cache, table, b, n, layer=0):
    return [D.rows_of(f64(x[layer]), table[b], n, cache.page_size) for x in (cache.k, cache.v)]


def check_row(out, lse, q, k, v, masks, n_new, scale, dtype):
    want, want_lse, reach, size = O.attention(f64(q), k, v, masks, n_new, scale)
    n, dim = k.shape[1], q.shape[2]
    e = 2 * (dim + 8) * 2.0 ** -24 * size
    rel = 2 * e + 2.0 ** -20 + n * 2.0 ** -24
    bound = (rel[..., None] + 2 * ULP[dtype]) * reach + ULP[dtype] * np.abs(want) + 1e-30 + (2.0 ** -24 if dtype == torch.float16 else 0)
    err = np.abs(f64(out) - want)
    assert (err <= bound).all(), float((err - bound).max())
    got = f64(lse)
    empty = want_lse == -np.inf
    assert (got[empty] == -np.inf).all() and (f64(out)[empty] == 0).all()
    fine = np.where(empty, 0.0, want_lse)
    assert (np.abs(np.where(empty, 0.0, got) - fine) <= e + 2.0 ** -20 + n * 2.0 ** -24 + 2.0 ** -22 * np.abs(fine)).all()


# ---- masks and positions ----

@pytest.mark.parametrize("T", [1, 2, 9, 31, 33, 63, 64])
def test_plan(T):
    rng = np.random.default_rng(T)
    rows = 7
    parents = np.array([some_parents(rng, T) for _ in range(rows)], dtype=np.int32)
    parents[1] = np.arange(T) - 1                                   # a chain
    parents[2] = 0                                                   # all below the root (which names itself)
    parents[3] = rng.integers(-3, T + 3, T)                          # anything: later nodes, none
    lens = [T, T + 5, 1000, 70, 0, T, 3]
    news = [T, T, max(1, T - 1), T, 0, 1, T + 100]                    # (the last: more new tokens than the row has)
    cache, _ = filled(T, lens, 16, 1, 64, torch.bfloat16)
    plan, offset = TreePlan(cache, T), i32([0, 10, -4, 5, 0, 2 ** 20, 7])
    csd_tree_plan(torch.from_numpy(parents).cuda(), cache, plan, n_new=i32(news), offset=offset)
    want = [O.plan(parents[b].tolist(), news[b], lens[b] - news[b], int(offset[b])) for b in range(rows)]
    assert torch.equal(plan.masks, as_i64([m for m, _ in want])) and plan.positions.tolist() == [p for _, p in want]
    wide = torch.full((rows, T + 3), -7, dtype=torch.int32, device="cuda")
    wide[:, 1:T + 1] = torch.from_numpy(parents).cuda()
    other = TreePlan(cache, T)
    csd_tree_plan(wide[:, 1:T + 1], cache, other, n_new=i32(news), offset=offset)
    assert torch.equal(other.masks, plan.masks) and torch.equal(other.positions, plan.positions)
    csd_tree_plan(torch.from_numpy(parents[0]).cuda(), cache, plan)
    one = O.plan(parents[0].tolist(), T, 0)
    assert torch.equal(plan.masks, as_i64([one[0]] * rows)) and plan.positions.tolist() == [[p + n - T for p in one[1]] for n in lens]
    csd_tree_plan(None, cache, plan)
    assert torch.equal(plan.masks, as_i64([[2 ** (t + 1) - 1 for t in range(T)]] * rows))


@pytest.mark.parametrize("layout,rot,dim", [("half", 64, 64), ("interleaved", 32, 80), ("half", 34, 72)])
def test_append_at_positions(layout, rot, dim):
    gen, T, rows = gen_of(dim), 7, 3
    cache = PagedCache(rows, 12, 16, 2, 2, dim, torch.bfloat16, 64)
    twin = PagedCache(rows, 12, 16, 2, 2, dim, torch.bfloat16, 64)
    plan = RopePlan(rot, layout=layout)
    qkv = rand(gen, rows, T, 8, dim)
    q, k, v = qkv.split([4, 2, 2], dim=2)
    positions = torch.randint(0, 100000, (rows, T), generator=gen, device="cuda", dtype=torch.int32)
    for c in (cache, twin):
        csd_cache_extend(c, T)
    got = csd_rope_append(q, k, v, cache, 1, plan, positions=positions)
    assert torch.equal(got, csd_rope(q.contiguous(), positions, plan))
    csd_rope_append(got, csd_rope(k.contiguous(), positions, plan), v, twin, 1, None)
    assert torch.equal(cache.k, twin.k) and torch.equal(cache.v, twin.v)
    places = torch.arange(T, dtype=torch.int32, device="cuda").expand(rows, T).contiguous()
    assert torch.equal(csd_rope_append(q, k, v, cache, 0, plan, positions=places), csd_rope_append(q, k, v, twin, 0, plan))
    assert torch.equal(cache.k[0], twin.k[0])


# ---- attention ----

CASES = [  # rows' lengths, T, query heads, key heads, dim, page
    ([1, 5, 40, 700], 1, 4, 2, 64, 16),
    ([9, 130, 64, 0, 65], 9, 2, 2, 128, 16),                          # 9 query rows to a key head
    ([16, 300, 63], 16, 2, 2, 80, 32),
    ([64, 65, 127, 128, 500], 5, 24, 2, 128, 64),                     # 60
    ([33, 1000], 33, 4, 2, 64, 16),                                   # 66
    ([64, 70, 3000], 64, 4, 1, 128, 128),                             # 256: two row tiles
    ([64, 129], 64, 2, 1, 256, 16),
    ([40, 200], 40, 10, 2, 96, 8),                                    # 200
    ([26, 26, 5000], 26, 3, 1, 72, 256),
]


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("lens,T,Hq,Hkv,dim,page", CASES)
def test_tree_attention(dtype, lens, T, Hq, Hkv, dim, page):
    rng = np.random.default_rng(len(lens) * T)
    cache, table = filled(T + dim, lens, page, Hkv, dim, dtype, token_major=dim in (64, 96), poison=float("nan"))
    q = rand(gen_of(dim), len(lens), T, Hq, dim, dtype=dtype, scale=1.5)
    news = [min(n, T if b % 2 == 0 else 1 + int(rng.integers(0, T))) for b, n in enumerate(lens)]
    plan, buf = TreePlan(cache, T), AttentionBuffers(cache, T, Hq, tree=True)
    parents = [some_parents(rng, T) for _ in lens]
    csd_tree_plan(i32(parents), cache, plan, n_new=i32(news))
    csd_attention_tree(q, cache, 0, buf, plan.masks, n_new=i32(news))
    for b, n in enumerate(lens):
        k, v = rows_of(cache, table, b, n)
        check_row(buf.out[b], buf.lse[b], q[b], k, v, O.plan(parents[b], news[b], 0)[0], news[b], dim ** -0.5, dtype)
    assert cache.stats()["flags"] == 0
    again = buf.out.clone()
    csd_attention_tree(q, cache, 0, buf, plan.masks, n_new=i32(news))
    assert torch.equal(again, buf.out)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("T,Hq,dim", [(8, 2, 64), (20, 4, 128), (64, 6, 128), (33, 1, 256), (64, 8, 128), (40, 4, 96)])
def test_any_masks(dtype, T, Hq, dim):
    """Bits at random, none at all, all, bits of tokens that do not exist; rows shorter than their new tokens, rows of new tokens alone."""
    rng = np.random.default_rng(T)
    lens, news = [T, T + 61, 200, 5, T // 2, 300], [T, T, T, 5, T, 300]
    cache, table = filled(3 * T, lens, 16, 1, dim, dtype, poison=float("inf"))
    masks = [[int(x) for x in rng.integers(0, 2 ** 63, T) * 2 + rng.integers(0, 2, T)] for _ in lens]
    masks[0] = [0 if t % 3 == 0 else 2 ** 64 - 1 for t in range(T)]
    masks[1][0], masks[2][T - 1], masks[2][0] = 0, 2 ** 64 - 1, 0
    masks[3] = [2 ** 63 | 2 ** 4] * T                                  # a token beyond the last, and the last
    q = rand(gen_of(T), len(lens), T, Hq, dim, dtype=dtype)
    buf = AttentionBuffers(cache, T, Hq, tree=True)
    csd_attention_tree(q, cache, 0, buf, as_i64(masks), n_new=i32(news), scale=0.3)
    for b, n in enumerate(lens):
        k, v = rows_of(cache, table, b, n)
        check_row(buf.out[b], buf.lse[b], q[b], k, v, masks[b], news[b], 0.3, dtype)


@pytest.mark.parametrize("T,Hq", [(8, 2), (40, 3), (64, 4)])
def test_what_a_node_does_not_see_does_not_reach_it(T, Hq):
    """Infinities and NaN in the keys and values of one branch: the other branch keeps its bits, the nodes below get them."""
    cache, table = filled(T, [T + 150, T], 16, 1, 128, torch.bfloat16)
    rng = np.random.default_rng(1)
    parents = [-1, 0, 0] + [int(rng.integers(1, t)) for t in range(3, T)]
    masks = O.plan(parents, T, 0)[0]
    q, buf, plan = rand(gen_of(4), 2, T, Hq, 128), AttentionBuffers(cache, T, Hq, tree=True), TreePlan(cache, T)
    csd_tree_plan(i32(parents), cache, plan)
    csd_attention_tree(q, cache, 0, buf, plan.masks)
    clean = buf.out.clone()
    for what, value in (("v", float("inf")), ("v", float("nan")), ("k", float("nan"))):
        for b, n in enumerate((T + 150, T)):
            place = n - T + 2                                          # node 2
            getattr(cache, what)[0, table[b, place // 16], 0, place % 16, 5] = value
        csd_attention_tree(q, cache, 0, buf, plan.masks)
        below = torch.tensor([m >> 2 & 1 for m in masks], dtype=torch.bool, device="cuda")
        assert torch.equal(buf.out[:, ~below], clean[:, ~below])
        assert not torch.isfinite(buf.out[:, below, :, 5]).any()
        for b, n in enumerate((T + 150, T)):
            place = n - T + 2
            getattr(cache, what)[0, table[b, place // 16], 0, place % 16, 5] = 1.0


def test_masks_of_a_chain_give_the_chain():
    lens, T, Hq = [700, 64, 9, 30, 0], 9, 8
    for heads in (8, 40):
        cache, _ = filled(5, lens, 16, 4, 128, torch.bfloat16)
        q, plan = rand(gen_of(6), len(lens), T, heads, 128), TreePlan(cache, T)
        csd_tree_plan(None, cache, plan)
        a, b = AttentionBuffers(cache, T, heads), AttentionBuffers(cache, T, heads, tree=True)
        assert torch.equal(csd_attention(q, cache, 0, a), csd_attention_tree(q, cache, 0, b, plan.masks)) and torch.equal(a.lse, b.lse)


def test_tree_refusals():
    cache, _ = filled(1, [70], 16, 1, 64, torch.bfloat16)
    with pytest.raises(CsdError):
        TreePlan(cache, 65)
    with pytest.raises(CsdError):
        AttentionBuffers(cache, 65, 1, tree=True)
    with pytest.raises(CsdError):
        AttentionBuffers(cache, 34, 1)                                 # a chain's limit stays what it was
    buf, q = AttentionBuffers(cache, 3, 1, tree=True), rand(gen_of(1), 1, 3, 1, 64)
    for masks in (torch.zeros(1, 3, dtype=torch.int32, device="cuda"), torch.zeros(1, 4, dtype=torch.int64, device="cuda"),
                  torch.zeros(1, 3, dtype=torch.int64)):
        with pytest.raises(AssertionError):
            csd_attention_tree(q, cache, 0, buf, masks)
    with pytest.raises(AssertionError):
        csd_tree_plan(i32([[0, 1]]), cache, TreePlan(cache, 3))
    with pytest.raises(CsdError, match="device"):
        csd_tree_plan(torch.zeros(3, dtype=torch.int32), cache, TreePlan(cache, 3))
