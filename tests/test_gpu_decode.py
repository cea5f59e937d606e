"""The decode-pass operators on the GPU against their 64-bit statements (oracle/decode_oracle.py).

Tolerances.  u = half a unit in the last place of the output's type, relative (2^-9 bf16, 2^-12 f16, 2^-25 f32, doubled
below so that a result next to a rounding boundary may fall either way).
  rope       float32 work: angle rounded to 2^-25 of a half turn (1e-7 rad), sine and cosine to 2 ulp, two products and
             a sum: at most 8e-7 (|x0| + |x1|) m per element, then u |y|.
  attention  scores: D products summed in float32, at most 2 (D + 8) 2^-24 max_j sum_d |scale q_d k_jd| =: e; weights
             off by a factor 1 + 2 e (numerator, sum) + 2^-20 (exponential) + n 2^-24 (the sum of n of them), rounded to the
             cache's type (u) and averaged over |v|; then u |out|.  lse: e + 2^-20 + n 2^-24 + 2^-22 |lse|.
"""

import ctypes
import math

import numpy as np
import pytest
import torch

from oracle import decode_oracle as O
from paper_2604_13634_b200 import (AttentionBuffers, PagedCache, RopePlan, StepBuffers, csd_attention, csd_cache_commit, csd_cache_compact,
                                   csd_cache_extend, csd_cache_fork, csd_cache_truncate, csd_rope, csd_rope_append, decode)

pytestmark = pytest.mark.gpu

ULP = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}
TINY = {torch.float32: 1e-37, torch.bfloat16: 1e-37, torch.float16: 2.0 ** -24}     # spacing of the smallest values


def f64(t):
    return t.detach().cpu().to(torch.float64).numpy()


def rand(gen, *shape, dtype=torch.bfloat16, scale=1.0):
    return (torch.randn(shape, generator=gen, device="cuda") * scale).to(dtype)


def gen_of(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


# ---- rotary positions ----

def check_rope(y, x, positions, plan, th, dtype, inverse=False):
    want = O.rope(f64(x), f64(positions), th, plan.magnitude, plan.layout, inverse)
    mag = O.rope(np.abs(f64(x)), np.zeros(positions.shape), th, 1.0, plan.layout)      # |x| where it lies
    rot, pair = plan.rot, mag.copy()
    a, b = (slice(0, rot // 2), slice(rot // 2, rot)) if plan.layout == "half" else (slice(0, rot, 2), slice(1, rot, 2))
    pair[..., a] = pair[..., b] = mag[..., a] + mag[..., b]
    bound = 8e-7 * pair * max(1.0, plan.magnitude) + ULP[dtype] * np.abs(want) + TINY[dtype]
    bound[..., rot:] = 0
    err = np.abs(f64(y) - want)
    assert (err <= bound).all(), float((err - bound).max())


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16, torch.float16])
@pytest.mark.parametrize("layout", ["half", "interleaved"])
@pytest.mark.parametrize("B,S,H,D,rot,scaling", [(2, 5, 3, 64, 64, "none"), (1, 1, 1, 128, 128, "parts"), (3, 7, 5, 80, 32, "yarn"),
                                                 (2, 3, 4, 72, 34, "linear"), (1, 4, 2, 7, 6, "base"), (1, 2, 9, 256, 2, "none"),
                                                 (2, 33, 8, 96, 96, "base"), (2, 3, 3, 168, 66, "none"), (1, 2, 2, 601, 70, "linear"), (2, 2, 7, 1024, 1002, "parts"),
                                                 (1, 3, 2, 4104, 4096, "none"), (2, 40, 1, 8, 2, "none")])
def test_rope(dtype, layout, B, S, H, D, rot, scaling):
    gen = gen_of(1)
    x = rand(gen, B, S, H, D, dtype=dtype, scale=2.0)
    pos = torch.randint(-5, 300000, (B, S), generator=gen, device="cuda", dtype=torch.int32)
    plan = RopePlan(rot, layout=layout, scaling=scaling, factor=8.0 if scaling != "none" else 1.0)
    th, m = O.thetas(rot, scaling=scaling, factor=8.0)
    y = csd_rope(x, pos, plan)
    check_rope(y, x, pos, plan, th, dtype)
    back = csd_rope(x, pos, plan, inverse=True)
    check_rope(back, x, pos, plan, th, dtype, inverse=True)
    z = x.clone()
    assert csd_rope(z, pos, plan, out=z) is z and torch.equal(z, y)                    # in place
    # slices of a wider tensor, of tokens-last order, and at an odd element offset: the same numbers, nothing else touched
    wide = torch.full((B, S, H + 2, D + 3), 7.0, device="cuda", dtype=dtype)
    for off in (0, 3):
        src, dst = wide.clone(), wide.clone()
        src[:, :, 1:H + 1, off:off + D] = x
        csd_rope(src[:, :, 1:H + 1, off:off + D], pos, plan, out=dst[:, :, 1:H + 1, off:off + D])
        assert torch.equal(dst[:, :, 1:H + 1, off:off + D], y)
        dst[:, :, 1:H + 1, off:off + D] = 7.0
        assert torch.equal(dst, wide)
    turned = x.permute(2, 0, 1, 3).contiguous().permute(1, 2, 0, 3)
    assert torch.equal(csd_rope(turned, pos, plan), y)
    shared = csd_rope(x, pos[0].contiguous(), plan)                                     # positions of a whole batch
    assert torch.equal(shared[0], y[0])
    check_rope(shared, x, pos[:1].expand(B, S), plan, th, dtype)


def test_rope_far_positions_and_empty_shapes():
    gen = gen_of(2)
    x = rand(gen, 1, 4, 2, 64, dtype=torch.float32)
    pos = torch.tensor([[2 ** 31 - 1, 2 ** 30 + 1, -2 ** 31, 16777217]], device="cuda", dtype=torch.int32)
    plan = RopePlan(64)
    th, _ = O.thetas(64)
    # the oracle's own product p theta is exact to 2^-53 p theta = 2.4e-7 rad here: as much as the kernel's bound, so both are granted
    want, got = O.rope(f64(x), f64(pos), th), f64(csd_rope(x, pos, plan))
    assert np.abs(got - want).max() <= (8e-7 + 2.5e-7) * 2 * np.abs(f64(x)).max() + 2.0 ** -23 * np.abs(want).max()
    for shape in ((0, 3, 2, 64), (2, 0, 2, 64), (2, 3, 0, 64)):
        e = torch.empty(shape, device="cuda")
        assert csd_rope(e, torch.zeros(shape[:2], device="cuda", dtype=torch.int32), plan).shape == shape


def test_rope_gradient_against_differences():
    gen = gen_of(3)
    plan = RopePlan(32, layout="interleaved", scaling="yarn", factor=4.0)
    x, g = rand(gen, 1, 3, 2, 40, dtype=torch.float32), rand(gen, 1, 3, 2, 40, dtype=torch.float32)
    pos = torch.tensor([[0, 17, 4097]], device="cuda", dtype=torch.int32)
    grad = f64(csd_rope(g, pos, plan, inverse=True))
    # the operation is linear: a difference over a step of 1 has no truncation error, only rounding (8e-7 per element
    # and value, |g| <= 5, 40 elements of which 2 move)
    for at in [(0, 0, 0, 0), (0, 1, 1, 31), (0, 2, 0, 30), (0, 2, 1, 39)]:
        e = torch.zeros_like(x)
        e[at] = 1.0
        d = float(((csd_rope(x + e, pos, plan) - csd_rope(x - e, pos, plan)).double() * g.double()).sum()) / 2
        assert abs(d - grad[at]) <= 4e-5


# ---- caches in known states ----

def filled_cache(seed, lens, page, Hkv, D, dtype, token_major, layers=1, extra=3, max_len=None, poison=None):
    """A cache whose rows hold random tokens in scattered pages; unused places hold `poison` (stale values otherwise)."""
    gen, host = gen_of(seed), np.random.default_rng(seed)
    rows, need = len(lens), sum(-(-n // page) for n in lens)
    n_pages = need + extra
    cache = PagedCache(rows, n_pages, page, layers, Hkv, D, dtype, max_len or max(1, max(lens)), token_major=token_major)
    for pool in (cache.k, cache.v):
        pool.copy_(rand(gen, *pool.shape, dtype=dtype))
    ids, at = host.permutation(n_pages), 0
    table = torch.full((rows, cache.max_pages), -1, dtype=torch.int32)
    used = torch.zeros(n_pages, page, dtype=torch.bool)
    for r, n in enumerate(lens):
        m = -(-n // page)
        table[r, :m] = torch.from_numpy(ids[at:at + m].astype(np.int32))
        for i in range(m):
            used[ids[at + i], :min(page, n - i * page)] = True
        at += m
    if poison is not None:
        for pool in (cache.k, cache.v):
            bad = torch.full_like(pool, poison)
            bad[..., ::2] = math.nan
            pool.copy_(torch.where(used.cuda()[None, :, None, :, None], pool, bad))
    cache.load(table.cuda(), torch.tensor(lens, dtype=torch.int32).cuda())
    return cache, gen


# ---- turn and store ----

@pytest.mark.parametrize("dtype,token_major,layout,D,rot,T,Hq,Hkv,page,ragged", [
    (torch.bfloat16, False, "half", 128, 128, 1, 32, 8, 16, False), (torch.bfloat16, True, "interleaved", 64, 64, 5, 6, 2, 8, True),
    (torch.float16, True, "half", 80, 32, 9, 4, 4, 32, True), (torch.float16, False, "interleaved", 96, 90, 3, 5, 1, 64, False),
    (torch.bfloat16, True, "half", 256, 250, 33, 2, 1, 256, True), (torch.bfloat16, False, "half", 8, 2, 2, 3, 3, 128, False)])
def test_rope_append(dtype, token_major, layout, D, rot, T, Hq, Hkv, page, ragged):
    lens = [0, 1, page, page + 1, 2 * page + T, 300]
    news = [min(n, i % (T + 1)) for i, n in enumerate(lens)] if ragged else [T] * len(lens)
    cache, gen = filled_cache(5, lens, page, Hkv, D, dtype, token_major, layers=2)
    plan = RopePlan(rot, layout=layout, scaling="parts", factor=8.0)
    th, _ = O.thetas(rot, scaling="parts", factor=8.0)
    qkv = rand(gen, len(lens), T, Hq + 2 * Hkv, D, dtype=dtype)
    q, k, v = qkv.split([Hq, Hkv, Hkv], dim=2)
    k0, v0 = cache.k.clone(), cache.v.clone()
    n_new = torch.tensor(news, dtype=torch.int32, device="cuda") if ragged else None
    out = csd_rope_append(q, k, v, cache, 1, plan, n_new=n_new)
    want_k, want_v = k0.clone(), v0.clone()
    place = torch.zeros(len(lens), T, dtype=torch.int32)
    table = cache.table.cpu().numpy()
    for b, n in enumerate(lens):
        for t in range(T):
            at = n - news[b] + t
            if t < news[b] and at >= 0:
                place[b, t] = at
                page_id = int(table[b, at // page])
                y = cache.k[1, page_id, :, at % page]
                check_rope(y[None], k[b, t][None], torch.tensor([at]), plan, th, dtype)
                want_k[1, page_id, :, at % page] = y
                want_v[1, page_id, :, at % page] = v[b, t]
                check_rope(out[b, t][None], q[b, t][None], torch.tensor([at]), plan, th, dtype)
            else:
                assert not out[b, t].any()
    assert torch.equal(cache.k, want_k) and torch.equal(cache.v, want_v)              # nothing else was touched
    # no rotation; and in place
    dense = q.contiguous()
    assert csd_rope_append(dense, k, v, cache, 0, None, q_out=dense, n_new=n_new) is dense
    for b in range(len(lens)):
        for t in range(T):
            real = t < news[b] and lens[b] - news[b] + t >= 0
            assert torch.equal(dense[b, t], q[b, t]) if real else not dense[b, t].any()
    assert cache.stats()["flags"] == 0


def test_a_table_with_an_id_outside_the_pool_is_flagged_and_skipped():
    cache, gen = filled_cache(6, [20, 20], 16, 2, 64, torch.bfloat16, False)
    k0 = cache.k.clone()
    cache.table[0, 1] = cache.n_pages
    q, k = rand(gen, 2, 1, 2, 64), rand(gen, 2, 1, 2, 64)
    csd_rope_append(q, k, k, cache, 0, None)
    assert cache.stats()["flags"] == decode.CACHE_BAD_PAGE
    at = int(cache.table[1, 1])
    k0[0, at, :, 3] = k[1, 0]
    assert torch.equal(cache.k, k0)
    buf = AttentionBuffers(cache, 1, 2)
    csd_attention(q, cache, 0, buf)                                  # reads nothing outside the pool; row 1 is right
    out, lse, reach, size = O.attention(f64(q[1]), O.rows_of(f64(cache.k[0]), cache.table[1].tolist(), 20, 16),
                                        O.rows_of(f64(cache.v[0]), cache.table[1].tolist(), 20, 16), 1, 1 / 8)
    assert np.abs(f64(buf.out[1]) - out).max() <= 0.05 and cache.stats()["flags"] == decode.CACHE_BAD_PAGE


# ---- attention ----

def check_attention(buf, q, cache, lens, news, scale, layer=0, rows=None):
    dtype, D, page = cache.dtype, cache.head_dim, cache.page_size
    u, table = ULP[dtype], cache.table.cpu().numpy()
    kp, vp, got, lse_got, q = f64(cache.k[layer]), f64(cache.v[layer]), f64(buf.out), f64(buf.lse), f64(q)
    for b in range(len(lens)) if rows is None else rows:
        k, v = O.rows_of(kp, table[b], lens[b], page), O.rows_of(vp, table[b], lens[b], page)
        out, lse, reach, size = O.attention(q[b], k, v, news[b], scale)
        e = 2 * (D + 8) * 2.0 ** -24 * size
        w = (2 * e + 2.0 ** -20 + lens[b] * 2.0 ** -24)[..., None]
        bound = (u + w) * reach + u * np.abs(out) + TINY[dtype]
        err = np.abs(got[b] - out)
        assert (err <= bound).all(), (b, float((err - bound).max()), float(err.max()))
        seen = np.isfinite(lse)
        assert np.array_equal(np.isneginf(lse_got[b]), ~seen)
        dl = np.abs(lse_got[b][seen] - lse[seen])
        assert (dl <= (e + 2.0 ** -20 + lens[b] * 2.0 ** -24)[seen] + 2.0 ** -22 * np.abs(lse[seen])).all(), (b, float(dl.max()))


CASES = [  # dtype, token_major, page, Hq, Hkv, D, T, lens
    (torch.bfloat16, False, 16, 4, 2, 64, 1, [1, 0, 15, 16, 17, 63, 64, 65, 127, 129]),
    (torch.bfloat16, False, 16, 32, 8, 128, 1, [700]),
    (torch.bfloat16, True, 64, 8, 2, 128, 5, [0, 3, 64, 700, 1300]),
    (torch.float16, True, 32, 16, 16, 64, 1, [0, 2, 31, 500, 1024]),
    (torch.float16, False, 8, 6, 2, 80, 3, [7, 8, 9, 100]),
    (torch.bfloat16, False, 128, 40, 8, 128, 6, [1, 129, 2000]),
    (torch.bfloat16, False, 16, 64, 8, 128, 9, [33, 1500, 8]),
    (torch.bfloat16, True, 256, 3, 1, 256, 2, [256, 257, 900]),
    (torch.float16, False, 16, 16, 2, 256, 9, [50, 0, 333]),
    (torch.bfloat16, False, 16, 16, 1, 96, 33, [20, 33, 34, 1000]),
    (torch.bfloat16, False, 32, 5, 5, 8, 4, [3, 40, 100]),
    (torch.float16, True, 16, 24, 2, 64, 16, [16, 15, 2100]),
    (torch.bfloat16, False, 16, 7, 7, 128, 1, [5000, 3, 2500, 0, 0, 1, 4999]),
    (torch.bfloat16, False, 64, 32, 1, 64, 1, [9000]),
]


@pytest.mark.parametrize("case", range(len(CASES)))
@pytest.mark.parametrize("ragged", [False, True])
def test_attention(case, ragged):
    dtype, token_major, page, Hq, Hkv, D, T, lens = CASES[case]
    news = [(2 * i + 1) % (T + 1) for i in range(len(lens))] if ragged else [T] * len(lens)
    cache, gen = filled_cache(10 + case, lens, page, Hkv, D, dtype, token_major, layers=2)
    q = rand(gen, len(lens), T, Hq, D, dtype=dtype, scale=2.0)
    buf = AttentionBuffers(cache, T, Hq)
    n_new = torch.tensor(news, dtype=torch.int32, device="cuda") if ragged else None
    csd_attention(q, cache, 1, buf, n_new=n_new)
    check_attention(buf, q, cache, lens, news, 1 / math.sqrt(D), layer=1)
    first, first_lse = buf.out.clone(), buf.lse.clone()
    for _ in range(3):                                                # the workspace is left ready; results repeat bit for bit
        csd_attention(q, cache, 1, buf, n_new=n_new)
        assert torch.equal(buf.out, first) and torch.equal(buf.lse, first_lse)
    # a strided query, another scale, without lse
    wide = torch.zeros(len(lens), T, Hq + 1, D + 8, device="cuda", dtype=dtype)
    wide[:, :, :Hq, 8:] = q
    csd_attention(wide[:, :, :Hq, 8:], cache, 1, buf, scale=-0.3, n_new=n_new)
    check_attention(buf, q, cache, lens, news, -0.3, layer=1)
    assert cache.stats()["flags"] == 0


@pytest.mark.parametrize("poison", [math.inf, -math.inf, math.nan])
@pytest.mark.parametrize("dtype,Hq,Hkv,D,T,page", [(torch.bfloat16, 4, 2, 128, 1, 16), (torch.float16, 8, 1, 64, 9, 32), (torch.bfloat16, 8, 2, 256, 5, 64),
                                                   (torch.bfloat16, 16, 2, 128, 9, 16), (torch.bfloat16, 32, 2, 64, 9, 256)])
def test_unseen_places_never_reach_a_result(poison, dtype, Hq, Hkv, D, T, page):
    """Stale infinities and NaN beyond a row's length, in free pages, and in the keys and values of later new tokens."""
    lens = [1, 5, 17, 40, 64, 100, 130, 0]
    cache, gen = filled_cache(40, lens, page, Hkv, D, dtype, False, poison=poison)
    q = rand(gen, len(lens), T, Hq, D, dtype=dtype, scale=2.0)
    buf = AttentionBuffers(cache, T, Hq)
    csd_attention(q, cache, 0, buf)
    check_attention(buf, q, cache, lens, [T] * len(lens), 1 / math.sqrt(D))
    if T == 1:
        return
    clean, clean_lse = buf.out.clone(), buf.lse.clone()
    for b, n in enumerate(lens):                                      # the last new token of every row
        if n:
            page_id = int(cache.table[b, (n - 1) // page])
            cache.k[0, page_id, :, (n - 1) % page] = poison
            cache.v[0, page_id, :, (n - 1) % page] = poison
    csd_attention(q, cache, 0, buf)
    assert torch.equal(buf.out[:, :T - 1], clean[:, :T - 1]) and torch.equal(buf.lse[:, :T - 1], clean_lse[:, :T - 1])
    assert not torch.isfinite(buf.out[:7, T - 1].float()).all(-1).any()   # the token that sees it shows it


def test_extreme_scores():
    """Scores far apart and far from zero: one place takes everything; the sum of exponentials never overflows."""
    cache, gen = filled_cache(41, [200, 70], 16, 2, 64, torch.bfloat16, False)
    q = rand(gen, 2, 3, 4, 64, scale=300.0)
    buf = AttentionBuffers(cache, 3, 4)
    csd_attention(q, cache, 0, buf)
    check_attention(buf, q, cache, [200, 70], [3, 3], 1 / 8)
    csd_attention(q, cache, 0, buf, scale=0.0)                        # all scores equal: the mean
    check_attention(buf, q, cache, [200, 70], [3, 3], 0.0)


def test_attention_on_a_stream_of_its_own_and_in_a_graph():
    lens = [300, 5, 1000]
    cache, gen = filled_cache(42, lens, 16, 2, 128, torch.bfloat16, False)
    q = rand(gen, 3, 5, 8, 128)
    buf, ref = AttentionBuffers(cache, 5, 8), AttentionBuffers(cache, 5, 8)
    csd_attention(q, cache, 0, ref)
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    csd_attention(q, cache, 0, buf, stream=s)
    s.synchronize()
    assert torch.equal(buf.out, ref.out) and torch.equal(buf.lse, ref.lse)
    buf.out.zero_()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        csd_attention(q, cache, 0, buf)
    for _ in range(3):
        g.replay()
    torch.cuda.synchronize()
    assert torch.equal(buf.out, ref.out)
    # a graph follows lengths that change on the device
    csd_cache_truncate(cache, torch.tensor([100, 0, 999], dtype=torch.int32, device="cuda"))
    g.replay()
    csd_attention(q, cache, 0, ref)
    assert torch.equal(buf.out, ref.out)
    check_attention(buf, q, cache, [100, 0, 999], [5] * 3, 1 / math.sqrt(128))


def test_one_workspace_serves_other_shapes():
    big, gen = filled_cache(43, [4000, 10, 900, 64], 16, 2, 128, torch.bfloat16, False)
    small, _ = filled_cache(44, [3000], 16, 1, 64, torch.float16, False)
    buf, other = AttentionBuffers(big, 9, 16), AttentionBuffers(small, 1, 4)
    other.workspace, other.ws_bytes = buf.workspace, max(buf.ws_bytes, other.ws_bytes)
    if other.ws_bytes > buf.ws_bytes:
        pytest.skip("the second shape wants more")
    qb, qs = rand(gen, 4, 9, 16, 128), rand(gen, 1, 1, 4, 64, dtype=torch.float16)
    for _ in range(3):
        csd_attention(qb, big, 0, buf)
        csd_attention(qs, small, 0, other)
        check_attention(other, qs, small, [3000], [1], 1 / 8)
        check_attention(buf, qb, big, [4000, 10, 900, 64], [9] * 4, 1 / math.sqrt(128))


def test_offsets_beyond_32_bits():
    """A pool of more than 2^32 bytes and 2^31 elements per tensor; the row's pages lie at its far end."""
    n_pages, page, Hkv, D = 33000, 256, 2, 128
    k = torch.empty(1, n_pages, Hkv, page, D, dtype=torch.bfloat16, device="cuda")
    assert k.numel() > 2 ** 31
    v = torch.empty_like(k)
    k.fill_(math.nan), v.fill_(math.nan)
    gen = gen_of(45)
    table = torch.tensor([[n_pages - 1, 0, n_pages - 2], [n_pages - 3, -1, -1]], dtype=torch.int32)
    for p in table.flatten().tolist():
        if p >= 0:
            k[0, p], v[0, p] = rand(gen, Hkv, page, D), rand(gen, Hkv, page, D)
    cache = PagedCache(2, n_pages, page, 1, Hkv, D, torch.bfloat16, 4 * page, k=k, v=v)
    lens = [600, 256]
    cache.load(table.cuda(), torch.tensor(lens, dtype=torch.int32).cuda())
    new = rand(gen, 2, 2, Hkv, D)
    q = rand(gen, 2, 2, 4, D)
    csd_rope_append(q, new, new, cache, 0, None)
    buf = AttentionBuffers(cache, 2, 4)
    csd_attention(q, cache, 0, buf)
    for b in range(2):
        ids = table[b][table[b] >= 0].long()
        kk, vv = (f64(x[0, ids]).transpose(1, 0, 2, 3).reshape(Hkv, -1, D)[:, :lens[b]] for x in (k, v))
        assert np.array_equal(kk[:, -2:], f64(new[b]).transpose(1, 0, 2))
        out, lse, reach, size = O.attention(f64(q[b]), kk, vv, 2, 1 / math.sqrt(D))
        assert np.abs(f64(buf.out[b]) - out).max() <= 2.0 ** -7 * reach.max() and np.abs(f64(buf.lse[b]) - lse).max() < 1e-4
    csd_cache_fork(cache, torch.tensor([0, 0], dtype=torch.int32, device="cuda"))
    csd_cache_extend(cache, 1)                                        # row 0 copies the shared page n_pages - 2
    assert cache.table[0].tolist()[:3] == [n_pages - 1, 0, 1] and torch.equal(cache.k[0, 1], cache.k[0, n_pages - 2])
    csd_cache_compact(cache)
    assert sorted(set(cache.table.flatten().tolist())) == [-1, 0, 1, 2, 3] and torch.equal(cache.v[0, 2], v[0, n_pages - 2])


# ---- pages ----

def check_pages(cache, c):
    assert cache.table.cpu().numpy().tolist() == c.table().tolist()
    assert cache.lens.tolist() == c.lens and cache.refs.tolist() == c.refs() and cache.granted.tolist() == c.granted
    lay = decode.CacheLayout()
    decode._lib().csd_cache_meta_layout(cache.rows, cache.max_pages, cache.n_pages, ctypes.byref(lay))
    words = cache.meta[lay.free_bits // 4:lay.free_bits // 4 + -(-cache.n_pages // 32)].cpu().numpy().view(np.uint32)
    bits = [(int(words[p // 32]) >> (p % 32)) & 1 for p in range(32 * len(words))]
    assert bits == [int(n == 0) for n in c.refs()] + [0] * (32 * len(words) - cache.n_pages)


@pytest.mark.parametrize("rows,n_pages,page,max_len,layers,Hkv,D,token_major", [
    (1, 3, 8, 40, 1, 1, 8, False), (5, 40, 16, 100, 2, 2, 64, False), (33, 200, 8, 120, 1, 1, 16, True), (1100, 3000, 8, 64, 1, 1, 8, False),
    (4096, 9000, 8, 32, 1, 1, 8, True), (7, 100000, 16, 200000, 1, 1, 8, False)])
def test_page_operations_follow_the_rules(rows, n_pages, page, max_len, layers, Hkv, D, token_major):
    host = np.random.default_rng(rows + n_pages)
    cache = PagedCache(rows, n_pages, page, layers, Hkv, D, torch.bfloat16, max_len, token_major=token_major)
    c = O.Cache(rows, n_pages, page, cache.max_pages)
    stamp = torch.arange(layers * n_pages, device="cuda").view(layers, n_pages, 1, 1, 1)
    cache.k.copy_(((stamp * 7) % 251).expand(cache.k.shape))
    cache.v.copy_(((stamp * 5) % 241).expand(cache.v.shape))
    want = [cache.k.cpu().clone(), cache.v.cpu().clone()]
    dev = lambda a: torch.tensor(np.asarray(a), dtype=torch.int32, device="cuda")  # noqa: E731
    big = n_pages // (3 * rows) * page
    for step in range(14 if rows < 1000 else 8):
        kind = step % 7
        if kind in (0, 2, 4):
            news = [int(x) for x in host.integers(-1, min(max_len // 2, max(big, 3 * page)) + 2, rows)]
            uniform = kind == 4
            if uniform:
                news = [3] * rows
            moves = c.extend(news)
            csd_cache_extend(cache, 3, None if uniform else dev(news))
        elif kind == 1:
            accept = [int(x) for x in host.integers(-2, 6, rows)]
            moves = c.commit(accept)
            csd_cache_commit(cache, dev(accept))
        elif kind == 3:
            parent = [int(x) for x in host.integers(-1, rows, rows)] if step < 7 else [int(x) for x in host.permutation(rows)]
            moves = c.fork(parent)
            csd_cache_fork(cache, dev(parent))
        elif kind == 5:
            moves = c.compact()
            csd_cache_compact(cache)
        else:
            lens = [int(x) for x in host.integers(-2, max(c.lens) + 3, rows)]
            moves = c.truncate(lens)
            csd_cache_truncate(cache, dev(lens))
        if moves:
            src, dst = (torch.tensor(x) for x in zip(*moves))
            for w in want:
                w[:, dst] = w[:, src]
        check_pages(cache, c)
        assert torch.equal(cache.k.cpu(), want[0]) and torch.equal(cache.v.cpu(), want[1]), (step, kind)
    flags = cache.stats()["flags"]
    assert bool(flags & decode.CACHE_FULL) == c.full and bool(flags & decode.CACHE_ROW_FULL) == c.row_full
    # bookkeeping rebuilt from tables and lengths alone is the same
    table, lens = cache.table.clone(), cache.lens.clone()
    cache.load(table, lens)
    c.granted = [0] * rows
    check_pages(cache, c)
    cache.reset()
    assert not cache.refs.any() and not cache.lens.any() and (cache.table == -1).all() and cache.stats()["flags"] == 0


def test_refused_extensions_change_nothing():
    cache = PagedCache(3, 4, 16, 1, 1, 64, torch.bfloat16, 48)
    csd_cache_extend(cache, 10)
    before = cache.meta.clone()
    csd_cache_extend(cache, 10)                                       # three pages wanted, one there
    assert cache.stats()["flags"] == decode.CACHE_FULL and not cache.granted.any() and torch.equal(cache.refs, torch.tensor([1, 1, 1, 0], device="cuda"))
    assert cache.lens.tolist() == [10] * 3
    csd_cache_extend(cache, 1, torch.tensor([39, 0, 0], dtype=torch.int32, device="cuda"))
    assert cache.stats()["flags"] == decode.CACHE_FULL | decode.CACHE_ROW_FULL and cache.lens.tolist() == [10] * 3
    csd_cache_extend(cache, 2 ** 31 - 1)
    assert cache.lens.tolist() == [10] * 3
    cache.meta.copy_(before)                                          # the bookkeeping as it was
    assert cache.granted.tolist() == [10] * 3 and cache.stats()["flags"] == 0
    csd_cache_fork(cache, torch.tensor([0, 7, -3], dtype=torch.int32, device="cuda"))
    assert cache.stats()["flags"] == decode.CACHE_BAD_ROW and cache.lens.tolist() == [10, 10, 0]


def test_unsupported_python_arguments_are_refused():
    from paper_2604_13634_b200 import CsdError
    with pytest.raises(CsdError):
        PagedCache(1, 4, 16, 1, 1, 64, torch.float32, 64)
    with pytest.raises(CsdError):
        PagedCache(1, 4, 12, 1, 1, 64, torch.bfloat16, 64)
    with pytest.raises(CsdError):
        PagedCache(5000, 4, 16, 1, 1, 64, torch.bfloat16, 64)
    cache = PagedCache(1, 4, 16, 1, 2, 64, torch.bfloat16, 64)
    with pytest.raises(CsdError):
        AttentionBuffers(cache, 34, 2)
    with pytest.raises(CsdError):
        AttentionBuffers(cache, 1, 3)
    with pytest.raises(CsdError):
        RopePlan(8, layout="other")
    buf = AttentionBuffers(cache, 1, 2)
    with pytest.raises(CsdError):
        csd_attention(torch.zeros(1, 1, 2, 64, dtype=torch.bfloat16, device="cuda"), cache, 1, buf)
    with pytest.raises(AssertionError):
        csd_attention(torch.zeros(1, 1, 2, 64, device="cuda"), cache, 0, buf)
    assert StepBuffers(1, 4, 100, torch.bfloat16).ws_bytes > 0


def test_more_tiles_than_can_be_counted_are_refused():
    from ctypes import byref
    cache = PagedCache(2, 4, 16, 1, 2, 64, torch.bfloat16, 64)
    many = decode.CacheStruct()
    for name, _ in decode.CacheStruct._fields_:
        setattr(many, name, getattr(cache._struct, name))
    many.rows, many.max_pages = 4096, 1 << 19                         # 2^29 tiles of 64 places for each head, 9 row tiles of T * 32 query rows
    q = torch.zeros(2, 33, 64, 64, dtype=torch.bfloat16, device="cuda")
    call = lambda c, ws: decode._lib().csd_attention(q.data_ptr(), *q.stride()[:3], 33, 64, byref(c), 0, 0.125, None, q.data_ptr(), None, q.data_ptr(), ws, None)  # noqa: E731
    for c, ws, why in ((many, 1 << 40, "unsupported"), (cache._struct, 16, "workspace")):
        with pytest.raises(decode.CsdError, match=why):
            decode._check(call(c, ws), "csd_attention")
    assert not q.any()
