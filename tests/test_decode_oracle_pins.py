"""Pins of the decode-pass oracle: closed forms, gradients against differences, the page rules traced by hand."""

import math

import numpy as np
import pytest

from oracle import decode_oracle as O
from paper_2604_13634_b200 import binding, build, decode


@pytest.fixture(scope="module", autouse=True)
def _built():
    build.build()


@pytest.mark.parametrize("layout", ["half", "interleaved"])
def test_rope_is_a_rotation_and_relative(layout):
    rng = np.random.default_rng(0)
    th, _ = O.thetas(12)
    x, y = rng.normal(size=(2, 1, 16)), rng.normal(size=(2, 1, 16))
    a, b = O.rope(x, [7, 7], th, layout=layout), O.rope(y, [3, 3], th, layout=layout)
    np.testing.assert_allclose((a * a).sum(-1), (x * x).sum(-1), rtol=1e-13)
    np.testing.assert_array_equal(a[..., 12:], x[..., 12:])
    # scores depend on the distance of the two places alone
    c, d = O.rope(x, [1007, 1007], th, layout=layout), O.rope(y, [1003, 1003], th, layout=layout)
    np.testing.assert_allclose((a * b).sum(-1), (c * d).sum(-1), rtol=1e-9, atol=1e-12)
    # one pair at a right angle
    z = O.rope(np.array([[[1.0, 2.0]]]), [1], np.array([math.pi / 2]), layout=layout)
    np.testing.assert_allclose(z, [[[-2.0, 1.0]]], atol=1e-15)


@pytest.mark.parametrize("layout", ["half", "interleaved"])
def test_rope_gradient_is_the_inverse_turn(layout):
    rng = np.random.default_rng(1)
    th, m = O.thetas(8, scaling="yarn", factor=4.0, original_len=64)
    x, g = rng.normal(size=(3, 2, 10)), rng.normal(size=(3, 2, 10))
    pos = [0, 5, 900]
    loss = lambda z: float((O.rope(z, pos, th, m, layout) * g).sum())  # noqa: E731
    want = O.rope(g, pos, th, m, layout, inverse=True)
    for at in [(0, 0, 0), (1, 1, 3), (2, 0, 7), (2, 1, 9), (1, 0, 5)]:
        e = np.zeros_like(x)
        e[at] = 1e-5
        assert abs((loss(x + e) - loss(x - e)) / 2e-5 - want[at]) < 1e-8


@pytest.mark.parametrize("scaling,factor", [("none", 1.0), ("linear", 8.0), ("base", 4.0), ("parts", 8.0), ("yarn", 16.0)])
@pytest.mark.parametrize("rot", [2, 10, 64, 128])
def test_steps_match_the_oracle(scaling, factor, rot):
    th, m = O.thetas(rot, 500000.0, scaling, factor, 8192)
    steps, magnitude = decode.csd_rope_steps(rot, 500000.0, scaling, factor, 8192)
    got = steps.numpy().view(np.uint64).astype(np.float64) / 2.0**64 * 2 * math.pi
    # float64 powers and logarithms a few units in the last place apart, and the rounding to 2^-64 of a turn
    np.testing.assert_allclose(got, th, rtol=1e-13, atol=1e-18)
    assert magnitude == np.float32(m)


def test_scalings_do_what_they_say():
    plain, _ = O.thetas(64, original_len=1024)
    slow, fast = plain[-1], plain[0]
    for kind in ("parts", "yarn"):
        th, _ = O.thetas(64, scaling=kind, factor=8.0, original_len=1024)
        assert th[0] == fast and th[-1] == pytest.approx(slow / 8) and np.all(th <= plain) and np.all(th >= plain / 8)
    th, _ = O.thetas(64, scaling="base", factor=8.0)
    assert th[0] == fast and th[-1] == pytest.approx(slow / 8)


def test_rope_steps_refusals():
    for bad in (dict(rot=3), dict(rot=0), dict(rot=8, base=1.0), dict(rot=8, base=math.nan), dict(rot=8, scaling="linear", factor=0.5),
                dict(rot=8, scaling="parts", original_len=0.0), dict(rot=8, scaling="yarn", low=4.0, high=4.0), dict(rot=8, scaling="other"),
                dict(rot=8, scaling="linear", factor=math.inf)):
        with pytest.raises(binding.CsdError):
            decode.csd_rope_steps(**bad)


def test_page_rules_by_hand():
    c = O.Cache(3, 6, 4, 4)
    assert c.extend([5, 0, 2]) == []
    assert c.tables == [[0, 1], [], [2]] and c.lens == [5, 0, 2]
    c.fork([0, 0, 2])
    assert c.tables == [[0, 1], [0, 1], [2]] and c.refs() == [2, 2, 1, 0, 0, 0]
    # row 0 comes first and copies the shared last page; row 1 is by then alone on it and keeps it
    assert c.extend([1, 1, 3]) == [(1, 3)]
    assert c.tables == [[0, 3], [0, 1], [2, 4]] and c.refs() == [2, 1, 1, 1, 1, 0] and c.granted == [1, 1, 3]
    c.commit([0, -1, 0])
    assert c.lens == [6, 5, 3] and c.tables == [[0, 3], [0, 1], [2]]
    # too few pages: nothing happens to anyone
    assert c.extend([1, 8, 4]) == [] and c.full and c.lens == [6, 5, 3] and c.granted == [0, 0, 0]
    assert c.extend([0, 12, 0]) == [] and c.row_full
    c.fork([-1, 1, 2])
    assert c.tables == [[], [0, 1], [2]]
    c.fork([-1, -1, 2])
    assert c.compact() == [(2, 0)] and c.tables == [[], [], [0]]
    c.truncate([5, 5, -1])
    assert c.lens == [0, 0, 0] and c.refs() == [0] * 6


def test_attention_of_one_place_and_of_equal_scores():
    rng = np.random.default_rng(2)
    k, v = rng.normal(size=(2, 3, 4)), rng.normal(size=(2, 3, 4))
    q = np.zeros((3, 4, 4))
    out, lse, _, _ = O.attention(q, k, v, 3, 0.5)
    for t in range(3):
        for h in range(4):
            np.testing.assert_allclose(out[t, h], v[h // 2, :t + 1].mean(0))
            assert lse[t, h] == pytest.approx(math.log(t + 1))
    # more new tokens than there are: the first one sees nothing; a token beyond n_new neither
    out, lse, _, _ = O.attention(np.zeros((4, 4, 4)), k[:, :2], v[:, :2], 3, 0.5)
    assert not out[0].any() and np.isinf(lse[0]).all() and not out[3].any() and np.isinf(lse[3]).all()
    np.testing.assert_allclose(out[1, 0], v[0, 0])
    # joining two halves by their lse gives the whole
    q = rng.normal(size=(1, 4, 4))
    whole, L, _, _ = O.attention(q, k, v, 1, 0.5)
    a, la, _, _ = O.attention(q, k[:, :2], v[:, :2], 1, 0.5)
    b, lb, _, _ = O.attention(q, k[:, 2:], v[:, 2:], 1, 0.5)
    np.testing.assert_allclose(np.logaddexp(la, lb), L)
    np.testing.assert_allclose(np.exp(la - L)[..., None] * a + np.exp(lb - L)[..., None] * b, whole)


def test_sizes_without_a_device():
    L = decode._lib()
    lay = decode.CacheLayout()
    for rows, width, pages in ((1, 1, 1), (3, 7, 40), (4096, 100, 100000), (128, 64, 33)):
        total = L.csd_cache_meta_bytes(rows, width, pages)
        assert L.csd_cache_meta_layout(rows, width, pages, lay) == 0 and lay.total == total
        ends = [(lay.lens, 4 * rows), (lay.granted, 4 * rows), (lay.table, 4 * rows * width), (lay.refs, 4 * pages), (lay.free_bits, 4 * -(-pages // 32))]
        at = lay.flags + 4
        for off, n in ends:                                       # in order, apart, on 256-byte boundaries
            assert off >= at and off % 256 == 0
            at = off + n
        assert at <= total
        assert L.csd_cache_scratch_bytes(rows, width, pages) >= 8 * max(rows, pages // 2) + 4 * pages + 4 * rows * (width + 1)
    for bad in ((0, 1, 1), (4097, 1, 1), (1, 0, 1), (1, 1, 0)):
        assert L.csd_cache_meta_bytes(*bad) == 0 and L.csd_cache_scratch_bytes(*bad) == 0 and L.csd_cache_meta_layout(*bad, lay) == 1
    assert L.csd_attention_workspace_bytes(4, 9, 32, 8, 128) > 0
    for bad in ((0, 1, 8, 8, 64), (4, 0, 8, 8, 64), (4, 34, 8, 8, 64), (4, 1, 9, 8, 64), (4, 1, 8, 8, 60), (4, 1, 8, 8, 264), (4097, 1, 8, 8, 64)):
        assert L.csd_attention_workspace_bytes(*bad) == 0


def _struct(**kw):
    """A cache description with addresses that are never dereferenced: every call on it has to refuse before a launch."""
    a = dict(k=4096, v=8192, dtype=1, layers=2, n_pages=10, page_size=16, heads=4, dim=64, stride_layer=10 * 4096, stride_page=4096,
             stride_head=1024, stride_token=64, rows=3, max_pages=5, meta=4096, scratch=4096)
    a.update(kw)
    return decode.CacheStruct(*[a[n] for n, _ in decode.CacheStruct._fields_])


@pytest.mark.parametrize("kw,status", [
    (dict(k=None), 1), (dict(v=None), 1), (dict(meta=None), 1), (dict(scratch=None), 1), (dict(dtype=0), 4), (dict(dtype=7), 1),
    (dict(layers=0), 1), (dict(n_pages=0), 1), (dict(rows=0), 1), (dict(max_pages=-1), 1), (dict(page_size=12), 4), (dict(page_size=4), 4),
    (dict(page_size=512), 4), (dict(dim=60), 4), (dict(dim=264), 4), (dict(rows=5000), 4), (dict(k=4104), 1), (dict(meta=4112), 1),
    (dict(stride_head=1032), 1), (dict(stride_token=72), 1), (dict(stride_page=4095), 1), (dict(stride_page=4000), 1),
    (dict(stride_layer=4096), 1), (dict(stride_layer=10 * 4096 + 4), 1), (dict(stride_layer=-40960), 1)])
def test_bad_caches_are_refused_before_a_launch(kw, status):
    L, c = decode._lib(), _struct(**kw)
    assert L.csd_cache_extend(c, 1, None, None) == status
    assert L.csd_cache_rebuild(c, None) == status and L.csd_cache_compact(c, None) == status
    assert L.csd_cache_truncate(c, 4096, None) == status and L.csd_cache_commit(c, 4096, None) == status
    assert L.csd_cache_fork(c, 4096, None) == status
    assert L.csd_attention(4096, 512, 256, 64, 2, 4, c, 0, 1.0, None, 4096, None, 4096, 1 << 30, None) == status
    assert L.csd_rope_append(4096, 512, 256, 64, 4, 4096, 512, 256, 64, 4096, 512, 256, 64, 4096, 2, c, 0, None, None, None) == status


def test_bad_calls_are_refused_before_a_launch():
    L, c = decode._lib(), _struct()
    assert L.csd_cache_extend(None, 1, None, None) == 1 and L.csd_cache_extend(c, -1, None, None) == 1
    assert L.csd_cache_truncate(c, None, None) == 1 and L.csd_cache_commit(c, None, None) == 1 and L.csd_cache_fork(c, None, None) == 1

    def attend(q=4096, sb=512, st=256, sh=64, T=2, Hq=4, layer=0, scale=1.0, out=4096, ws=4096, n=1 << 30):
        return L.csd_attention(q, sb, st, sh, T, Hq, c, layer, scale, None, out, None, ws, n, None)
    assert attend(q=None) == 1 and attend(out=None) == 1 and attend(ws=None) == 1 and attend(T=0) == 1 and attend(layer=2) == 1 and attend(layer=-1) == 1
    assert attend(scale=math.nan) == 1 and attend(scale=math.inf) == 1 and attend(q=4100) == 1 and attend(sh=60) == 1 and attend(out=4104) == 1
    assert attend(T=34) == 4 and attend(Hq=6) == 4 and attend(n=16) == 5 and attend(ws=4112) == 5

    turn = decode.RopeStruct(4096, 16, 0, 1.0)
    def rope(x=4096, y=4096, dt=1, B=1, S=1, H=1, D=16, pos=4096, r=turn):
        return L.csd_rope(x, y, dt, B, S, H, D, 16, 16, 16, 16, 16, 16, pos, 1, 1, r, 0, None)
    assert rope(x=None) == 1 and rope(y=None) == 1 and rope(pos=None) == 1 and rope(r=None) == 1 and rope(dt=3) == 1 and rope(dt=-1) == 1
    assert rope(B=-1) == 1 and rope(D=0) == 1 and rope(D=14) == 1
    for bad in (decode.RopeStruct(None, 16, 0, 1.0), decode.RopeStruct(4096, 15, 0, 1.0), decode.RopeStruct(4096, 0, 0, 1.0),
                decode.RopeStruct(4096, 16, 2, 1.0), decode.RopeStruct(4096, 16, 0, math.nan)):
        assert rope(r=bad) == 1
    assert rope(B=0, x=None) == 0 and rope(S=0) == 0 and rope(H=0) == 0      # nothing to do
