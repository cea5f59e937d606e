"""Pins of the tree and budget oracle (oracle/tree_oracle.py): closed forms, the chain's oracles, brute force, hand traces; and what the
host refuses before anything is launched.  No GPU."""

import itertools
import math
import os
import re
from ctypes import byref

import numpy as np
import pytest

from oracle import csd_oracle
from oracle import decode_oracle as D
from oracle import tree_oracle as O
from paper_2604_13634_b200 import binding, build, decode

INVALID_ARG, UNSUPPORTED, WORKSPACE = 1, 4, 5
SOMEWHERE = 1 << 20                                                  # an aligned address that nothing may follow


@pytest.fixture(scope="module", autouse=True)
def _built():
    build.build()


def test_plans_by_hand():
    assert O.plan([-1, 0, 0, 1, 3, 2], 6, 10) == ([1, 3, 5, 11, 27, 37], [10, 11, 11, 12, 13, 12])
    assert O.plan([-1, 0, 1, 2], 3, 0, offset=5) == ([1, 3, 7, 0], [5, 6, 7, 0])
    assert O.plan([9, 1, -4], 3, 7) == ([1, 2, 4], [7, 7, 7])           # no earlier node: on its own
    assert O.plan(list(range(-1, 63)), 64, 0)[0] == [2 ** (t + 1) - 1 for t in range(64)]


def test_masks_of_a_chain_are_the_chain():
    rng = np.random.default_rng(0)
    T, n = 5, 12
    q, k, v = rng.normal(size=(T, 4, 8)), rng.normal(size=(2, n, 8)), rng.normal(size=(2, n, 8))
    for n_new in (5, 3, 12, 14):
        a = O.attention(q, k, v, [2 ** (t + 1) - 1 for t in range(T)], n_new, 0.3)
        b = D.attention(q, k, v, n_new, 0.3)
        for x, y in zip(a, b):
            np.testing.assert_allclose(x, y, rtol=1e-13)


def test_a_branch_is_attention_without_the_others():
    rng = np.random.default_rng(1)
    q, k, v = rng.normal(size=(4, 1, 8)), rng.normal(size=(1, 9, 8)), rng.normal(size=(1, 9, 8))
    masks = O.plan([-1, 0, 0, 2], 4, 0)[0]
    out = O.attention(q, k, v, masks, 4, 0.5)[0]
    for t, branch in ((1, [0, 1]), (3, [0, 2, 3])):
        keep = list(range(5)) + [5 + u for u in branch]
        want = D.attention(q[branch], k[:, keep], v[:, keep], len(branch), 0.5)[0]
        np.testing.assert_allclose(out[t], want[-1], rtol=1e-13)
    assert (O.attention(q, k[:, :4], v[:, :4], [0, 1, 2, 0], 4, 0.5)[0][[0, 3]] == 0).all()


def test_mass_is_the_softmax():
    rng = np.random.default_rng(2)
    q, k, v = rng.normal(size=(3, 4, 8)), rng.normal(size=(2, 10, 8)), rng.normal(size=(2, 10, 8))
    masks = O.plan([-1, 0, 0], 3, 0)[0]
    out, lse, _, _ = O.attention(q, k, v, masks, 3, 0.7)
    got = O.mass(q, k, lse, masks, 3, 0.7, np.zeros(10), False)[0]
    assert abs(got.sum() - 12) < 1e-12 and got[8] > 0 and got[9] > 0
    # the weights that rebuild the output: with values that are places, the sum of outputs is the mean place
    places = np.broadcast_to(np.arange(10.0)[None, :, None], (2, 10, 1))
    mean = O.attention(q, k, np.repeat(places, 8, axis=2), masks, 3, 0.7)[0][..., 0].sum()
    assert abs(mean - got @ np.arange(10)) < 1e-10
    before = np.arange(10.0)
    np.testing.assert_allclose(O.mass(q, k, lse, masks, 3, 0.7, before, True)[0], got + np.where(np.arange(10) < 7, before, 0))


def test_a_chain_verifies_as_csd_verify_does():
    rng = np.random.default_rng(3)
    for trial in range(60):
        K, V = 4, 6
        z = np.round(rng.normal(size=(1, K + 1, V)) * 2).astype(np.float32)
        draft = rng.integers(0, V, (1, K)).astype(np.int32)
        mem, counts = csd_oracle.OCM(256, lam=2), {}
        for d, t in itertools.product(range(V), range(V)):
            for _ in range(int(rng.integers(0, 4))):
                mem.update([(d, t)])
                counts[(d, t)] = counts.get((d, t), 0) + 1
        ref = csd_oracle.step(z, draft, mem, 0.3)
        tokens = np.concatenate([[[0]], draft], axis=1)[0]
        accept, nxt, path, rescued, records = O.verify(z[0], tokens, list(range(-1, K)), K + 1, counts, 2, csd_oracle.scg_threshold(0.3))
        assert accept == ref["accept_len"][0] and nxt == ref["next_token"][0] and path == list(range(accept + 1))
        assert [int(t in rescued) for t in range(1, K + 1)] == ref["rescued_mask"][0].tolist()
        assert [records.get(t, (-1, -1))[0] for t in range(1, K + 1)] == ref["rej_draft"][0].tolist()
        assert [records.get(t, (-1, -1))[1] for t in range(1, K + 1)] == ref["rej_target"][0].tolist()


def test_verification_by_hand():
    z = np.zeros((5, 8), dtype=np.float32)
    z[0, [3, 4, 5]] = 2.0, 1.9, 1.9                                     # after the root: 3
    z[2, 6] = 1.0
    tokens, parents, known = [0, 4, 5, 4, 6], [-1, 0, 0, 0, 2], {(4, 3): 5, (5, 3): 9}
    assert O.verify(z, tokens, parents, 5, known, 6, -1.0) == (2, 0, [0, 2, 4], {2}, {1: (4, 3), 2: (5, 3), 3: (4, 3)})
    known[(4, 3)] = 6                                                    # now nodes 1, 2 and 3 would do: the same logit, the lowest node
    assert O.verify(z, tokens, parents, 5, known, 6, -1.0)[2] == [0, 1]
    assert O.verify(z, tokens, parents, 5, known, 6, -0.05)[2] == [0]
    assert O.verify(z, [0, 3, 5, 3, 6], parents, 5, known, 6, -1.0)[2] == [0, 1]
    assert O.verify(z, tokens, parents, 0, known, 6, -1.0) == (0, -1, [], set(), {})


def test_paths_and_budgets_by_hand():
    assert O.kept_of_path(5, 2, [0, 3, 4, -1]) == ([0, 3, 4], False)
    assert O.kept_of_path(5, 9, [0, 1, 2, 3, 4]) == ([0, 1, 2, 3, 4], False)
    assert O.kept_of_path(5, 3, [0, 2, 2, 3]) == ([0, 2], True) and O.kept_of_path(0, 3, [0]) == ([], False)
    assert O.evict([5, 1, 4, 2, 3, 0], 6, 4, 1, 1) == [0, 4, 2, 5]       # 2 and 4 are the best between; 4 fills the hole at 1
    assert O.evict([1, 1, 1, 1, 1], 5, 3, 0, 0) == [0, 1, 2] and O.evict([1, 2, 3], 3, 3, 0, 0) == [0, 1, 2]
    assert O.evict([9, 0, 0, 9, 9, 1], 6, 3, 0, 2) == [0, 4, 5] and O.evict([1, 2], 2, 0, 5, 5) == []
    assert O.evict([math.nan, -math.inf, 1.0, math.nan], 4, 2, 0, 0) == [2, 1]


def test_budgets_against_brute_force():
    """Of all ways to keep W places, the rule's has the largest sum; the recent ones stay in order; as many move as leave, and the recent."""
    rng = np.random.default_rng(4)
    for _ in range(200):
        n = int(rng.integers(1, 9))
        keep, sinks, recent = int(rng.integers(0, n + 1)), int(rng.integers(0, 3)), int(rng.integers(0, 4))
        mass = rng.integers(0, 5, n).astype(float)
        got = O.evict(mass, n, keep, sinks, recent)
        assert len(got) == len(set(got)) == keep
        if keep < n:
            r = min(recent, keep)
            s = min(sinks, keep - r)
            assert got[keep - r:] == list(range(n - r, n)) and got[:s] == list(range(s))
            middle = range(s, n - r)
            best = max(sum(mass[list(c)]) for c in itertools.combinations(middle, keep - r - s))
            assert sum(mass[got[s:keep - r]]) == best
            assert sum(i != j for i, j in enumerate(got)) <= n - keep + r


# ---- the host ----

def _cache(**kw):
    f = dict(layers=1, n_pages=4, page=16, heads=2, dim=64, rows=2, max_pages=4)
    f.update(kw)
    e = f["heads"] * f["page"] * f["dim"]
    return decode.CacheStruct(SOMEWHERE, SOMEWHERE, binding.CSD_BF16, f["layers"], f["n_pages"], f["page"], f["heads"], f["dim"], f["n_pages"] * e, e,
                              f["page"] * f["dim"], f["dim"], f["rows"], f["max_pages"], SOMEWHERE, SOMEWHERE)


def test_tree_calls_refuse_what_they_cannot_do():
    L, c = decode._lib(), _cache()
    s3 = (2 * 8 * 64, 8 * 64, 64)
    plan = lambda T, masks, stride=0: L.csd_tree_plan(None, stride, T, byref(c), None, None, masks, None, None)  # noqa: E731
    assert plan(0, SOMEWHERE) == plan(3, None) == plan(3, SOMEWHERE + 4) == plan(3, SOMEWHERE, -1) == INVALID_ARG and plan(65, SOMEWHERE) == UNSUPPORTED
    tree = lambda T=3, heads=8, masks=SOMEWHERE, ws=1 << 40, at=SOMEWHERE, scale=1.0: L.csd_attention_tree(  # noqa: E731
        at, *s3, T, heads, byref(c), 0, scale, None, masks, SOMEWHERE, None, SOMEWHERE, ws, None)
    assert tree(masks=None) == tree(masks=SOMEWHERE + 4) == tree(at=SOMEWHERE + 8) == tree(scale=math.inf) == INVALID_ARG
    assert tree(T=65) == tree(heads=7) == UNSUPPORTED and tree(ws=100) == WORKSPACE
    assert L.csd_attention_tree_workspace_bytes(2, 65, 8, 2, 64) == 0 and L.csd_attention_tree_workspace_bytes(2, 64, 8, 2, 64) > 0
    assert L.csd_attention_workspace_bytes(2, 34, 8, 2, 64) == 0
    mass = lambda T=3, heads=8, lse=SOMEWHERE, masks=None, to=SOMEWHERE, stride=64, layer=0: L.csd_attention_mass(  # noqa: E731
        SOMEWHERE, *s3, T, heads, lse, byref(c), layer, 1.0, None, masks, to, stride, 0, None)
    assert mass(lse=None) == mass(to=None) == mass(masks=SOMEWHERE + 4) == mass(stride=63) == mass(layer=1) == INVALID_ARG
    assert mass(T=65) == mass(heads=3) == UNSUPPORTED
    path = lambda T=3, accept=SOMEWHERE, at=SOMEWHERE, mass=None, stride=0: L.csd_cache_commit_path(byref(c), accept, at, T, mass, stride, None)  # noqa: E731
    assert path(accept=None) == path(at=None) == path(T=0) == path(mass=SOMEWHERE, stride=63) == INVALID_ARG and path(T=65) == UNSUPPORTED


def test_eviction_refuses_what_it_cannot_do():
    L, c = decode._lib(), _cache()
    need = L.csd_cache_evict_workspace_bytes(2, 20)
    assert need > 0 and L.csd_cache_evict_workspace_bytes(0, 20) == L.csd_cache_evict_workspace_bytes(4097, 20) == L.csd_cache_evict_workspace_bytes(2, -1) == 0
    call = lambda mass=SOMEWHERE, stride=64, keep=10, sinks=1, recent=1, kept=SOMEWHERE, width=20, evicted=SOMEWHERE, ws=SOMEWHERE, size=need: (  # noqa: E731
        L.csd_cache_evict(byref(c), mass, stride, keep, None, sinks, recent, kept, width, evicted, ws, size, None))
    for bad in (dict(mass=None), dict(stride=63), dict(keep=-1), dict(keep=21), dict(sinks=-1), dict(recent=-1), dict(kept=None), dict(width=-1),
                dict(evicted=None), dict(ws=None)):
        assert call(**bad) == INVALID_ARG, bad
    assert call(size=need - 1) == call(ws=SOMEWHERE + 128) == WORKSPACE


def test_verification_refuses_what_it_cannot_do():
    L = binding.lib()
    call = lambda z=SOMEWHERE, dtype=1, B=2, T=3, V=50, sb=150, st=50, tok=SOMEWHERE, par=SOMEWHERE, ps=0, ocm=SOMEWHERE, tau=0.3, out=SOMEWHERE: (  # noqa: E731
        L.csd_verify_tree(z, dtype, B, T, V, sb, st, tok, par, ps, None, ocm, tau, out, SOMEWHERE, SOMEWHERE, SOMEWHERE, SOMEWHERE, SOMEWHERE, None))
    for bad in (dict(z=None), dict(dtype=2), dict(B=0), dict(T=0), dict(V=0), dict(sb=149), dict(st=49), dict(tok=None), dict(par=None), dict(ps=-1),
                dict(ocm=None), dict(tau=-0.1), dict(tau=math.nan), dict(tau=math.inf), dict(out=None)):
        assert call(**bad) == INVALID_ARG, bad
    assert call(T=65, sb=65 * 50) == UNSUPPORTED


# ---- rules of the sources ----

CSRC = os.path.join(os.path.dirname(os.path.abspath(build.__file__)), "csrc")


def _code(name):
    with open(os.path.join(CSRC, name)) as f:
        return re.sub(r"//[^\n]*", "", f.read())


@pytest.mark.parametrize("name", ["csd_tree.cuh", "csd_verify_tree.cuh", "csd_keep.cuh", "csd_mass.cuh"])
def test_nothing_is_loaded_as_read_only(name):
    """Kernels that start beside their predecessor must not load what it writes as data that nobody writes; each waits before anything else."""
    code = _code(name)
    assert not re.findall(r"__ldg\(|ld_stream16|\.nc\b", code)
    for kernel in re.split(r"__global__", code)[1:]:
        assert "wait_for_stream();" in kernel


def test_blocks_that_give_up_still_meet_and_stay():
    """The kernel of the attention mass: a wait that ran out leaves no barrier of the cluster out, and the block lingers before its memory goes."""
    code = _code("csd_mass.cuh")
    end = code[code.rindex("if (*give_up)"):]
    assert "CSD_CACHE_INTERNAL" in end and end.index("ptx::linger();") < end.index("tmem_dealloc")
    # three roles, each with the same two meetings to a run and none inside a test of `ok`
    assert len(re.findall(r"if \(blocks > 1\) \{\s*cluster_meet\(\);\s*cluster_meet\(\);\s*\}", code)) == 2
    assert len(re.findall(r"if \(blocks > 1\) cluster_meet\(\);", code)) == 2
    assert not re.search(r"ok[^\n;]*\)\s*\{?\s*cluster_meet", code)
