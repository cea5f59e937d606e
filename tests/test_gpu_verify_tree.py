"""csd_verify_tree against its statement (oracle/tree_oracle.py): every result is a whole number or a copy, and equal."""

import numpy as np
import pytest
import torch

from oracle import tree_oracle as O
from paper_2604_13634_b200 import CsdError, Ocm, StepBuffers, TreeBuffers, csd_scg_threshold, csd_verify, csd_verify_tree

pytestmark = pytest.mark.gpu


def i32(x):
    return torch.tensor(np.asarray(x), dtype=torch.int32, device="cuda")


def make_case(seed, B, T, V, dtype, close=True):
    """Trees whose walk goes by matches, rescues of several candidates, ties and dead ends."""
    rng = np.random.default_rng(seed)
    parents = np.array([[-1] + [int(rng.integers(max(0, t - 6), t)) for t in range(1, T)] for _ in range(B)])
    z = torch.from_numpy(rng.normal(size=(B, T, V)).astype(np.float32)).to(dtype)
    tokens = rng.integers(0, V, (B, T))
    counts = {}
    for b in range(B):
        for c in range(T):
            below = [t for t in range(c + 1, T) if parents[b, t] == c]
            star = int(tokens[b, below[int(rng.integers(len(below)))]]) if below and rng.random() < 0.5 else int(rng.integers(V))
            z[b, c, star] = 9.0
            for t in below:
                d = int(tokens[b, t])
                if rng.random() < 0.7 and d != star:
                    z[b, c, d] = 9.0 - float(rng.choice([0.25, 0.25, 0.5, 1.0, 3.0])) if close else 9.0
                    counts[(d, star)] = int(rng.choice([1, 5, 6, 7, 100]))
    return parents, z, tokens, counts


def memory(counts, lam=6):
    ocm = Ocm(1 << 14, lam=lam)
    if counts:
        d, t, n = (i32(x) for x in zip(*[(d, t, n) for (d, t), n in counts.items()]))
        ocm.import_(d, t, n)
    return ocm


def check(buf, z, tokens, parents, nodes, counts, lam, tau):
    z, T = z.float().numpy(), z.shape[1]
    for b in range(len(z)):
        accept, nxt, path, rescued, records = O.verify(z[b], tokens[b], parents[b], nodes[b], counts, lam, csd_scg_threshold(tau))
        assert (int(buf.accept_len[b]), int(buf.next_token[b])) == (accept, nxt), b
        assert buf.path[b].tolist() == path + [-1] * (T - len(path)), b
        assert buf.rescued_mask[b].tolist() == [int(t in rescued) for t in range(T)], b
        assert buf.rej_draft[b].tolist() == [records.get(t, (-1, -1))[0] for t in range(T)], b
        assert buf.rej_target[b].tolist() == [records.get(t, (-1, -1))[1] for t in range(T)], b


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("B,T,V", [(1, 1, 7), (3, 2, 33), (5, 9, 1000), (2, 33, 32000), (9, 64, 5003), (1, 26, 128256), (40, 5, 2049), (3, 64, 151936)])
def test_verify_tree(dtype, B, T, V):
    parents, z, tokens, counts = make_case(B * T, B, T, V, dtype)
    nodes = [T if b % 3 == 0 else b * 7 % (T + 1) for b in range(B)]
    ocm, buf = memory(counts), TreeBuffers(B, T)
    for tau in (0.3, 0.0, 0.7):
        csd_verify_tree(z.cuda(), i32(tokens), i32(parents), ocm, tau, buf, n_nodes=i32(nodes))
        check(buf, z, tokens, parents, nodes, counts, 6, tau)
    st = ocm.stats()
    assert st["flags"] == 0 and st["steps"] == 3 and st["positions"] == 3 * sum(max(0, n - 1) for n in nodes)
    assert st["n_keys"] == len(counts)
    # strides, and rows that begin anywhere: the same results
    off = torch.zeros(B, T + 1, V + 5, dtype=dtype, device="cuda")
    off[:, :T, 3:V + 3] = z.cuda()
    again = TreeBuffers(B, T)
    csd_verify_tree(off[:, :T, 3:V + 3], i32(tokens), i32(parents), ocm, 0.7, again, n_nodes=i32(nodes))
    for name in ("accept_len", "next_token", "path", "rescued_mask", "rej_draft", "rej_target"):
        assert torch.equal(getattr(again, name), getattr(buf, name)), name
    ocm.close()


@pytest.mark.parametrize("lam", [0, 6])
def test_ties(lam):
    """Equal logits everywhere: the lowest token is the target's, the lowest node is taken."""
    B, T, V = 4, 12, 640
    parents, z, tokens, counts = make_case(5, B, T, V, torch.bfloat16, close=False)
    z = torch.where(torch.rand(z.shape, generator=torch.Generator().manual_seed(0)) < 0.3, torch.tensor(9.0), z.float()).bfloat16()
    z[0, :, 5] = -0.0
    z[0][z[0] > 0] = 0.0                                              # zeros of both signs are the same logit
    tokens[1] = tokens[1, 1]                                           # siblings with one token
    ocm, buf = memory(counts, lam), TreeBuffers(B, T)
    csd_verify_tree(z.cuda(), i32(tokens), i32(parents), ocm, 0.3, buf)
    check(buf, z, tokens, parents, [T] * B, counts, lam, 0.3)
    csd_verify_tree(z.cuda(), i32(tokens), i32(parents[2]), ocm, 0.3, buf)
    check(buf, z, tokens, [parents[2]] * B, [T] * B, counts, lam, 0.3)
    ocm.close()


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_a_chain_gives_what_csd_verify_gives(dtype):
    B, K, V = 6, 8, 4096
    parents, z, tokens, counts = make_case(3, B, K + 1, V, dtype)
    chain = np.arange(K + 1) - 1
    for b in range(B):
        for t in range(K):                                             # drafts that go on: matches, and pairs that the memory knows
            z[b, t, tokens[b, t + 1]] = 10.0 if (b + t) % 2 else 9.9
            counts[(int(tokens[b, t + 1]), int(z[b, t].float().argmax()))] = 50
    ocm, buf, flat = memory(counts), TreeBuffers(B, K + 1), StepBuffers(B, K, V, dtype)
    csd_verify_tree(z.cuda(), i32(tokens), i32(chain), ocm, 0.3, buf)
    csd_verify(z.cuda(), i32(tokens[:, 1:]), ocm, 0.3, flat)
    assert torch.equal(buf.accept_len, flat.accept_len) and torch.equal(buf.next_token, flat.next_token)
    assert torch.equal(buf.rescued_mask[:, 1:], flat.rescued_mask)
    assert torch.equal(buf.rej_draft[:, 1:], flat.rej_draft) and torch.equal(buf.rej_target[:, 1:], flat.rej_target)
    assert int(buf.accept_len.max()) > 1
    ocm.update(buf.rej_draft, buf.rej_target)
    assert ocm.stats()["flags"] == 0
    ocm.close()


def test_odd_inputs():
    """Tokens outside the vocabulary, parents that are no earlier nodes, NaN and infinities where the walk passes and where it does not."""
    V, T = 1003, 6
    z = torch.zeros(1, T, V)
    z[0, :, 7] = 1.0
    tokens, parents = np.array([[0, V, -5, 7, 8, 9]]), np.array([[-1, 0, 0, 0, 3, 9]])
    z[0, 1] = z[0, 5] = float("nan")
    ocm, buf = Ocm(64, lam=0), TreeBuffers(1, T)
    csd_verify_tree(z.cuda(), i32(tokens), i32(parents), ocm, 0.0, buf)
    assert buf.path.tolist() == [[0, 3, 4, -1, -1, -1]] and int(buf.next_token[0]) == 7 and ocm.stats()["flags"] == 0
    tokens[0, 3] = 2                                                     # now a divergence at the root: the two bad tokens are seen
    csd_verify_tree(z.cuda(), i32(tokens), i32(parents), ocm, 0.0, buf)
    assert buf.path.tolist() == [[0, 3, 4, -1, -1, -1]] and buf.rej_draft.tolist() == [[-1, -1, -1, 2, 8, -1]] and ocm.stats()["flags"] == 2
    for value in (float("nan"), float("inf")):
        ocm.reset()
        z[0, 3, 1002] = value
        csd_verify_tree(z.cuda(), i32(tokens), i32(parents), ocm, 0.0, buf)
        assert ocm.stats()["flags"] & 1
    ocm.reset()
    z[0, 0] = -float("inf")
    csd_verify_tree(z.cuda(), i32(tokens), i32(parents), ocm, 0.5, buf)
    assert ocm.stats()["flags"] & 1 and 0 <= int(buf.next_token[0]) < V
    ocm.close()


def test_refusals():
    ocm, z = Ocm(64), torch.zeros(2, 3, 50, device="cuda")
    buf, tok = TreeBuffers(2, 3), i32(np.zeros((2, 3)))
    for tau in (-1.0, float("nan"), float("inf")):
        with pytest.raises(CsdError):
            csd_verify_tree(z, tok, tok, ocm, tau, buf)
    with pytest.raises(CsdError):
        csd_verify_tree(z.half(), tok, tok, ocm, 0.3, buf)
    with pytest.raises(CsdError):
        csd_verify_tree(torch.zeros(2, 65, 50, device="cuda"), i32(np.zeros((2, 65))), i32(np.zeros(65)), ocm, 0.3, TreeBuffers(2, 65))
    with pytest.raises(CsdError, match="device"):
        csd_verify_tree(z, tok, tok.cpu(), ocm, 0.3, buf)
    with pytest.raises(AssertionError):
        csd_verify_tree(z, tok.long(), tok, ocm, 0.3, buf)
    with pytest.raises(CsdError):
        csd_verify_tree(z.as_strided((2, 3, 50), (10, 5, 1)), tok, tok, ocm, 0.3, buf)
    ocm.close()
