"""Timed cases of the tree form of a verification pass and of a cache kept to a budget: attention of a tree of drafted tokens over
the paged cache, verification of the tree, keeping the accepted path, attention weight accumulated per place, eviction by it.

`own = False` computes each operator in elementary torch operations (32 bits, rounded once at the end);
`own = True` makes the package's calls on the same inputs.  `exact` states the computed ones a second time, in 64 bits.
"""

import math

import numpy as np
import torch

own = False

DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
BYTES = {"f32": 4, "bf16": 2, "f16": 2}
LAMBDA, TAU = 6, 0.3


# ---- the cases -------------------------------------------------------------------------------------------------

def listed():
    tree = dict(op="tree", dtype="bf16", ragged=False, token_major=False)
    ver = dict(op="verify", dtype="bf16", ragged=False)
    path = dict(op="path", dtype="bf16", token_major=False)
    mass = dict(op="mass", dtype="bf16", ragged=False, token_major=False, tree=False, back=2.0, fresh=True)
    evict = dict(op="evict", dtype="bf16", token_major=False)
    return [
        # a small draft model scoring the eight nodes of its own beam for 16 rows: half precision, a key head to every query head
        dict(tree, name="tree_small_f16", B=16, T=8, Hq=16, Hkv=16, D=64, page=32, lo=0, hi=3000, back=2.0, dtype="f16", token_major=True),
        # one conversation, a tree of 26 nodes, a short history: an ordinary verification pass, mostly latency
        dict(tree, name="tree_one", B=1, T=26, Hq=32, Hkv=8, D=128, page=16, lo=2000, hi=2000, back=3.0),
        # one row, the widest tree, many query heads to a key head, a long history: 512 query rows to every key
        dict(tree, name="tree_wide_long", B=1, T=64, Hq=64, Hkv=8, D=128, page=64, lo=30001, hi=30001, back=4.0),
        # batched serving with trees of up to 40 nodes, ragged lengths and ragged trees, empty rows among them
        dict(tree, name="tree_batch", B=32, T=40, Hq=40, Hkv=8, D=128, page=16, lo=0, hi=8191, back=3.0, ragged=True),
        # the end of the pass of one conversation: 26 nodes over a large vocabulary
        dict(ver, name="verify_one", B=1, T=26, V=128256, back=3.0, depth=4),
        # the end of the pass of a batch: trees of up to 40 nodes, some paths long, some none
        dict(ver, name="verify_batch", B=48, T=40, V=151936, back=3.0, depth=9, ragged=True),
        # one conversation's accepted path in all layers: four tokens move; all latency
        dict(path, name="path_one", B=1, T=26, layers=32, Hkv=8, D=128, page=16, lo=45, hi=45, keep=5),
        # a batch's accepted paths, tokens of a page side by side
        dict(path, name="path_batch", B=64, T=40, layers=28, Hkv=8, D=128, page=16, lo=40, hi=75, keep=10, token_major=True),
        # the weight that one new token gives the places of a short history: all latency
        dict(mass, name="mass_one_short", B=1, T=1, Hq=32, Hkv=8, D=128, page=16, lo=700, hi=700),
        # the weights of a batch's drafted trees
        dict(mass, name="mass_batch", B=96, T=9, Hq=32, Hkv=8, D=128, page=64, lo=500, hi=4000, tree=True, fresh=False),
        # a step of a batch at its budget: each row has a few tokens too many
        dict(evict, name="evict_step", B=16, layers=16, Hkv=8, D=128, page=16, lo=1009, hi=1033, keep=1008, sinks=4, recent=128),
        # long prompts cut down to a budget before decoding
        dict(evict, name="evict_prompts", B=8, layers=4, Hkv=8, D=128, page=64, lo=6000, hi=16384, keep=4096, sinks=16, recent=512),
    ]


def _spread(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _drawn(rng):
    op = rng.choice(["tree", "tree", "verify", "path", "mass", "evict"])
    if op == "verify":
        T = rng.choice([1, 2, 5, 9, 16, 26, 33, 40, 63, 64])
        return dict(op=op, dtype=rng.choice(["bf16", "f32"]), B=_spread(rng, 1, 96), T=T, V=rng.choice([32000, 128256, 151936, _spread(rng, 500, 200000)]),
                    back=rng.choice([0.5, 1.0, 3.0, 6.0]), depth=rng.randint(1, 12), ragged=rng.random() < 0.5)
    page, layout = rng.choice([16, 32, 64, 128]), dict(token_major=rng.random() < 0.5, dtype=rng.choice(["bf16", "bf16", "f16"]))
    if op in ("tree", "mass"):
        h, g = rng.choice([1, 2, 4, 8, 16]), rng.choice([1, 2, 3, 4, 5, 7, 8, 12, 16])
        hi = _spread(rng, 70, 131072)
        T = rng.choice([1, 3, 8, 16, 26, 33, 40, 60, 64] if op == "tree" else [1, 1, 1, 2, 5, 9, 16, 33, 64])
        c = dict(layout, op=op, B=_spread(rng, 1, 128), T=T, Hq=h * g, Hkv=h, D=rng.choice([64, 64, 80, 96, 128, 128, 128, 256]), page=page,
                 lo=rng.choice([0, T, hi // 2, hi]), hi=hi, ragged=rng.random() < 0.5, back=rng.choice([0.5, 2.0, 4.0]))
        return c if op == "tree" else dict(c, tree=rng.random() < 0.5, fresh=rng.random() < 0.5)
    c = dict(layout, op=op, B=_spread(rng, 1, 64), layers=rng.randint(1, 24), Hkv=rng.choice([1, 2, 4, 8, 16]), D=rng.choice([64, 80, 128, 128]), page=page)
    if op == "path":
        T = rng.choice([2, 8, 16, 26, 40, 64])
        hi = _spread(rng, T, 500)
        return dict(c, T=T, lo=rng.randint(T, hi), hi=hi, keep=rng.randint(1, min(T, 16)))
    hi = _spread(rng, 200, 32768)
    keep = rng.randint(max(64, hi // 8), hi)
    return dict(c, lo=rng.randint(hi // 2, hi), hi=hi, keep=keep, sinks=rng.choice([0, 1, 4, 16]), recent=rng.randint(0, keep // 2))


def draw(rng):
    """One more case: no more work than the largest listed one, and a plain form whose padded 32-bit tensors fit."""
    top = max(work(c)["bytes"] for c in listed())
    flops = max(work(c)["flops"] for c in listed())
    while True:
        c = _drawn(rng)
        w = work(c)
        if w["bytes"] > top or w["flops"] > flops:
            continue
        if c["op"] == "verify" and c["B"] * c["T"] * c["V"] > 3.2e8:
            continue
        if c["op"] != "verify" and _pool_bytes(c) > 1.2e9:
            continue
        if c["op"] in ("tree", "mass") and c["B"] * c["hi"] * max(c["Hq"] * c["T"], c["Hkv"] * c["D"]) > 1.5e9:
            continue
        return c


# ---- what follows from a case alone ----------------------------------------------------------------------------

def _lens(c):
    """Cached tokens of each row, the new ones among them: evenly from lo to hi."""
    b = c["B"]
    return [c["hi"]] if b == 1 else [round(c["lo"] + (c["hi"] - c["lo"]) * i / (b - 1)) for i in range(b)]


def _news(c):
    """New tokens of each row: T, or 1 .. T in turn; no more than there are."""
    return [min(n, 1 + 7 * i % c["T"] if c["ragged"] else c["T"]) for i, n in enumerate(_lens(c))]


def _parents(c):
    """[B, T] parent of each node (the root's is -1): an earlier node, `back` places before it on average."""
    rng = np.random.default_rng([c["B"], c["T"], int(10 * c["back"])])
    t = np.arange(c["T"])
    return np.maximum(t - 1 - rng.exponential(c["back"], (c["B"], c["T"])).astype(np.int64), np.where(t > 0, 0, -1))


def _ancestors(parents):
    """[B, T, T] bool: node t sees node u, itself among them."""
    B, T = parents.shape
    seen = np.zeros((B, T, T), dtype=bool)
    for t in range(T):
        if t:
            seen[:, t] = seen[np.arange(B), parents[:, t]]
        seen[:, t, t] = True
    return seen


def _seen_bits(c):
    """[B, T, T] bool of a tree's nodes, or of a chain's."""
    return _ancestors(_parents(c)) if c["op"] == "tree" or c["tree"] else np.broadcast_to(np.tri(c["T"], dtype=bool), (c["B"], c["T"], c["T"]))


def _walk(c):
    """The plan of a verification: nodes of each row, the parents, and the nodes that each row's walk takes."""
    parents = _parents(c)
    rng = np.random.default_rng([c["B"], c["T"], c["depth"]])
    nodes = [1 + 5 * i % c["T"] if c["ragged"] else c["T"] for i in range(c["B"])]
    paths = []
    for b, n in enumerate(nodes):
        taken, want = [0], int(rng.integers(0, c["depth"] + 1))
        while len(taken) <= want:
            below = [t for t in range(1, n) if parents[b, t] == taken[-1]]
            if not below:
                break
            taken.append(int(rng.choice(below)))
        paths.append(taken)
    return nodes, parents, paths


def _accepted(c):
    """[B][k] places, among a row's T new tokens, of the path that stays: ascending, the root first."""
    rng = np.random.default_rng([c["B"], c["T"], c["keep"]])
    return [[0] + sorted(rng.choice(np.arange(1, c["T"]), int(n) - 1, replace=False).tolist()) for n in rng.integers(1, c["keep"] + 1, c["B"])]


def _page_bytes(c):
    return 2 * c.get("layers", 1) * c["Hkv"] * c["D"] * c["page"] * BYTES[c["dtype"]]


def _pool_bytes(c):
    return _page_bytes(c) * (sum(-(-n // c["page"]) for n in _lens(c)) * 9 // 8 + 2)


def work(c):
    e = BYTES[c["dtype"]]
    if c["op"] == "verify":
        visited = sum(len(p) for p in _walk(c)[2])
        return {"bytes": visited * c["V"] * e + c["B"] * c["T"] * 24, "flops": visited * c["V"]}
    lens = _lens(c)
    if c["op"] in ("tree", "mass"):
        news, seen = _news(c), _seen_bits(c)
        rows = c["B"] * c["T"] * c["Hq"]
        pairs = sum(n * (m - n) + int(seen[b, :n, :n].sum()) for b, (m, n) in enumerate(zip(lens, news)))
        kv = sum(lens) * c["Hkv"] * c["D"] * e
        if c["op"] == "tree":
            return {"bytes": 2 * kv + 2 * rows * c["D"] * e + 4 * rows + 8 * c["B"] * c["T"], "flops": 4 * c["Hq"] * c["D"] * pairs}
        return {"bytes": kv + rows * (c["D"] * e + 4) + 8 * sum(lens), "flops": 2 * c["Hq"] * c["D"] * pairs}
    token = 2 * c["layers"] * c["Hkv"] * c["D"] * e
    if c["op"] == "path":
        moved = sum(sum(t != i for i, t in enumerate(p)) for p in _accepted(c))
        return {"bytes": 2 * moved * token + 8 * c["B"] * (c["T"] + 2), "flops": c["B"] * c["T"]}
    # the recent tokens, and as many of the others as stay among the last places that are given up
    long = [n for n in lens if n > c["keep"]]
    moved = sum(c["recent"] + (n - c["keep"]) * (c["keep"] - c["sinks"] - c["recent"]) // (n - c["sinks"] - c["recent"]) for n in long)
    return {"bytes": 2 * moved * token + 4 * sum(long) + 4 * c["B"] * c["keep"] + 8 * moved, "flops": sum(lens)}


# ---- inputs ----------------------------------------------------------------------------------------------------

def _rows(c, s, host, layers):
    """Page tables, lengths and a pool with holes, every page with values in it."""
    order = np.arange(c["B"]) if c["op"] in ("path", "tree", "mass") else host.permutation(c["B"])
    lens = np.array(_lens(c))[order]
    held = -(-lens // c["page"])
    total = int(held.sum())
    n_pages = total * 9 // 8 + 2
    ids = host.permutation(n_pages)[:total]
    table, at = np.full((c["B"], max(1, int(held.max()))), -1, dtype=np.int32), 0
    for b, m in enumerate(held):
        table[b, :m] = ids[at:at + m]
        at += m
    s["table"], s["lens"] = torch.from_numpy(table).cuda(), torch.tensor(lens, dtype=torch.int32).cuda()
    s["n_pages"] = n_pages
    shape = (layers, n_pages, c["page"], c["Hkv"], c["D"]) if c["token_major"] else (layers, n_pages, c["Hkv"], c["page"], c["D"])
    gen = torch.Generator(device="cuda").manual_seed(int(host.integers(1 << 40)))
    for x in ("k", "v"):
        t = torch.randn(shape, generator=gen, device="cuda", dtype=DTYPES[c["dtype"]])
        s[x] = t.transpose(2, 3) if c["token_major"] else t
    return gen


def _cache(c, s):
    """The package's handle on the pool, the table and the lengths in hand."""
    import paper_2604_13634_b200 as csd
    cache = csd.PagedCache(c["B"], s["n_pages"], c["page"], s["k"].shape[0], c["Hkv"], c["D"], DTYPES[c["dtype"]], s["table"].shape[1] * c["page"],
                           k=s["k"], v=s["v"])
    cache.load(s["table"], s["lens"])
    return cache


def prepare(c, seed):
    host = np.random.default_rng(seed)
    s = {"case": c}
    if c["op"] == "verify":
        return _prepare_verify(c, s, host)
    gen = _rows(c, s, host, c.get("layers", 1))
    places = s["table"].shape[1] * c["page"]
    if c["op"] in ("tree", "mass"):
        q = torch.randn((c["B"], c["T"], c["Hq"], c["D"]), generator=gen, device="cuda", dtype=DTYPES[c["dtype"]])
        s["q"] = 2.0 * q if c["op"] == "tree" else q
        s["news"] = torch.tensor(_news(c), dtype=torch.int32).cuda()
        s["seen"] = torch.from_numpy(np.ascontiguousarray(_seen_bits(c))).cuda()
        parents = torch.from_numpy(_parents(c).astype(np.int32)).cuda()
        if c["op"] == "mass":
            # what attention leaves for such rows: n independent scores of variance |scale q|^2
            t = torch.arange(c["T"], device="cuda")
            n = (s["lens"] - s["news"])[:, None] + (s["seen"] & (t < s["news"][:, None])[:, None, :]).sum(-1)
            lse = n[:, :, None].clamp(min=1).float().log() + 0.5 * s["q"].float().square().sum(-1) / c["D"]
            s["lse"] = torch.where((t < s["news"][:, None])[:, :, None], lse, -math.inf)
            before = torch.rand((c["B"], places), generator=gen, device="cuda") * 4.0
            s["mass"] = before.masked_fill(torch.arange(places, device="cuda") >= s["lens"][:, None], 0.0)
        if own:
            import paper_2604_13634_b200 as csd
            s["cache"] = _cache(c, s)
            s["plan"] = csd.TreePlan(s["cache"], c["T"])
            csd.csd_tree_plan(parents, s["cache"], s["plan"], n_new=s["news"])
            if c["op"] == "tree":
                s["buf"] = csd.AttentionBuffers(s["cache"], c["T"], c["Hq"], tree=True)
            else:
                s["sum"] = torch.empty_like(s["mass"])
        return s
    if c["op"] == "path":
        chosen = _accepted(c)
        path = np.full((c["B"], c["T"]), -1, dtype=np.int32)
        for b, p in enumerate(chosen):
            path[b, :len(p)] = p
        s["path"], s["accept"] = torch.from_numpy(path).cuda(), torch.tensor([len(p) - 1 for p in chosen], dtype=torch.int32).cuda()
    else:
        # few places carry most of the weight
        s["mass"] = torch.exp(2.0 * torch.randn((c["B"], places), generator=gen, device="cuda"))
    if own:
        import paper_2604_13634_b200 as csd
        s["cache"] = _cache(c, s)
        if c["op"] == "path":
            s["cache"].granted.fill_(c["T"])
        else:
            s["buf"] = csd.EvictBuffers(s["cache"], c["keep"])
            s["sum"] = torch.empty_like(s["mass"])
        s["start"] = s["cache"].meta.clone()
    return s


def _prepare_verify(c, s, host):
    nodes, parents, paths = _walk(c)
    B, T, V = c["B"], c["T"], c["V"]
    gen = torch.Generator(device="cuda").manual_seed(int(host.integers(1 << 40)))
    z = torch.randn((B, T, V), generator=gen, device="cuda", dtype=DTYPES[c["dtype"]])
    tokens = np.stack([host.choice(V, T, replace=False) for _ in range(B)])
    top = host.integers(0, V, (B, T))  # the target's token after each node
    put, pairs = [], []  # (row, node, token, logit); (draft, target, count)
    for b, taken in enumerate(paths):
        drafted = set(tokens[b].tolist())
        for c_ in range(T):
            while top[b, c_] in drafted:
                top[b, c_] = host.integers(0, V)
        for at, node in enumerate(taken):
            below = [t for t in range(1, nodes[b]) if parents[b, t] == node]
            follows = taken[at + 1] if at + 1 < len(taken) else None
            if follows is not None and host.random() < 0.7:
                top[b, node] = tokens[b, follows]  # the target says it too
                continue
            for t in below:  # a divergence: pairs the memory has seen often or seldom, near the target's choice or far from it
                if t == follows:
                    pairs.append((tokens[b, t], top[b, node], LAMBDA + int(host.integers(0, 50))))
                    put.append((b, node, tokens[b, t], 12.0 - 0.25))
                elif host.random() < 0.5:
                    pairs.append((tokens[b, t], top[b, node], int(host.integers(LAMBDA, 50))))
                else:
                    pairs.append((tokens[b, t], top[b, node], int(host.integers(1, LAMBDA))))
                    put.append((b, node, tokens[b, t], 12.0 - 1.0))
    bs, ns = np.divmod(np.arange(B * T), T)
    index = np.array([(b, n, v) for b, n, v, _ in put], dtype=np.int64).reshape(-1, 3)
    rows = torch.from_numpy(np.concatenate([np.stack([bs, ns, top.reshape(-1)], 1), index])).cuda()
    values = torch.tensor([12.0] * (B * T) + [x for *_, x in put], device="cuda", dtype=z.dtype)
    z[rows[:, 0], rows[:, 1], rows[:, 2]] = values
    merged = {}
    for d, t, n in pairs + [(int(d), int(t), 9) for d, t in host.integers(0, V, (1000, 2))]:
        merged[(int(d), int(t))] = max(n, merged.get((int(d), int(t)), 0))
    known = sorted(merged)
    s["logits"], s["tokens"] = z, torch.from_numpy(tokens.astype(np.int32)).cuda()
    s["parents"], s["nodes"] = torch.from_numpy(parents.astype(np.int32)).cuda(), torch.tensor(nodes, dtype=torch.int32).cuda()
    s["keys"] = torch.tensor([(d << 32) + t for d, t in known], dtype=torch.int64).cuda()
    s["counts"] = torch.tensor([merged[x] for x in known], dtype=torch.int32).cuda()
    if own:
        import paper_2604_13634_b200 as csd
        s["ocm"] = csd.Ocm(1 << 16, lam=LAMBDA)
        d, t = (torch.tensor(x, dtype=torch.int32, device="cuda") for x in zip(*known))
        s["ocm"].import_(d, t, s["counts"])
        s["buf"] = csd.TreeBuffers(B, T)
    return s


# ---- the operators in plain form -------------------------------------------------------------------------------

def _visible(s, size):
    """[B, T, size] bool: which places each new token sees."""
    c = s["case"]
    j, t = torch.arange(size, device="cuda"), torch.arange(c["T"], device="cuda")
    first = (s["lens"] - s["news"])[:, None, None]
    there = t < s["news"][:, None]
    new = s["seen"].gather(2, (j - first).clamp(0, c["T"] - 1).expand(-1, c["T"], -1)) & (j >= first) & (j < s["lens"][:, None, None])
    return ((j < first) | new) & there[:, :, None]


def _scores(s, q, size):
    """[B, Hkv, T, group, size] scale q.k in 32 bits."""
    c = s["case"]
    group = c["Hq"] // c["Hkv"]
    q = q.float().reshape(c["B"], c["T"], c["Hkv"], group, c["D"]).permute(0, 2, 1, 3, 4).flatten(2, 3)
    return (torch.matmul(q, _gathered(s, "k", size).transpose(2, 3)) * c["D"] ** -0.5).unflatten(2, (c["T"], group))


def _gathered(s, which, size):
    """[B, Hkv, size, D] in 32 bits."""
    c = s["case"]
    return s[which][0][s["table"].clamp(min=0).long()].permute(0, 2, 1, 3, 4).reshape(c["B"], c["Hkv"], size, c["D"]).float()


def _tree(s):
    c = s["case"]
    size = s["table"].shape[1] * c["page"]
    x = _scores(s, s["q"], size).masked_fill_(~_visible(s, size)[:, None, :, None], -math.inf)
    m = x.amax(-1, keepdim=True)
    p = x.sub_(m.clamp(min=-1e30)).exp_()
    total = p.sum(-1, keepdim=True)
    v = _gathered(s, "v", size).masked_fill_((torch.arange(size, device="cuda") >= s["lens"][:, None])[:, None, :, None], 0.0)
    out = torch.matmul(p.flatten(2, 3), v).unflatten(2, (c["T"], -1)) / total.clamp(min=1e-30)
    back = lambda y: y.permute(0, 2, 1, 3, 4).flatten(2, 3)  # noqa: E731
    return back(out).to(s["q"].dtype), back(m + total.log())[..., 0]


def _mass(s):
    c = s["case"]
    size = s["mass"].shape[1]
    lse = s["lse"].reshape(c["B"], c["T"], c["Hkv"], -1).permute(0, 2, 1, 3)[..., None]
    there = _visible(s, size)[:, None, :, None] & (lse > -math.inf)
    given = _scores(s, s["q"], size).sub_(lse).masked_fill_(~there, -math.inf).exp_().sum((1, 2, 3))
    j = torch.arange(size, device="cuda")
    if c["fresh"]:
        begun = (j >= (s["lens"] - s["news"])[:, None]) & (j < s["lens"][:, None]) & (s["news"][:, None] > 0)
        return s["mass"].masked_fill(begun, 0.0) + given
    return s["mass"] + given


def _verify(s):
    c = s["case"]
    z, tokens, parents, n = s["logits"].float(), s["tokens"].long(), s["parents"].clamp(min=0).long(), s["nodes"][:, None]
    t = torch.arange(c["T"], device="cuda")
    m = z.amax(-1)
    star = torch.where(z == m[..., None], torch.arange(c["V"], device="cuda", dtype=torch.int32), c["V"]).amin(-1).long()
    there = (t > 0) & (t < n)
    said, best = star.gather(1, parents), m.gather(1, parents)
    zd = z[torch.arange(c["B"], device="cuda")[:, None], parents, tokens]
    match = there & (tokens == said)
    key = (tokens << 32) + said
    at = torch.searchsorted(s["keys"], key).clamp(max=s["keys"].numel() - 1)
    often = (s["keys"][at] == key) & (s["counts"][at] >= LAMBDA)
    gate = float(np.float32(np.log(np.float64(np.float32(TAU)))))
    rescue = there & ~match & often & (zd.double() - best.double() >= gate)
    # child[b, p, t]: t is a child of p.  Of a node's children the match goes first, then the likeliest rescue; ties to the lowest
    child = (parents[:, None, :] == t[:, None]) & there[:, None, :]
    rank = torch.where(match, math.inf, torch.where(rescue, zd, -math.inf))[:, None, :].expand_as(child).masked_fill(~child, -math.inf)
    first = torch.where(rank == rank.amax(-1, keepdim=True), t, c["T"]).amin(-1)
    taken = (first.gather(1, parents) == t) & (match | rescue) | ((t == 0) & (n > 0))
    # on the path: taken, and all nodes above as well
    above = torch.linalg.matrix_power(child.transpose(1, 2).float() + torch.eye(c["T"], device="cuda"), c["T"]) > 0
    on = ~(above & ~taken[:, None, :]).any(-1) & (t < n)
    length = on.sum(1)
    path = torch.where(on, t, c["T"]).sort(1)[0]
    last = torch.where(on, t, -1).amax(1)
    agreed = (child & match[:, None, :]).any(-1)
    diverged = there & on.gather(1, parents) & ~agreed.gather(1, parents)
    i32 = lambda x: x.to(torch.int32)  # noqa: E731
    return (i32((length - 1).clamp(min=0)), i32(torch.where(last >= 0, star.gather(1, last.clamp(min=0)[:, None])[:, 0], -1)),
            i32(path.masked_fill(path == c["T"], -1)), (on & rescue).to(torch.uint8),
            i32(torch.where(diverged, tokens, -1)), i32(torch.where(diverged, said, -1)))


def _moved(s, table, src, dst, valid):
    """Tokens at places src [B, n] of their rows go to places dst, in every layer, where valid."""
    page = s["case"]["page"]
    rows, cols = valid.nonzero(as_tuple=True)
    a, b = src[rows, cols].long(), dst[rows, cols].long()
    from_, to = table[rows, a // page].long(), table[rows, b // page].long()
    for pool in (s["k"], s["v"]):
        pool[:, to, :, b % page] = pool[:, from_, :, a % page]


def _shortened(s, table, lens):
    """The bookkeeping of rows of these lengths."""
    cols = torch.arange(table.shape[1], device="cuda") * s["case"]["page"]
    kept = torch.where(cols < lens[:, None], table, -1)
    return kept, lens, torch.bincount(kept[kept >= 0].long(), minlength=s["n_pages"]).to(torch.int32)


def _path(s):
    c = s["case"]
    i = torch.arange(c["T"], device="cuda")
    base = s["lens"] - c["T"]
    _moved(s, s["table"], base[:, None] + s["path"], base[:, None] + i, (i <= s["accept"][:, None]) & (s["path"] != i))
    return *_shortened(s, s["table"], base + s["accept"] + 1), s["k"], s["v"]


def _evict(s):
    c = s["case"]
    size = s["mass"].shape[1]
    j, lens = torch.arange(size, device="cuda"), s["lens"][:, None]
    after = lens.clamp(max=c["keep"])
    recent = lens - c["recent"]  # from here on the tokens stay the last, in order
    there = j < lens
    value = torch.where((j < c["sinks"]) | (j >= recent), math.inf, s["mass"]).masked_fill(~there, -math.inf)
    order = value.sort(dim=1, descending=True, stable=True)[1]
    chosen = torch.zeros_like(there).scatter_(1, order, j.expand_as(there) < after)
    # of the others, those that lie beyond where the recent ones go fill the places that become free below it, both in order
    front = after - c["recent"]
    movers = torch.where(chosen & (j >= front) & (j < recent), j, size).sort(1)[0]
    hole = ~chosen & (j < front)
    filled = torch.where(hole, movers.gather(1, (hole.cumsum(1) - 1).clamp(min=0)), j)
    kept = torch.where((j >= front) & (lens > c["keep"]), recent + j - front, filled)[:, :c["keep"]]
    i = j[:c["keep"]]
    valid = i < after
    _moved(s, s["table"], kept, i.expand_as(kept), valid & (kept != i))
    mass = s["mass"].clone()
    mass[:, :c["keep"]] = torch.where(valid, mass.gather(1, kept.clamp(max=size - 1)), mass[:, :c["keep"]])
    mass = mass.masked_fill(there & (j >= after), 0.0)
    return *_shortened(s, s["table"], after[:, 0]), kept.masked_fill(~valid, -1).to(torch.int32), (lens - after)[:, 0], mass, s["k"], s["v"]


def run(s):
    c = s["case"]
    if own:
        return _run_own(c, s)
    return {"tree": _tree, "mass": _mass, "verify": _verify, "path": _path, "evict": _evict}[c["op"]](s)


def _run_own(c, s):
    import paper_2604_13634_b200 as csd
    if c["op"] == "verify":
        buf = s["buf"]
        csd.csd_verify_tree(s["logits"], s["tokens"], s["parents"], s["ocm"], TAU, buf, n_nodes=s["nodes"])
        return buf.accept_len, buf.next_token, buf.path, buf.rescued_mask, buf.rej_draft, buf.rej_target
    cache = s["cache"]
    if c["op"] == "tree":
        csd.csd_attention_tree(s["q"], cache, 0, s["buf"], s["plan"].masks, n_new=s["news"])
        return s["buf"].out, s["buf"].lse
    if c["op"] == "mass":
        s["sum"].copy_(s["mass"])  # the same weights before every pass
        csd.csd_attention_mass(s["q"], s["lse"], cache, 0, s["sum"], n_new=s["news"], masks=s["plan"].masks if c["tree"] else None, fresh=c["fresh"])
        return s["sum"]
    cache.meta.copy_(s["start"])  # the same tokens too many for every pass
    if c["op"] == "path":
        csd.csd_cache_commit_path(cache, s["accept"], s["path"])
        return cache.table, cache.lens, cache.refs, cache.k, cache.v
    s["sum"].copy_(s["mass"])
    csd.csd_cache_evict(cache, s["sum"], c["keep"], s["buf"], sinks=c["sinks"], recent=c["recent"])
    return cache.table, cache.lens, cache.refs, s["buf"].kept, s["buf"].evicted, s["sum"], cache.k, cache.v


# ---- the definitions in 64 bits --------------------------------------------------------------------------------

def exact(c, seed):
    global own
    if c["op"] not in ("tree", "mass"):
        return None  # whole numbers and copies
    kept, own = own, False
    try:
        s = prepare(c, seed)
    finally:
        own = kept
    lens, news, group = s["lens"].tolist(), s["news"].tolist(), c["Hq"] // c["Hkv"]
    sums = torch.zeros_like(s["mass"], dtype=torch.float64) if c["op"] == "mass" else None
    out = torch.zeros(s["q"].shape, dtype=torch.float64, device="cuda")
    lse = torch.full(s["q"].shape[:3], -math.inf, dtype=torch.float64, device="cuda")
    for b in range(c["B"]):
        n, base = news[b], lens[b] - news[b]
        if n == 0:
            continue
        ids = s["table"][b][:-(-lens[b] // c["page"])].long()
        unseen = torch.zeros((n, lens[b]), dtype=torch.bool, device="cuda")
        unseen[:, base:] = ~s["seen"][b, :n, :n]
        for h in range(c["Hkv"]):
            k, v = (s[x][0, ids, h].double().reshape(-1, c["D"])[:lens[b]] for x in "kv")
            mine = slice(h * group, (h + 1) * group)
            x = torch.einsum("tgd,jd->tgj", s["q"][b, :n, mine].double(), k) / math.sqrt(c["D"])
            if c["op"] == "mass":
                w = torch.exp(x - s["lse"][b, :n, mine].double()[..., None]).masked_fill(unseen[:, None], 0.0)
                sums[b, :lens[b]] += w.sum((0, 1))
                continue
            x = x.masked_fill(unseen[:, None], -math.inf)
            lse[b, :n, mine] = torch.logsumexp(x, -1)
            out[b, :n, mine] = torch.softmax(x, -1) @ v
    if c["op"] == "tree":
        return out.cpu(), lse.cpu()
    before = s["mass"].double()
    if c["fresh"]:
        for b in range(c["B"]):
            before[b, lens[b] - news[b]:lens[b]] = 0.0
    return (before + sums).cpu()
