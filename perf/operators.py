"""Timed cases of the decode-pass operators: rotary positions, attention over the paged cache, the cache's pages.

`own = False` computes each operator in elementary torch operations (32 bits, rounded once at the end);
`own = True` makes the package's calls on the same inputs.  `exact` states the operators a second time, in 64 bits.
"""

import math

import numpy as np
import torch

own = False

DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
BYTES = {"f32": 4, "bf16": 2, "f16": 2}


# ---- the cases -------------------------------------------------------------------------------------------------

def listed():
    rope = dict(op="rope", dtype="bf16", layout="half", scaling="none", factor=1.0, inverse=False, start=0)
    app = dict(op="append", dtype="bf16", layout="half", scaling="none", factor=1.0, ragged=False, token_major=False)
    att = dict(op="attention", dtype="bf16", ragged=False, token_major=False)
    return [
        # the queries of four prompts, as a target's prompt pass or a draft model's training step rotates them
        dict(rope, name="rope_prompt_bf16", B=4, S=4096, H=32, D=128, rot=128),
        # the gradient of the same operation in a training step in full precision: part of an odd-sized head, pairs side by
        # side, an odd length far into a context stretched four times
        dict(rope, name="rope_gradient_f32", B=2, S=1023, H=12, D=80, rot=32, dtype="f32", layout="interleaved", scaling="yarn",
             factor=4.0, inverse=True, start=20000),
        # one new token of one row: what every layer of a plain decode step writes; all latency
        dict(app, name="append_one_token", B=1, T=1, Hq=32, Hkv=8, D=128, rot=128, page=16, lo=700, hi=700),
        # eight drafted tokens and the last one, for 128 rows at once, tokens of a page side by side
        dict(app, name="append_batch", B=128, T=9, Hq=32, Hkv=8, D=128, rot=128, page=64, lo=200, hi=6000, layout="interleaved",
             scaling="parts", factor=8.0, token_major=True),
        # the smallest read: one token of one row with a short history; all latency
        dict(att, name="attend_one_short", B=1, T=1, Hq=32, Hkv=8, D=128, page=16, lo=700, hi=700),
        # one row, one token, a long context: the length has to be split
        dict(att, name="attend_one_long", B=1, T=1, Hq=32, Hkv=8, D=128, page=64, lo=131071, hi=131071),
        # one row's verification pass with eight drafted tokens, many query heads to a key head: 72 query rows to each key
        dict(att, name="attend_draft_wide", B=1, T=9, Hq=64, Hkv=8, D=128, page=16, lo=30001, hi=30001),
        # batched serving with five drafted tokens, ragged lengths and ragged drafts, empty rows among them
        dict(att, name="attend_draft_batch", B=32, T=6, Hq=40, Hkv=8, D=128, page=16, lo=0, hi=8191, ragged=True),
        # a large batch with eight drafted tokens
        dict(att, name="attend_large_batch", B=128, T=9, Hq=32, Hkv=8, D=128, page=64, lo=500, hi=4000),
        # a small draft model: one token, a key head to every query head, half precision, tokens of a page side by side
        dict(att, name="attend_heads_f16", B=16, T=1, Hq=16, Hkv=16, D=64, page=32, lo=0, hi=3000, dtype="f16", token_major=True),
        # a step of 16 searches of 4 beams each: rows continue another row's pages, get room for a token, and give it back
        dict(op="beams", name="pages_beams", groups=16, beams=4, layers=16, Hkv=8, D=128, page=16, lo=301, hi=2047, dtype="bf16"),
        # a pool with holes after many rows have left: the pages at the top move down
        dict(op="compact", name="pages_compact", rows=48, layers=8, Hkv=8, D=128, page=16, live=6000, moves=2500, n_pages=12000, dtype="bf16"),
    ]


def _spread(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _drawn(rng):
    op = rng.choice(["rope", "append", "attention", "attention", "attention", "beams", "compact"])
    heads = lambda: (lambda h, g: (h * g, h))(rng.choice([1, 2, 4, 8, 16]), rng.choice([1, 2, 3, 4, 5, 7, 8, 12, 16]))  # noqa: E731
    turn = lambda d: dict(layout=rng.choice(["half", "interleaved"]), rot=2 * rng.randint(d // 8, d // 2),  # noqa: E731
                          scaling=rng.choice(["none", "linear", "base", "parts", "yarn"]), factor=float(rng.choice([2, 4, 8, 32])))
    if op == "rope":
        d = 8 * rng.randint(4, 32)
        return dict(turn(d), op=op, dtype=rng.choice(["f32", "bf16", "f16"]), B=rng.randint(1, 8), S=_spread(rng, 1, 8192),
                    H=rng.randint(1, 40), D=d, inverse=rng.random() < 0.5, start=rng.choice([0, 0, _spread(rng, 1, 200000)]))
    page = rng.choice([16, 32, 64, 128])
    if op in ("append", "attention"):
        hq, hkv = heads()
        d = rng.choice([64, 64, 80, 96, 128, 128, 128, 256])
        b = _spread(rng, 1, 128)
        hi = _spread(rng, 16, 131072)
        lo = rng.choice([0, 1, hi // 2, hi])
        c = dict(op=op, dtype=rng.choice(["bf16", "bf16", "f16"]), B=b, T=rng.choice([1, 1, 2, 4, 5, 6, 7, 9, 16, 33]), Hq=hq, Hkv=hkv, D=d,
                 page=page, lo=lo, hi=hi, ragged=rng.random() < 0.5, token_major=rng.random() < 0.5)
        return dict(c, **turn(d)) if op == "append" else c
    hkv, d, layers = rng.choice([1, 2, 4, 8, 16]), rng.choice([64, 128]), rng.randint(1, 24)
    if op == "beams":
        hi = _spread(rng, page, 8192)
        return dict(op=op, groups=_spread(rng, 1, 64), beams=rng.randint(2, 8), layers=layers, Hkv=hkv, D=d, page=page, lo=rng.randint(1, hi),
                    hi=hi, dtype=rng.choice(["bf16", "f16"]))
    live = _spread(rng, 50, 20000)
    moves = _spread(rng, 1, live // 2)
    return dict(op=op, rows=rng.randint(1, 100), layers=layers, Hkv=hkv, D=d, page=page, live=live, moves=moves,
                n_pages=live + moves + rng.randint(0, live), dtype=rng.choice(["bf16", "f16"]))


def _pool_bytes(c):
    """Bytes of the key and value pages that a case holds."""
    one = 2 * c["Hkv"] * c["D"] * c["page"] * 2 * c.get("layers", 1)
    if c["op"] == "compact":
        return one * c["n_pages"]
    if c["op"] == "beams":
        return one * _beam_pages(c)
    return one * (sum(-(-(n + c["T"]) // c["page"]) for n in _lens(c)) * 5 // 4 + 4)


def draw(rng):
    most = {"beams": 1.5e9, "compact": 3e9, "append": 1.5e9, "attention": 1.4e9}
    top = max(work(c)["bytes"] for c in listed())
    flops = max(work(c)["flops"] for c in listed())
    while True:
        c = _drawn(rng)
        w = work(c)
        if w["bytes"] > top or w["flops"] > flops:
            continue
        if c["op"] != "rope" and _pool_bytes(c) > most[c["op"]]:
            continue
        if c["op"] == "attention" and (c["B"] * c["hi"] * c["Hq"] * c["T"] > 1.5e9 or c["B"] * c["hi"] * c["Hkv"] * c["D"] > 1.5e9):
            continue  # the padded 32-bit tensors of the plain form
        return c


def _lens(c):
    """Cached tokens of each row, the new ones among them: evenly from lo to hi."""
    b = c["B"]
    return [c["hi"]] if b == 1 else [round(c["lo"] + (c["hi"] - c["lo"]) * i / (b - 1)) for i in range(b)]


def _news(c):
    """New tokens of each row: T, or 1 .. T in turn; no more than there are."""
    return [min(n, 1 + i % c["T"] if c["ragged"] else c["T"]) for i, n in enumerate(_lens(c))]


def _beam_lens(c):
    """Tokens of each group's rows; the last page is never full, so that sharing it means copying it."""
    g = c["groups"]
    lens = [c["hi"]] if g == 1 else [round(c["lo"] + (c["hi"] - c["lo"]) * i / (g - 1)) for i in range(g)]
    return [n + 1 if n % c["page"] == 0 else n for n in lens]


def _beam_pages(c):
    return sum(-(-n // c["page"]) * c["beams"] for n in _beam_lens(c)) + 2 * c["groups"] * c["beams"]


def work(c):
    e = BYTES[c["dtype"]]
    if c["op"] == "rope":
        n = c["B"] * c["S"] * c["H"]
        return {"bytes": 2 * n * c["D"] * e + 4 * c["B"] * c["S"], "flops": 3 * n * c["rot"]}
    if c["op"] == "append":
        n = sum(_news(c))
        return {"bytes": (c["B"] * c["T"] * c["Hq"] + n * c["Hq"] + 4 * n * c["Hkv"]) * c["D"] * e, "flops": 3 * n * (c["Hq"] + c["Hkv"]) * c["rot"]}
    if c["op"] == "attention":
        lens, news = _lens(c), _news(c)
        rows = c["B"] * c["T"] * c["Hq"]
        seen = sum(t * n - t * (t - 1) // 2 for n, t in zip(lens, news))
        return {"bytes": 2 * sum(lens) * c["Hkv"] * c["D"] * e + 2 * rows * c["D"] * e + 4 * rows, "flops": 4 * c["Hq"] * c["D"] * seen}
    page = 2 * c["layers"] * c["Hkv"] * c["D"] * c["page"] * e
    if c["op"] == "beams":
        rows = c["groups"] * c["beams"]
        table = 4 * sum(-(-n // c["page"]) for n in _beam_lens(c)) * c["beams"]
        return {"bytes": 2 * c["groups"] * (c["beams"] - 1) * page + 2 * table + 12 * rows, "flops": rows}
    return {"bytes": 2 * c["moves"] * page + 12 * c["live"], "flops": c["live"]}


# ---- inputs ----------------------------------------------------------------------------------------------------

def _thetas(c):
    """Rotation per position of each pair, and the factor on the rotated values."""
    rot, f, base, trained = c["rot"], c["factor"], 10000.0, 8192.0
    i = np.arange(rot // 2, dtype=np.float64)
    th = base ** (-2.0 * i / rot)
    kind = c["scaling"]
    if kind == "linear":
        return th / f, 1.0
    if kind == "base":
        return (base * f ** (rot / max(rot - 2.0, 1.0))) ** (-2.0 * i / rot), 1.0
    if kind == "parts":  # by the turns that a pair makes within the trained length
        keep = np.clip((trained * th / (2 * np.pi) - 1.0) / (4.0 - 1.0), 0.0, 1.0)
        return th * keep + th / f * (1 - keep), 1.0
    if kind == "yarn":  # by the pair's index, between the pairs that make 32 turns and 1 turn within the trained length
        at = lambda turns: rot * math.log(trained / (turns * 2 * math.pi)) / (2 * math.log(base))  # noqa: E731
        lo, hi = max(math.floor(at(32.0)), 0), min(math.ceil(at(1.0)), rot - 1)
        far = np.clip((i - lo) / max(hi - lo, 0.001), 0.0, 1.0)
        return th * (1 - far) + th / f * far, 0.1 * math.log(f) + 1.0
    return th, 1.0


def _plan(c):
    """The rotations as 64-bit fractions of a turn: a product with a position wraps to the angle, exactly."""
    th, magnitude = _thetas(c)
    turns = [int(round(x / (2 * math.pi) * 2.0**64)) & (2**64 - 1) for x in th.tolist()]
    steps = torch.tensor([t - 2**64 if t >= 2**63 else t for t in turns], dtype=torch.int64, device="cuda")
    return steps, magnitude


def _rope_plan(c):
    import paper_2604_13634_b200 as csd
    return csd.RopePlan(c["rot"], base=10000.0, layout=c["layout"], scaling=c["scaling"], factor=c["factor"], original_len=8192)


def _pool(c, n_pages, layers, gen):
    """Key and value pages [layers, n_pages, heads, page, D], all of them with values of some row in them."""
    shape = (layers, n_pages, c["page"], c["Hkv"], c["D"]) if c.get("token_major") else (layers, n_pages, c["Hkv"], c["page"], c["D"])
    two = [torch.randn(shape, generator=gen, device="cuda", dtype=DTYPES[c["dtype"]]) for _ in range(2)]
    return [t.transpose(2, 3) if c.get("token_major") else t for t in two]


def _cache(c, s, n_pages, layers):
    """The package's handle on the pool, the table and the lengths in hand."""
    import paper_2604_13634_b200 as csd
    cache = csd.PagedCache(s["table"].shape[0], n_pages, c["page"], layers, c["Hkv"], c["D"], DTYPES[c["dtype"]],
                           s["table"].shape[1] * c["page"], k=s["k"], v=s["v"])
    cache.load(s["table"], s["lens"])
    s["cache"] = cache


def prepare(c, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    host = np.random.default_rng(seed)
    dt = DTYPES[c["dtype"]]
    s = {"case": c}
    if c["op"] == "rope":
        s["x"] = torch.randn((c["B"], c["S"], c["H"], c["D"]), generator=gen, device="cuda", dtype=dt)
        first = torch.tensor(host.integers(0, 1 + c["start"], c["B"]), dtype=torch.int32)
        s["positions"] = (first[:, None] + torch.arange(c["S"], dtype=torch.int32)).cuda()
        s["steps"], s["magnitude"] = _plan(c)
        if own:
            s["plan"] = _rope_plan(c)
            s["out"] = torch.empty_like(s["x"])
        return s
    if c["op"] in ("append", "attention"):
        order = host.permutation(c["B"])
        lens, news = np.array(_lens(c))[order], np.array(_news(c))[order]
        width = max(1, int(max(-(-n // c["page"]) for n in lens)))
        total = int(sum(-(-n // c["page"]) for n in lens))
        n_pages = total * 9 // 8 + 2
        ids = host.permutation(n_pages)[:total]
        table, at = np.full((c["B"], width), -1, dtype=np.int32), 0
        for b, n in enumerate(lens):
            m = -(-int(n) // c["page"])
            table[b, :m] = ids[at:at + m]
            at += m
        s["table"], s["lens"] = torch.from_numpy(table).cuda(), torch.tensor(lens, dtype=torch.int32).cuda()
        s["news"] = torch.tensor(news, dtype=torch.int32).cuda() if c["ragged"] else None
        s["k"], s["v"] = _pool(c, n_pages, 1, gen)
        if c["op"] == "append":
            qkv = torch.randn((c["B"], c["T"], c["Hq"] + 2 * c["Hkv"], c["D"]), generator=gen, device="cuda", dtype=dt)
            s["q"], s["new_k"], s["new_v"] = qkv.split([c["Hq"], c["Hkv"], c["Hkv"]], dim=2)
            s["steps"], s["magnitude"] = _plan(c)
        else:
            s["q"] = 2.0 * torch.randn((c["B"], c["T"], c["Hq"], c["D"]), generator=gen, device="cuda", dtype=dt)
        if own:
            import paper_2604_13634_b200 as csd
            _cache(c, s, n_pages, 1)
            if c["op"] == "append":
                s["plan"] = _rope_plan(c)
                s["q_out"] = torch.empty((c["B"], c["T"], c["Hq"], c["D"]), device="cuda", dtype=dt)
            else:
                s["buf"] = csd.AttentionBuffers(s["cache"], c["T"], c["Hq"])
        return s
    if c["op"] == "beams":
        lens, n_pages = _beam_lens(c), _beam_pages(c)
        rows, g = c["groups"] * c["beams"], c["beams"]
        width = max(-(-n // c["page"]) for n in lens) + 1
        ids, at = host.permutation(n_pages), 0
        table = np.full((rows, width), -1, dtype=np.int32)
        for r in range(rows):
            m = -(-lens[r // g] // c["page"])
            kept = m // 2 if r % g else 0  # the prompt's pages are the group's first row's
            table[r, :kept] = table[r - r % g, :kept]
            table[r, kept:m] = ids[at:at + m - kept]
            at += m - kept
        s["parent"] = torch.tensor(np.repeat(np.arange(c["groups"]) * g + host.integers(0, g, c["groups"]), g), dtype=torch.int32).cuda()
        s["lens"] = torch.tensor(np.repeat(lens, g), dtype=torch.int32).cuda()
        s["back"] = s["lens"].clone()
    else:
        n_pages, live = c["n_pages"], c["live"]
        low = host.permutation(live)[:live - c["moves"]]
        ids = host.permutation(np.concatenate([low, live + host.permutation(n_pages - live)[:c["moves"]]]))
        cuts = live * np.arange(c["rows"] + 1) * (np.arange(c["rows"] + 1) + 1) // (c["rows"] * (c["rows"] + 1))
        counts = np.diff(cuts)  # rows of all lengths, from nearly none to the longest
        table = np.full((c["rows"], max(1, int(counts.max()))), -1, dtype=np.int32)
        for r, n in enumerate(counts):
            table[r, :n] = ids[cuts[r]:cuts[r + 1]]
        s["lens"] = torch.tensor(counts * c["page"], dtype=torch.int32).cuda()
    s["table"] = torch.from_numpy(table).cuda()
    s["refs"] = torch.bincount(s["table"][s["table"] >= 0].long(), minlength=n_pages).to(torch.int32)
    s["k"], s["v"] = _pool(c, n_pages, c["layers"], gen)
    if own:
        _cache(c, s, n_pages, c["layers"])
        s["holes"] = s["cache"].meta.clone()
    else:
        s["start"] = {x: s[x].clone() for x in ("table", "refs")}
    return s


# ---- the operators in plain form -------------------------------------------------------------------------------

def _rotated(x, positions, steps, magnitude, layout, inverse=False):
    """x [..., tokens, heads, D] by the angles of positions [..., tokens]."""
    rot = 2 * steps.numel()
    phase = positions.long()[..., None] * steps
    angle = (phase >> 32).float() * (2 * math.pi / 2.0**32)
    c, s = (angle.cos() * magnitude)[..., None, :], (angle.sin() * magnitude)[..., None, :]
    if inverse:
        s = -s
    y = x.float()
    if layout == "half":
        a, b = y[..., :rot // 2], y[..., rot // 2:rot]
        turned = torch.cat([a * c - b * s, b * c + a * s], dim=-1)
    else:
        a, b = y[..., 0:rot:2], y[..., 1:rot:2]
        turned = torch.stack([a * c - b * s, b * c + a * s], dim=-1).flatten(-2)
    return torch.cat([turned, y[..., rot:]], dim=-1).to(x.dtype)


def _append(s):
    c = s["case"]
    t = torch.arange(c["T"], device="cuda")
    news = torch.full_like(s["lens"], c["T"]) if s["news"] is None else s["news"]
    at = (s["lens"] - news)[:, None] + t  # place of each token in its row
    fine = (t < news[:, None]) & (at >= 0)
    q = _rotated(s["q"], at, s["steps"], s["magnitude"], c["layout"])
    k = _rotated(s["new_k"], at, s["steps"], s["magnitude"], c["layout"])
    rows, cols = fine.nonzero(as_tuple=True)
    place = at[rows, cols].long()
    pages = s["table"][rows, place // c["page"]].long()
    s["k"][0][pages, :, place % c["page"]] = k[rows, cols]
    s["v"][0][pages, :, place % c["page"]] = s["new_v"][rows, cols]
    return q.masked_fill(~fine[:, :, None, None], 0.0), s["k"], s["v"]


def _attention(s):
    c = s["case"]
    group = c["Hq"] // c["Hkv"]
    size = s["table"].shape[1] * c["page"]
    j = torch.arange(size, device="cuda")
    t = torch.arange(c["T"], device="cuda")
    news = torch.full_like(s["lens"], c["T"]) if s["news"] is None else s["news"]
    last = torch.where(t < news[:, None], (s["lens"] - news)[:, None] + t, -1)  # last place that each token sees
    gather = lambda pool: pool[0][s["table"].clamp(min=0).long()].permute(0, 2, 1, 3, 4).reshape(c["B"], c["Hkv"], size, c["D"])  # noqa: E731
    q = s["q"].float().reshape(c["B"], c["T"], c["Hkv"], group, c["D"]).permute(0, 2, 1, 3, 4).flatten(2, 3)
    x = torch.matmul(q, gather(s["k"]).float().transpose(2, 3)) * c["D"] ** -0.5
    x = x.unflatten(2, (c["T"], group)).masked_fill_((j > last[:, :, None])[:, None, :, None], -math.inf)
    m = x.amax(-1, keepdim=True)
    p = (x - m.clamp(min=-1e30)).exp_()
    total = p.sum(-1, keepdim=True)
    v = gather(s["v"]).float().masked_fill_((j >= s["lens"][:, None])[:, None, :, None], 0.0)
    out = torch.matmul(p.flatten(2, 3), v).unflatten(2, (c["T"], group)) / total.clamp(min=1e-30)
    back = lambda y: y.permute(0, 2, 1, 3, 4).flatten(2, 3)  # noqa: E731
    return back(out).to(s["q"].dtype), back(m + total.log())[..., 0]


def _counted(table, n_pages):
    return torch.bincount(table[table >= 0].long(), minlength=n_pages).to(torch.int32)


def _beams(s):
    c = s["case"]
    page, rows, width = c["page"], s["table"].shape[0], s["table"].shape[1]
    # every row continues its parent's pages
    table, lens = s["table"][s["parent"].long()], s["lens"][s["parent"].long()]
    refs = _counted(table, s["refs"].numel())
    # room for one token: a shared last page is copied first, except by the last row that still has it
    r = torch.arange(rows, device="cuda")
    held = (lens + page - 1) // page
    tail = torch.where(lens % page > 0, table[r, (held - 1).clamp(min=0).long()], -1)
    before = ((tail[:, None] == tail) & (r[:, None] > r)).sum(1)
    copied = (tail >= 0) & (refs[tail.clamp(min=0).long()] - before > 1)
    cols = torch.arange(width, device="cuda")
    wanted = (cols >= held[:, None]) & (cols < ((lens + page) // page)[:, None]) | copied[:, None] & (cols == held[:, None] - 1)
    free = (refs == 0).nonzero()[:, 0]
    fresh = torch.where(wanted, free[(wanted.flatten().cumsum(0) - 1).clamp(min=0)].view(rows, width).int(), table)
    source, target = tail[copied].long(), fresh[r, (held - 1).clamp(min=0).long()][copied].long()
    for pool in (s["k"], s["v"]):
        pool[:, target] = pool[:, source]
    # and the room is given back
    lens = torch.minimum(lens + 1, s["back"])
    table = torch.where(cols < ((lens + page - 1) // page)[:, None], fresh, -1)
    s["table"], s["lens"], s["refs"] = table, lens, _counted(table, refs.numel())
    return s["table"], s["lens"], s["refs"], s["k"], s["v"]


def _compact(s):
    table, refs = s["start"]["table"], s["start"]["refs"]
    live = refs > 0
    n = int(live.sum())
    low, high = (~live[:n]).nonzero()[:, 0], live[n:].nonzero()[:, 0] + n
    to = torch.arange(refs.numel(), device="cuda", dtype=torch.int32)
    to[high] = low.int()
    for pool in (s["k"], s["v"]):
        pool[:, low] = pool[:, high]
    moved = refs.clone()
    moved[low], moved[high] = refs[high], 0
    return torch.where(table >= 0, to[table.clamp(min=0).long()], -1), s["lens"], moved, s["k"], s["v"]


def run(s):
    c = s["case"]
    if own:
        return _run_own(c, s)
    if c["op"] == "rope":
        return _rotated(s["x"], s["positions"], s["steps"], s["magnitude"], c["layout"], c["inverse"])
    return {"append": _append, "attention": _attention, "beams": _beams, "compact": _compact}[c["op"]](s)


def _run_own(c, s):
    import paper_2604_13634_b200 as csd
    if c["op"] == "rope":
        return csd.csd_rope(s["x"], s["positions"], s["plan"], out=s["out"], inverse=c["inverse"])
    cache = s["cache"]
    if c["op"] == "append":
        csd.csd_rope_append(s["q"], s["new_k"], s["new_v"], cache, 0, s["plan"], q_out=s["q_out"], n_new=s["news"])
        return s["q_out"], cache.k, cache.v
    if c["op"] == "attention":
        csd.csd_attention(s["q"], cache, 0, s["buf"], n_new=s["news"])
        return s["buf"].out, s["buf"].lse
    if c["op"] == "beams":
        csd.csd_cache_fork(cache, s["parent"])
        csd.csd_cache_extend(cache, 1)
        csd.csd_cache_truncate(cache, s["back"])
    else:
        cache.meta.copy_(s["holes"])  # the same holes for every pass: the pages above are still what they were
        csd.csd_cache_compact(cache)
    return cache.table, cache.lens, cache.refs, cache.k, cache.v


# ---- the definitions in 64 bits --------------------------------------------------------------------------------

def _turned64(x, positions, c, sign):
    """x [n, heads, D] as complex numbers turned by positions [n]."""
    th, magnitude = _thetas(c)
    a = positions.double()[:, None] * torch.from_numpy(th).cuda()
    w = torch.polar(torch.full_like(a, magnitude), sign * a)[:, None]
    y = x.double().clone()
    r = c["rot"]
    first, second = (slice(0, r // 2), slice(r // 2, r)) if c["layout"] == "half" else (slice(0, r, 2), slice(1, r, 2))
    z = torch.complex(y[..., first], y[..., second]) * w
    y[..., first], y[..., second] = z.real, z.imag
    return y


def exact(c, seed):
    global own
    if c["op"] in ("beams", "compact"):
        return None  # whole numbers and copies
    kept, own = own, False
    try:
        s = prepare(c, seed)
    finally:
        own = kept
    if c["op"] == "rope":
        return torch.stack([_turned64(x, p, c, -1.0 if c["inverse"] else 1.0) for x, p in zip(s["x"], s["positions"])]).cpu()
    lens = s["lens"].tolist()
    news = [c["T"]] * c["B"] if s["news"] is None else s["news"].tolist()
    if c["op"] == "append":
        q, k, v = torch.zeros(s["q"].shape, dtype=torch.float64, device="cuda"), s["k"].double(), s["v"].double()
        for b in range(c["B"]):
            for t in range(max(0, news[b] - lens[b]), news[b]):
                at = lens[b] - news[b] + t
                where = torch.tensor([at], device="cuda")
                page = int(s["table"][b, at // c["page"]])
                q[b, t] = _turned64(s["q"][b, t:t + 1], where, c, 1.0)[0]
                k[0, page, :, at % c["page"]] = _turned64(s["new_k"][b, t:t + 1], where, c, 1.0)[0]
                v[0, page, :, at % c["page"]] = s["new_v"][b, t].double()
        return q, k, v
    out = torch.zeros(s["q"].shape, dtype=torch.float64, device="cuda")
    lse = torch.full(s["q"].shape[:3], -math.inf, dtype=torch.float64, device="cuda")
    group = c["Hq"] // c["Hkv"]
    for b in range(c["B"]):
        ids = s["table"][b][:-(-lens[b] // c["page"])].long()
        if not len(ids):
            continue
        for h in range(c["Hkv"]):
            k, v = (s[x][0, ids, h].double().reshape(-1, c["D"]) for x in "kv")
            mine = slice(h * group, (h + 1) * group)
            seen = [max(0, lens[b] - news[b] + t + 1) if t < news[b] else 0 for t in range(c["T"])]
            if min(seen) == max(seen):  # one token, or nothing to see
                seen, tokens = seen[:1], [slice(0, c["T"])]
            else:
                tokens = [slice(t, t + 1) for t in range(c["T"])]
            for n, ts in zip(seen, tokens):
                if n > 0:
                    x = (s["q"][b, ts, mine].double() @ k[:n].T) / math.sqrt(c["D"])
                    lse[b, ts, mine] = torch.logsumexp(x, -1)
                    out[b, ts, mine] = torch.softmax(x, -1) @ v[:n]
    return out.cpu(), lse.cpu()
