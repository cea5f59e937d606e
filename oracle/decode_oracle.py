"""Plain 64-bit statements of the decode-pass operators (test infrastructure only): rotary positions, the paged cache's
bookkeeping taken row by row, attention over a row's tokens.  Shares no code with the CUDA path."""

import math

import numpy as np


# ---- rotary positions ----

def thetas(rot, base=10000.0, scaling="none", factor=1.0, original_len=8192.0, low=None, high=None):
    """([rot/2] rotation per position in radians, factor on turned elements)."""
    i = np.arange(rot // 2, dtype=np.float64)
    th = base ** (-2.0 * i / rot)
    if scaling == "none":
        return th, 1.0
    if scaling == "linear":
        return th / factor, 1.0
    if scaling == "base":
        grown = base * factor ** (rot / (rot - 2)) if rot > 2 else base
        return grown ** (-2.0 * i / rot), 1.0
    if scaling == "parts":
        low, high = low or 1.0, high or 4.0
        turns = original_len / (2 * math.pi / th)
        mix = (turns - low) / (high - low)
        return np.where(turns <= low, th / factor, np.where(turns >= high, th, mix * th + (1 - mix) * th / factor)), 1.0
    assert scaling == "yarn"
    low, high = low or 1.0, high or 32.0
    pair_with = lambda turns: rot / 2 * math.log(original_len / (2 * math.pi * turns), base)  # noqa: E731
    a, b = max(0, math.floor(pair_with(high))), min(rot - 1, math.ceil(pair_with(low)))
    ramp = np.array([min(1.0, max(0.0, (x - a) / max(b - a, 0.001))) for x in i])
    return th / factor * ramp + th * (1 - ramp), 1 + 0.1 * math.log(factor)


def rope(x, positions, th, magnitude=1.0, layout="half", inverse=False):
    """x [..., H, D] (positions [...]) -> the same shape, float64."""
    x = np.asarray(x, dtype=np.float64)
    rot = 2 * len(th)
    a = np.asarray(positions, dtype=np.float64)[..., None] * th * (-1.0 if inverse else 1.0)
    y = x.copy()
    for i in range(rot // 2):
        j0, j1 = (i, i + rot // 2) if layout == "half" else (2 * i, 2 * i + 1)
        c, s = magnitude * np.cos(a[..., i])[..., None], magnitude * np.sin(a[..., i])[..., None]
        y[..., j0] = x[..., j0] * c - x[..., j1] * s
        y[..., j1] = x[..., j1] * c + x[..., j0] * s
    return y


# ---- the paged cache ----

class Cache:
    """Page tables as Python lists; one row, one page at a time."""

    def __init__(self, rows, n_pages, page, max_pages):
        self.n_pages, self.page, self.max_pages = n_pages, page, max_pages
        self.tables = [[] for _ in range(rows)]
        self.lens = [0] * rows
        self.granted = [0] * rows
        self.full = self.row_full = False

    def refs(self):
        n = [0] * self.n_pages
        for t in self.tables:
            for p in t:
                n[p] += 1
        return n

    def table(self):
        out = np.full((len(self.tables), self.max_pages), -1, dtype=np.int32)
        for r, t in enumerate(self.tables):
            out[r, :len(t)] = t
        return out

    def extend(self, news):
        """Returns the page copies (source, destination) in order."""
        tables, lens, refs, copies = [list(t) for t in self.tables], list(self.lens), self.refs(), []
        free = [p for p in range(self.n_pages) if refs[p] == 0]
        news = [max(0, n) for n in news]
        self.granted = [0] * len(lens)
        if any(n > 0 and self.lens[r] + n > self.max_pages * self.page for r, n in enumerate(news)):
            self.row_full = True
            return []
        for r, n in enumerate(news):
            if n == 0:
                continue
            if lens[r] % self.page and refs[tables[r][-1]] > 1:
                if not free:
                    self.full = True
                    return []
                src, dst = tables[r][-1], free.pop(0)
                refs[src] -= 1
                refs[dst] = 1
                tables[r][-1] = dst
                copies.append((src, dst))
            lens[r] += n
            while len(tables[r]) * self.page < lens[r]:
                if not free:
                    self.full = True
                    return []
                tables[r].append(free.pop(0))
                refs[tables[r][-1]] = 1
        self.tables, self.lens, self.granted = tables, lens, news
        return copies

    def truncate(self, new_lens):
        for r, n in enumerate(new_lens):
            self.lens[r] = min(self.lens[r], max(0, n))
            del self.tables[r][-(-self.lens[r] // self.page):]
        self.granted = [0] * len(self.lens)

    def commit(self, accept):
        self.truncate([n - g + min(g, max(a, -1) + 1) for n, g, a in zip(self.lens, self.granted, accept)])

    def fork(self, parent):
        rows = range(len(self.tables))
        parent = [r if parent[r] >= len(self.tables) else parent[r] for r in rows]
        self.tables, self.lens = [list(self.tables[p]) if p >= 0 else [] for p in parent], [self.lens[p] if p >= 0 else 0 for p in parent]
        self.granted = [0] * len(self.lens)

    def compact(self):
        """Returns the moves (source, destination)."""
        refs = self.refs()
        n = sum(c > 0 for c in refs)
        moves = list(zip([p for p in range(n, self.n_pages) if refs[p]], [p for p in range(n) if not refs[p]]))
        to = dict(moves)
        self.tables = [[to.get(p, p) for p in t] for t in self.tables]
        return moves


def rows_of(pool, table, n_tokens, page):
    """Tokens 0 .. n-1 of a row from a layer's pages [n_pages, heads, page, D] -> [heads, n, D]."""
    if n_tokens == 0:
        return np.zeros((pool.shape[1], 0, pool.shape[3]))
    got = np.concatenate([pool[table[i]] for i in range(-(-n_tokens // page))], axis=1)
    return got[:, :n_tokens]


# ---- attention ----

def attention(q, k, v, n_new, scale):
    """One row: q [T, Hq, D], k, v [Hkv, n, D] with the new tokens last -> out [T, Hq, D], lse [T, Hq], and
    reach [T, Hq, D] = sum_j w_j |v_j|, size [T, Hq] = max_j sum_d |scale q_d k_jd| (for error bounds)."""
    T, Hq, D = q.shape
    group = Hq // k.shape[0]
    n = k.shape[1]
    out, reach = np.zeros((T, Hq, D)), np.zeros((T, Hq, D))
    lse, size = np.full((T, Hq), -np.inf), np.zeros((T, Hq))
    for t in range(T):
        last = n - n_new + t
        if t >= n_new or last < 0:
            continue
        for h in range(Hq):
            kk, vv = k[h // group, :last + 1], v[h // group, :last + 1]
            s = scale * (kk @ q[t, h])
            m = s.max()
            w = np.exp(s - m)
            lse[t, h] = m + math.log(w.sum())
            w /= w.sum()
            out[t, h] = w @ vv
            reach[t, h] = w @ np.abs(vv)
            size[t, h] = abs(scale) * (np.abs(kk) @ np.abs(q[t, h])).max()
    return out, lse, reach, size
