"""Plain 64-bit statements of the tree form of a verification pass and of a cache kept to a budget (test infrastructure only), one row,
one node, one place at a time.  Shares no code with the CUDA path."""

import math

import numpy as np


def plan(parents, n_new, base, offset=0):
    """One row: parents [T] -> (masks: T ints of 64 bits, positions [T])."""
    masks, depths = [], []
    for t, p in enumerate(parents):
        if t >= n_new:
            masks.append(0)
            depths.append(None)
        elif 0 <= p < t:
            masks.append(masks[p] | 1 << t)
            depths.append(depths[p] + 1)
        else:
            masks.append(1 << t)
            depths.append(0)
    return masks, [0 if d is None else base + offset + d for d in depths]


def sees(mask, n_new, n, t):
    """Places of a row of n tokens, n_new of them new, that its new token t sees."""
    first = n - n_new
    if t >= n_new or first + t < 0:
        return []
    return list(range(0, max(first, 0))) + [first + u for u in range(min(64, n_new)) if mask >> u & 1 and 0 <= first + u < n]


def attention(q, k, v, masks, n_new, scale):
    """One row: q [T, Hq, D], k, v [Hkv, n, D] -> out, lse, and (for error bounds) reach = sum_j w_j |v_j|, size = max_j sum_d |scale q k|."""
    T, Hq, D = q.shape
    group, n = Hq // k.shape[0], k.shape[1]
    out, reach = np.zeros((T, Hq, D)), np.zeros((T, Hq, D))
    lse, size = np.full((T, Hq), -np.inf), np.zeros((T, Hq))
    for t in range(T):
        at = sees(masks[t], n_new, n, t)
        if not at:
            continue
        for h in range(Hq):
            kk, vv = k[h // group, at], v[h // group, at]
            s = scale * (kk @ q[t, h])
            m = s.max()
            w = np.exp(s - m)
            lse[t, h] = m + math.log(w.sum())
            w /= w.sum()
            out[t, h] = w @ vv
            reach[t, h] = w @ np.abs(vv)
            size[t, h] = abs(scale) * (np.abs(kk) @ np.abs(q[t, h])).max()
    return out, lse, reach, size


def mass(q, k, lse, masks, n_new, scale, before, fresh):
    """One row: the places' weights after the call, [n], and a bound's ingredients: sum of the weights, largest sum_d |scale q k| + |lse|."""
    T, Hq, D = q.shape
    group, n = Hq // k.shape[0], k.shape[1]
    out, size = np.array(before[:n], dtype=np.float64), 0.0
    if fresh and n_new > 0:
        out[max(n - n_new, 0):] = 0.0
    for t in range(T):
        at = sees(masks[t], n_new, n, t)
        for h in range(Hq):
            if not at or lse[t, h] == -np.inf:
                continue
            kk = k[h // group, at]
            out[at] += np.exp(scale * (kk @ q[t, h]) - lse[t, h])
            size = max(size, float((abs(scale) * (np.abs(kk) @ np.abs(q[t, h]))).max() + abs(lse[t, h])))
    return out, size


# ---- verification ----

def verify(z, tokens, parents, n_nodes, counts, lam, threshold):
    """One row: z [T, V]; counts: dict (draft, target) -> count.  Returns accept_len, next_token, path, rescued nodes, records {node: pair}."""
    T, V = z.shape
    n = min(n_nodes, T)
    if n <= 0:
        return 0, -1, [], set(), {}
    cur, path, rescued, records = 0, [0], set(), {}
    while True:
        star = int(np.flatnonzero(z[cur] == z[cur].max())[0])
        below = [t for t in range(cur + 1, n) if parents[t] == cur]
        match = [t for t in below if tokens[t] == star]
        if match:
            nxt = match[0]
        else:
            nxt, best = None, None
            for t in below:
                d = int(tokens[t])
                if not 0 <= d < V:
                    continue
                records[t] = (d, star)
                if counts.get((d, star), 0) >= lam and float(z[cur, d]) - float(z[cur, star]) >= threshold and (best is None or z[cur, d] > best):
                    nxt, best = t, z[cur, d]
            if nxt is not None:
                rescued.add(nxt)
        if nxt is None:
            return len(path) - 1, star, path, rescued, records
        path.append(nxt)
        cur = nxt


# ---- the cache: contents as well as bookkeeping, one Python list of tokens per row ----

def kept_of_path(granted, accept, path):
    """How many of the granted tokens stay, and where among them they were."""
    keep = min(granted, max(accept, -1) + 1)
    out = []
    for i in range(keep):
        if i >= len(path) or not 0 <= path[i] < granted or (out and path[i] <= out[-1]):
            return out, True
        out.append(int(path[i]))
    return out, False


def evict(mass, n, keep, sinks, recent):
    """One row of n tokens: the place before of every place after."""
    keep = max(keep, 0)
    if n <= keep:
        return list(range(n))
    recent = min(max(recent, 0), keep)
    sinks = min(max(sinks, 0), keep - recent)
    value = [float(x) for x in mass[:n]]
    below_all = [math.isnan(x) for x in value]                         # NaN is smaller than minus infinity
    middle = sorted(range(sinks, n - recent), key=lambda j: (below_all[j], 0.0 if below_all[j] else -value[j], j))[:keep - recent - sinks]
    chosen = set(range(sinks)) | set(middle)
    front = keep - recent
    movers = iter(sorted(j for j in chosen if j >= front))
    return [j if j in chosen else next(movers) for j in range(front)] + list(range(n - recent, n))
