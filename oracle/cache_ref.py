"""Plain 64-bit reference of the operators on the paged cache, token by token in
numpy from their definitions (test infrastructure only; it shares no code with
the library).  Arrays are float64; caches [pages, heads, page_size, D]."""
import numpy as np


def lines(parent, n):
    """Nodes 0 .. n-1: each with its ancestors, root first, itself last; None
    for an invalid tree.  parent None: a chain."""
    out = []
    for i in range(n):
        up = i - 1 if parent is None else int(parent[i])
        if i and not 0 <= up < i:
            return None
        out.append((out[up] if i else []) + [i])
    return out


def place(table, pages, page_size, j):
    """(page, slot) of token j, None outside the table or the cache."""
    at = j // page_size
    if j < 0 or at >= len(table) or not 0 <= table[at] < pages:
        return None
    return int(table[at]), j % page_size


def rotate(x, turn, pairs):
    """x [heads, D], turn [R]: R/2 cosines, R/2 sines."""
    R = len(turn)
    c, s = turn[:R // 2], turn[R // 2:]
    y = x.copy()
    a, b = (slice(0, R, 2), slice(1, R, 2)) if pairs else (slice(0, R // 2), slice(R // 2, R))
    y[:, a] = x[:, a] * c - x[:, b] * s
    y[:, b] = x[:, b] * c + x[:, a] * s
    return y


def append(q, k, v, k_cache, v_cache, table, seq_len, rotation=None, pairs=False, parent=None, new_len=None):
    """Returns q_out, k_cache, v_cache (copies)."""
    B, N = k.shape[:2]
    P, H, S, D = k_cache.shape
    kc, vc, out = k_cache.copy(), v_cache.copy(), np.zeros_like(q)
    for b in range(B):
        c, n = int(seq_len[b]), N if new_len is None else int(new_len[b])
        if c < 0:
            continue
        if not 0 <= n <= N:
            out[b] = np.nan
            continue
        tree = lines(None if parent is None else parent[b], n) if parent is not None else None
        for i in range(n):
            at = place(table[b], P, S, c + i)
            pos = None
            if parent is None:
                pos = c + i
            elif tree is not None:
                pos = c + len(tree[i]) - 1
            if at is None or pos is None or (rotation is not None and pos >= len(rotation)):
                out[b, i] = np.nan
                continue
            turn = rotation[pos] if rotation is not None else np.zeros(0)
            out[b, i] = rotate(q[b, i], turn, pairs)
            kc[at[0], :, at[1]] = rotate(k[b, i], turn, pairs)
            vc[at[0], :, at[1]] = v[b, i]
    return out, kc, vc


def attention(q, k_cache, v_cache, table, seq_len, scale, parent=None, new_len=None):
    """Returns out, and for each row what bounds its rounding errors: the sums
    p |v| [.., D], and the largest scale sum |q| |k| over its keys."""
    B, N, Hq, D = q.shape
    P, H, S = k_cache.shape[:3]
    out, mass, reach = np.zeros(q.shape), np.zeros(q.shape), np.zeros(q.shape[:3])
    for b in range(B):
        c, n = int(seq_len[b]), N if new_len is None else int(new_len[b])
        if c < 0:
            continue
        if not 0 <= n <= N:
            out[b] = np.nan
            continue
        tree = lines(None if parent is None else parent[b], n)
        at = [place(table[b], P, S, j) for j in range(c + n)]
        if tree is None or None in at:
            out[b, :n] = np.nan
            continue
        page, slot = (np.array(x, np.int64) for x in zip(*at)) if at else (np.zeros(0, np.int64),) * 2
        for h in range(H):
            K, V = k_cache[page, h, slot], v_cache[page, h, slot]
            for i in range(n):
                keys = list(range(c)) + [c + a for a in tree[i]]
                for g in range(h * (Hq // H), (h + 1) * (Hq // H)):
                    with np.errstate(invalid="ignore", over="ignore"):
                        x = scale * (K[keys] @ q[b, i, g])
                        p = np.exp(x - x.max())
                        p /= p.sum()
                        out[b, i, g] = p @ V[keys]
                        mass[b, i, g] = p @ np.abs(V[keys])
                        reach[b, i, g] = abs(scale) * (np.abs(K[keys]) @ np.abs(q[b, i, g])).max()
    return out, mass, reach


def keep(k_cache, v_cache, table, seq_len, path, accepted):
    """Caches [layers, pages, ...], moved in place; returns the new lengths."""
    P, S = k_cache.shape[1], k_cache.shape[3]
    B, N = path.shape
    out = np.array(seq_len, np.int32)
    for b in range(B):
        c, a = int(seq_len[b]), int(accepted[b])
        if c < 0 or not 0 <= a < N:
            continue
        nodes = [0] + [int(x) for x in path[b, :a]]
        if any(not i < j < N for i, j in zip(nodes, nodes[1:])):
            continue
        src = [place(table[b], P, S, c + j) for j in nodes]
        if None in src:
            continue
        rows = [(k_cache[:, s[0], :, s[1]].copy(), v_cache[:, s[0], :, s[1]].copy()) for s in src]
        for i, (k, v) in enumerate(rows):
            at = place(table[b], P, S, c + i)
            k_cache[:, at[0], :, at[1]], v_cache[:, at[0], :, at[1]] = k, v
        out[b] = c + 1 + a
    return out
