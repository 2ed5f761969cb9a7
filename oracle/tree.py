"""Oracle of trees of drafted tokens: layout, attention of one unit (batch entry,
kv-head) and verification of one sequence, in plain Python and fp64."""
import numpy as np


def ancestors(parents):
    """For each node the list of its ancestors, from the root, and itself."""
    chains = []
    for i, p in enumerate(parents):
        chains.append((chains[p] if p >= 0 else []) + [i])
    return chains


def sees(parents):
    """bool [n][n]: row i, the nodes that node i sees."""
    out = np.zeros((len(parents), len(parents)), bool)
    for i, chain in enumerate(ancestors(parents)):
        out[i, chain] = True
    return out


def words(seen, n):
    """uint32 [m][ceil(n / 32)] of bool [m][m]."""
    m = len(seen)
    out = np.zeros((m, (n + 31) // 32), np.uint32)
    for i in range(m):
        for j in np.flatnonzero(seen[i]):
            out[i, j // 32] |= np.uint32(1) << np.uint32(j % 32)
    return out


def attend(unit, k, v, seen, depth, q, scale, cap=0.0, window=0, slopes=None):
    """unit: block.Unit with the cached tokens; k, v: [m][D] and q: [m][G][D], the
    nodes' -> fp64 [m][G][D]."""
    K = np.concatenate([unit.values(0), k]).astype(np.float64)
    V = np.concatenate([unit.values(1), v]).astype(np.float64)
    first = unit.pos[-1] + 1 if unit.length else 0
    pos = np.concatenate([unit.pos, first + np.asarray(depth, np.int64)])
    out = np.zeros(q.shape)
    for i in range(len(k)):
        t = np.concatenate([np.arange(unit.length), unit.length + np.flatnonzero(seen[i])])
        away = (first + depth[i] - pos[t]).astype(np.float64)
        if window:
            t, away = t[away < window], away[away < window]
        if not len(t):
            continue
        for g in range(q.shape[1]):
            x = scale * (K[t] @ q[i, g].astype(np.float64))
            if cap:
                x = cap * np.tanh(x / cap)
            if slopes is not None:
                x = x - float(slopes[g]) * away
            p = np.exp(x - x.max())
            out[i, g] = p @ V[t] / p.sum()
    return out


def verify(parents, tokens, target, draft, uniforms, room):
    """target, draft (or None): float [m][V]; -> (accepted nodes, next token)."""
    path = [0]
    while True:
        at = path[-1]
        r, s, child = np.asarray(target[at], np.float64).copy(), 1.0, None
        for c in range(1, len(parents)) if len(path) < room else ():
            if parents[c] != at:
                continue
            x = tokens[c]
            q = 1.0 if draft is None else float(draft[at][x])
            if float(uniforms[c]) * q * s < r[x]:
                child = c
                break
            if draft is None:
                s = max(0.0, s - r[x])
                r[x] = 0.0
            else:
                r = np.maximum(0.0, r / s - np.asarray(draft[at], np.float64)) if s > 0 else 0 * r
                s = float(r.sum())
        if child is None:
            break
        path.append(child)
    if not r.sum() > 0:
        r = np.asarray(target[path[-1]], np.float64)
    if not r.sum() > 0:
        return path, 0
    run = np.cumsum(r)
    over = np.flatnonzero(run > float(uniforms[0]) * run[-1])
    return path, int(over[0] if len(over) else np.flatnonzero(r > 0)[-1])
