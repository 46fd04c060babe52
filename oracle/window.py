"""CPU oracle of the 8-bit token window and of the verification of drafts -- TEST INFRASTRUCTURE ONLY.

Plain numpy from the definitions, fp64 (the verification's sums: whole numbers).  Arrays are those
of one window: numbers k [B, Hkv, C, 64] and v [B, Hkv, C / 64, 64, 64] (column, row) as fp64 values,
scales [B, Hkv, C], length [B].
"""

import numpy as np

from . import cache as oc

NEG_INF = -np.inf
FIX = 2**44


def quantise_row(x, fmt, values):
    """Numbers (fp64) and scale of one token's 64 keys or values."""
    x = np.asarray(x, np.float64)
    n, scale = oc.quantise(x, fmt)
    if np.isnan(x).any():
        scale = np.nan
        if values:
            n = np.where(np.isnan(n), 0.0, n)
    return n, scale


def row_of(pos, C, window):
    """The row of a position, or -1."""
    return pos % C if window else (pos if pos < C else -1)


def counts(lengths, B, T):
    return np.full(B, T, np.int64) if lengths is None else np.clip(np.asarray(lengths, np.int64), 0, T)


def append(w, k, v, lengths, fmt, window):
    """Appends k, v [B, Hkv, T, 64] to w = dict(k, v, k_scale, v_scale, length), in place."""
    B, Hkv, T, _ = k.shape
    C = w["k"].shape[2]
    n = counts(lengths, B, T)
    for b in range(B):
        for i in range(max(0, n[b] - C) if window else 0, n[b]):
            r = row_of(w["length"][b] + i, C, window)
            if r < 0:
                continue
            for h in range(Hkv):
                w["k"][b, h, r], w["k_scale"][b, h, r] = quantise_row(k[b, h, i], fmt, False)
                w["v"][b, h, r // 64, :, r % 64], w["v_scale"][b, h, r] = quantise_row(v[b, h, i], fmt, True)
        w["length"][b] += n[b]


def keep(w, path, lengths, T, window):
    """Keeps the path's tokens of the newest T, in place."""
    B, Hkv, C, _ = w["k"].shape
    n = counts(lengths, B, T)
    for b in range(B):
        base, last, m = max(0, int(w["length"][b] - n[b])), -1, 0
        for x in path[b]:
            if x <= last or x >= n[b] or (not window and base + x >= C and base + m < C):
                break
            last, m = x, m + 1
        for i in range(m):
            f, t = row_of(base + path[b, i], C, window), row_of(base + i, C, window)
            if f < 0 or t < 0:
                continue
            w["k"][b, :, t], w["k_scale"][b, :, t], w["v_scale"][b, :, t] = (
                w["k"][b, :, f].copy(), w["k_scale"][b, :, f].copy(), w["v_scale"][b, :, f].copy())
            w["v"][b, :, t // 64, :, t % 64] = w["v"][b, :, f // 64, :, f % 64].copy()
        w["length"][b] = base + m


def tree(parents, n):
    """Depths, and sees[i, a]: whether node a is node i or above it."""
    depth, sees = np.zeros(n, np.int64), np.eye(n, dtype=bool)
    for i in range(n):
        p = parents[i]
        if 0 <= p < i:
            depth[i] = depth[p] + 1
            sees[i] |= sees[p]
    return depth, sees


def visible(length, n, C, window, parents=None):
    """Which rows row i of the n newest tokens sees: a list of (rows, distances), distances = the key's
    position less the row's."""
    base = length - n
    depth, sees = tree(parents, n) if parents is not None else (np.arange(n), np.tril(np.ones((n, n), bool)))
    out = []
    for i in range(n):
        lo = max(0, base + depth[i] - window + 1) if window else 0
        old = np.arange(lo, max(lo, base))
        new = np.array([a for a in range(n) if sees[i, a] and base + a >= 0 and (not window or depth[i] - depth[a] < window)],
                       np.int64)
        pos = np.concatenate([old, base + new])
        dist = np.concatenate([old - base - depth[i], depth[new] - depth[i]])
        rows = pos % C if window else pos
        there = np.ones(len(pos), bool) if window else pos < C
        out.append((rows[there].astype(np.int64), dist[there]))
    return out


def attn(q, k, v, ks, vs, length, lengths, parents, slopes, window, scale, off_by_one):
    """out [B, H, T, 64], lse [B, H, T], and what bounds a computed row's error: dot (the largest
    scale sum |q| |key| of its keys), bias (the largest |slope| (|distance| + 64)), mag (sum p |value|), num
    (the largest value scale times sum |number|), seen (keys)."""
    B, H, T, d = q.shape
    Hkv, C = k.shape[1], k.shape[2]
    n = counts(lengths, B, T)
    r = dict(out=np.zeros(q.shape), lse=np.full((B, H, T), NEG_INF), dot=np.zeros((B, H, T)), bias=np.zeros((B, H, T)),
             mag=np.zeros(q.shape), num=np.zeros(q.shape), seen=np.zeros((B, H, T)))
    for b in range(B):
        vis = visible(int(length[b]), int(n[b]), C, window, None if parents is None else parents[b])
        nu = np.zeros(Hkv)  # a row block's largest value scale: of anything that the sequence's rows see
        allrows = np.unique(np.concatenate([x[0] for x in vis])) if vis else np.zeros(0, np.int64)
        for h in range(Hkv):
            nu[h] = np.nanmax(np.append(vs[b, h, allrows], 0.0))
        for i, (rows, dist) in enumerate(vis):
            if not len(rows):
                continue
            for h in range(H):
                j = h // (H // Hkv)
                kk = k[b, j, rows] * ks[b, j, rows][:, None]
                num = v[b, j, rows // 64, :, rows % 64]
                vv = num * vs[b, j, rows][:, None]
                sl = 0.0 if slopes is None else float(slopes[h])
                s = scale * (kk @ q[b, h, i]) + sl * dist
                top = max(s.max(), 0.0) if off_by_one else s.max()
                e = np.exp(s - top)
                den = e.sum() + (np.exp(-top) if off_by_one else 0.0)
                p = e / den
                r["out"][b, h, i] = p @ vv
                r["lse"][b, h, i] = top + np.log(den)
                r["dot"][b, h, i] = abs(scale) * (np.abs(kk) @ np.abs(q[b, h, i])).max()
                r["bias"][b, h, i] = abs(sl) * (np.abs(dist).max() + 64.0)
                r["mag"][b, h, i] = p @ np.abs(vv)
                r["num"][b, h, i] = 2.0 * nu[j] * np.abs(num).sum(axis=0)
                r["seen"][b, h, i] = len(rows)
    return r


def _clean(x):
    x = np.asarray(x, np.float64)
    return np.where(x > 0, np.minimum(x, 1.0), 0.0)


def _whole(r):
    return np.rint(r * FIX).astype(np.uint64)


def verify(p, tokens, u, q=None, parents=None, lengths=None):
    """path [B, T], count [B], next [B] by the walk, one sequence after the other."""
    B, T, V = p.shape
    n = counts(lengths, B, T)
    path, count, nxt = np.full((B, T), -1, np.int64), np.zeros(B, np.int64), np.full(B, -1, np.int64)
    uu = np.where(u > 0, np.minimum(u, np.float32(1 - 2.0**-24)), 0).astype(np.float64)
    for b in range(B):
        if n[b] == 0:
            continue
        par = [i - 1 for i in range(T)] if parents is None else [int(x) for x in parents[b]]
        walk, a = [0], 0
        while True:
            r, z, go = _clean(p[b, a]), 1.0, None
            for c in range(a + 1, n[b]):
                if par[c] != a:
                    continue
                x = int(tokens[b, c])
                if not 0 <= x < V:
                    continue
                qa = _clean(q[b, a]) if q is not None else None
                if uu[b, c] * (z * (qa[x] if q is not None else 1.0)) < r[x]:
                    go = c
                    break
                if q is not None:
                    r = np.maximum(r - z * qa, 0.0)
                    z = float(int(_whole(r).sum())) / FIX
                else:
                    z = max(z - r[x], 0.0)
                    r[x] = 0.0
            if go is None:
                break
            a = go
            walk.append(a)
        path[b, :len(walk)], count[b] = walk, len(walk)
        w = _whole(r)
        if w.sum() == 0:
            w = _whole(_clean(p[b, a]))
        total = int(w.sum())
        if total:
            at = np.uint64(np.floor(uu[b, 0] * float(total)))
            nxt[b] = int(np.searchsorted(np.cumsum(w, dtype=np.uint64), at, side="right"))
    return path, count, nxt
