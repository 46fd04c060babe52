"""CPU oracle of the bounded 8-bit chunk cache -- TEST INFRASTRUCTURE ONLY.

Plain fp64 numpy from the definitions: quantised tiles, masked landmark retrieval,
grouped cross attention over cached chunks (Eq. 2-3), and eviction by accumulated
weight.  Arrays are those of one cache: numbers [B, Hkv, C, 64, 64] (keys [token,
column], values [column, token]) as fp64 values, scales [B, Hkv, C], tokens [B, C].
"""

import numpy as np

NEG_INF = -np.inf


def e4m3_round(y):
    """Nearest e4m3 value, ties to even: 3 mantissa bits, exponents -6 .. 8, subnormal steps of 2^-9."""
    a = np.abs(y)
    exp = np.floor(np.log2(np.maximum(a, 2.0**-6)))
    step = 2.0 ** (exp - 3)
    r = np.round(a / step) * step          # numpy rounds halves to even
    return np.copysign(np.minimum(r, 448.0), y)


def e4m3_values():
    """The value of every e4m3 code, by code (0x7f and 0xff: NaN)."""
    v = np.empty(256)
    for c in range(256):
        s, e, m = -1.0 if c >> 7 else 1.0, (c >> 3) & 15, c & 7
        v[c] = np.nan if c & 0x7F == 0x7F else s * (m * 2.0**-9 if e == 0 else (8 + m) * 2.0 ** (e - 10))
    return v


def quantise(x, fmt):
    """Numbers (fp64) and scale of one 64 x 64 tile."""
    x = np.asarray(x, np.float64)
    fin = np.abs(x[np.isfinite(x)])
    top = fin.max() if fin.size else 0.0
    if fmt == "e4m3":
        scale = 2.0**-126
        while top / scale > 448.0:
            scale *= 2.0
        n = np.where(np.isnan(x), np.nan, e4m3_round(np.clip(np.where(np.isnan(x), 0.0, x) / scale, -448.0, 448.0)))
        return n, scale
    scale = max(top, 2.0**-100) / 127.0
    n = np.clip(np.round(np.where(np.isnan(x), 0.0, x) / scale), -127, 127)
    return n, (np.nan if np.isnan(x).any() else scale)


def select(lmk_q, lmk, tokens, topk, scale):
    """idx, sel, w [B, Hr, 1, topk] of landmark queries [B, Hr, 1, D] over slots in use."""
    B, Hr, C, _ = lmk.shape
    idx = np.full((B, Hr, 1, topk), -1, np.int64)
    sel = np.full((B, Hr, 1, topk), NEG_INF)
    w = np.zeros((B, Hr, 1, topk))
    for b in range(B):
        for h in range(Hr):
            with np.errstate(invalid="ignore", over="ignore"):
                s = scale * (lmk[b, h].astype(np.float64) @ lmk_q[b, h, 0].astype(np.float64))
            cand = np.nonzero((tokens[b] > 0) & np.isfinite(s))[0]
            best = np.sort(cand[np.argsort(-s[cand], kind="stable")][:topk])
            n = len(best)
            idx[b, h, 0, :n], sel[b, h, 0, :n] = best, s[best]
            if n:
                e = np.exp(s[best] - s[best].max())
                w[b, h, 0, :n] = e / e.sum()
    return idx, sel, w


def weights(idx, sel, tokens):
    """Which entries are valid, and the fusion weights of every list."""
    B, Hr, nQ, k = idx.shape
    ok = np.zeros(idx.shape, bool)
    w = np.zeros(idx.shape)
    for b in range(B):
        named = (idx[b] >= 0) & (idx[b] < tokens.shape[1])
        ok[b] = named & (tokens[b][np.where(named, idx[b], 0)] > 0)
        for h in range(Hr):
            for t in range(nQ):
                v = ok[b, h, t]
                if v.any():
                    s = sel[b, h, t, v].astype(np.float64)
                    e = np.exp(s - s.max())
                    w[b, h, t, v] = e / e.sum()
    return ok, w


def xattn(q, idx, sel, k, v, k_scale, v_scale, tokens, attn_scale, rows, lag=0, off_by_one=False):
    """Dict out, lse, w, and four bounds' ingredients: `mag` = sum_s w sum_keys p |v|, `num` =
    (largest value scale of the list) x sum_s sum_keys |number| and `wnum`, the same with the largest
    product of value scale and fusion weight (all of out's shape), and `dot` = the largest
    sum |attn_scale q k| over the row's valid entries [B, H, Lq]."""
    B, H, Lq, d = q.shape
    Hkv = k.shape[1]
    _, Hr, nQ, K = idx.shape
    ok, w = weights(idx, sel, tokens)
    out, mag, num, wnum = (np.zeros((B, H, Lq, d)) for _ in range(4))
    lse = np.full((B, H, Lq, K), NEG_INF)
    dot = np.zeros((B, H, Lq))
    for b in range(B):
        for h in range(H):
            kv = h // (H // Hkv)
            hr = 0 if Hr == 1 else kv
            for t in range(lag, nQ):
                r = slice(t * rows, (t + 1) * rows)
                qq = q[b, h, r].astype(np.float64)
                top = max((float(v_scale[b, kv, j]) for j, o in zip(idx[b, hr, t - lag], ok[b, hr, t - lag]) if o),
                          default=0.0)
                wtop = max((float(v_scale[b, kv, j]) * x for j, o, x in
                            zip(idx[b, hr, t - lag], ok[b, hr, t - lag], w[b, hr, t - lag]) if o), default=0.0)
                for s in range(K):
                    if not ok[b, hr, t - lag, s]:
                        continue
                    j = idx[b, hr, t - lag, s]
                    n = min(int(tokens[b, j]), 64)
                    kk = k[b, kv, j, :n] * float(k_scale[b, kv, j])
                    vv = v[b, kv, j, :, :n].T * float(v_scale[b, kv, j])
                    a = attn_scale * (qq @ kk.T)
                    dot[b, h, r] = np.maximum(dot[b, h, r], (abs(attn_scale) * (np.abs(qq) @ np.abs(kk).T)).max(axis=1))
                    m = a.max(axis=1, keepdims=True)
                    if off_by_one:
                        m = np.maximum(m, 0.0)
                    e = np.exp(a - m)
                    den = e.sum(axis=1, keepdims=True) + (np.exp(-m) if off_by_one else 0.0)
                    p = e / den
                    out[b, h, r] += w[b, hr, t - lag, s] * (p @ vv)
                    mag[b, h, r] += w[b, hr, t - lag, s] * (p @ np.abs(vv))
                    num[b, h, r] += top * np.abs(v[b, kv, j, :, :n]).sum(axis=1)
                    wnum[b, h, r] += wtop * np.abs(v[b, kv, j, :, :n]).sum(axis=1)
                    lse[b, h, r, s] = (m + np.log(den))[:, 0]
    return dict(out=out, lse=lse, w=w, mag=mag, num=num, wnum=wnum, dot=dot)


def evict(tokens, mass, number, nxt, n, idx=None, w=None, decay=1.0, keep_first=0, keep_last=0, want=None):
    """New tokens, mass (fp32, one rounding), number, next, and slots [B, n]."""
    B, C = tokens.shape
    tokens, number, nxt = tokens.copy(), number.copy(), nxt.copy()
    new = np.zeros((B, C), np.float32)
    slots = np.full((B, n), -1, np.int64)
    for b in range(B):
        add = np.zeros(C, object)          # exact integers, in units of 2^-48 or as 2^16 entries or more need
        bits = 64 - max(16, int(idx[b].size).bit_length()) if idx is not None else 48
        if idx is not None:
            for j, x in zip(idx[b].reshape(-1), w[b].reshape(-1)):
                if 0 <= j < C and x > 0:
                    add[j] += int(np.floor(min(float(x), 1.0) * 2.0**bits + 0.5))
        used = tokens[b] > 0
        total = np.array([float(a) for a in add]) * 2.0**-bits
        with np.errstate(over="ignore", invalid="ignore"):
            m = (np.float64(np.float32(decay)) * mass[b].astype(np.float64) + total).astype(np.float32)
        new[b] = np.where(used, m, 0)
        stays = used & ((number[b] < keep_first) | (number[b] >= int(nxt[b]) - keep_last))
        rank = [(0, 0.0, j) if not used[j] else (1, float(new[b, j]) if new[b, j] > 0 else 0.0, j)
                for j in range(C) if not stays[j]]
        m = n if want is None else max(0, min(int(want[b]), n))
        took = sorted(j for _, _, j in sorted(rank)[:m])
        slots[b, :len(took)] = took
        for i, j in enumerate(took):
            tokens[b, j], new[b, j], number[b, j] = 0, 0, nxt[b] + i
        if n:
            nxt[b] += m
    return tokens, new, number, nxt, slots
