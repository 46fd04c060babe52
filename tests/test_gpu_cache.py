"""GPU parity of the chunk cache against its fp64 oracle (oracle/cache.py), at the sizes and
lists where an operator can go wrong.

Tolerances, in units of u = 2^-24 (half an fp32 step, relative).  Scores are sums of 64 exact
products in fp32: off by at most 66 u times the sum of the products' magnitudes (`dot`; the
product with the scale included).  An exponential of such a score is off by that relative
amount (twice, once through the maximum) and by 4 u of its own; a normalised weight twice that.
So a row's output is off by at most 4 x 66 u dot + 64 u (its fp32 sums and the fusion weights)
plus the rounding of the probabilities (bf16 tensors: 2^-11 for fp16; fp32: 2^-22 for two terms) of
sum w p |v| (`mag`), and by its own rounding (2^-8 bf16, 2^-24 fp32) of its value.  That is so
for normal fp16 numbers; below 2^-14 fp16 has steps of 2^-24, so a scaled probability (2^15 w p
times its value scale over the list's largest, nu) is off by up to 2^-25 whatever its size, which
nu 2^-15 turns into 2^-40 nu of each number's magnitude (`num` = nu sum |number|): it shows only
in outputs some 1e-12 of the values, where every heavy key's value is nearly zero."""

import numpy as np
import pytest

from _helpers import ensure_built, host64
from oracle import cache as oc

pytestmark = pytest.mark.gpu
U = 2.0**-24


@pytest.fixture(scope="module")
def dev():
    torch = pytest.importorskip("torch")
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    ensure_built()
    return torch.device("cuda:0")


def _elem(dtype):
    import torch
    return torch.bfloat16 if dtype == "bf16" else torch.float32


def _values(t):
    """8-bit numbers as fp64."""
    import torch
    if t.dtype == torch.int8:
        return t.cpu().numpy().astype(np.float64)
    return oc.e4m3_values()[t.view(torch.uint8).cpu().numpy()]


def _fill(c, seed, lengths=None):
    """Random numbers and scales in every slot, and lengths (default: all full)."""
    import torch
    g = torch.Generator(device=c.device).manual_seed(seed)
    for t in (c.k, c.v):
        x = torch.randint(-127, 128, t.shape, generator=g, device=c.device, dtype=torch.int8)
        if t.dtype != torch.int8:     # any code but NaN
            x = torch.where((x & 0x7F) == 0x7F, x & ~1, x)
        t.view(torch.int8).copy_(x)
    wide = 2.0**-5 if c.k.dtype == torch.int8 else 2.0**-6
    for s in (c.k_scale, c.v_scale):
        s.copy_(wide * torch.exp(torch.randn(s.shape, generator=g, device=c.device)))
    c.tokens.copy_(torch.full_like(c.tokens, 64) if lengths is None else torch.from_numpy(lengths).to(c.device))
    return g


def _lists(rng, B, Hr, nQ, C, k, holes):
    idx = np.full((B, Hr, nQ, k), -1, np.int32)
    for b in range(B):
        for h in range(Hr):
            for t in range(nQ):
                n = int(rng.integers(0, min(k, C) + 1)) if holes else min(k, C)
                at = rng.permutation(k)[:n] if holes else np.arange(n)
                idx[b, h, t, at] = rng.choice(C, n, replace=False)
    sel = np.where(idx >= 0, 2 * rng.standard_normal(idx.shape), -np.inf).astype(np.float32)
    return idx, sel


def _check_xattn(c, q, idx, sel, got, rows, lag):
    out, lse, w = got
    s = c.struct
    ref = oc.xattn(host64(q), idx, sel, _values(c.k), _values(c.v), host64(c.k_scale), host64(c.v_scale),
                   c.tokens.cpu().numpy(), s.attn_scale, rows, lag, bool(s.off_by_one))
    bf16 = s.dtype == 1
    rel = 4 * 66 * U * ref["dot"] + 64 * U
    bound = (rel[..., None] + (2.0**-11 if bf16 else 2.0**-22)) * ref["mag"] + (2.0**-8 if bf16 else U) * np.abs(ref["out"])
    bound += 2.0**-40 * ref["num"]
    err = np.abs(host64(out) - ref["out"])
    assert (err <= bound * (1 + 2.0**-7) + 1e-30).all(), float((err / (bound + 1e-300)).max())
    if lse is not None:
        x, f = host64(lse), np.isfinite(ref["lse"])
        assert np.array_equal(f, np.isfinite(x)) and (x[~f] == -np.inf).all()
        lim = 2 * 66 * U * ref["dot"][..., None] + 16 * U * (1 + np.abs(np.where(f, ref["lse"], 0.0)))
        assert (np.abs(np.where(f, x - np.where(f, ref["lse"], 0.0), 0.0)) <= lim).all()
    if w is not None:
        # exponents of sel - max (at most 16): exact difference, 4 u, and the sum's and quotient's roundings
        assert (np.abs(host64(w) - ref["w"]) <= 64 * U * ref["w"] + 1e-30).all()
    return ref


XATTN = [
    # B, H, Hkv, Hr, C, k, nQ, rows, lag, dtype, format, off_by_one, holes
    (1, 1, 1, 1, 1, 1, 1, 1, 0, "bf16", "e4m3", False, False),      # one of everything
    (1, 1, 1, 1, 1, 32, 1, 1, 0, "fp32", "int8", True, False),      # a list longer than the cache
    (2, 4, 2, 1, 9, 5, 1, 1, 0, "bf16", "int8", False, True),       # a token, grouped heads
    (2, 6, 2, 2, 9, 5, 1, 7, 0, "fp32", "e4m3", True, True),        # 21 rows of a group
    (1, 16, 1, 1, 40, 32, 1, 1, 0, "bf16", "e4m3", False, True),    # 16 rows, the longest list
    (1, 17, 1, 1, 40, 32, 1, 1, 0, "bf16", "e4m3", True, True),     # 17 rows
    (1, 2, 2, 2, 70, 16, 1, 33, 0, "bf16", "int8", False, True),    # 33 rows
    (2, 2, 1, 1, 20, 8, 3, 32, 1, "bf16", "e4m3", False, True),     # 64 rows, heads apart in memory
    (1, 3, 3, 3, 20, 8, 5, 64, 1, "bf16", "e4m3", True, False),     # chunks over causal lists
    (1, 3, 3, 1, 20, 8, 5, 65, 1, "bf16", "int8", False, True),     # S + 1 rows
    (1, 4, 2, 1, 12, 3, 2, 65, 0, "fp32", "int8", False, True),     # 130 rows, fp32
    (1, 1, 1, 1, 300, 1, 260, 1, 1, "bf16", "e4m3", False, True),   # many lists of one entry
    (3, 2, 2, 2, 30, 9, 90, 40, 0, "bf16", "e4m3", False, True),    # more items than waves
    (1, 1, 1, 1, 5, 4, 1, 1000, 0, "fp32", "e4m3", True, False),    # many row blocks
    # enough groups for 64 rows per wave: full, a row over half, two heads' rows apart, four blocks
    (2, 4, 4, 1, 40, 3, 256, 64, 1, "bf16", "e4m3", False, True),
    (2, 4, 4, 4, 17, 2, 260, 33, 0, "bf16", "int8", True, True),
    (1, 8, 4, 1, 30, 2, 520, 32, 1, "bf16", "e4m3", True, True),
    (1, 2, 2, 2, 9, 1, 270, 250, 0, "bf16", "int8", False, True),
]


@pytest.mark.parametrize("B,H,Hkv,Hr,C,k,nQ,rows,lag,dtype,fmt,obo,holes", XATTN)
def test_attention(dev, B, H, Hkv, Hr, C, k, nQ, rows, lag, dtype, fmt, obo, holes):
    import torch
    from paper_2410_01651_amd import gca
    rng = np.random.default_rng(C + 7 * rows)
    c = gca.cache(B, H, C, k, Hkv=Hkv, Hr=Hr, D=64, dtype=dtype, format=fmt, off_by_one=obo)
    lengths = rng.choice([-3, 0, 1, 15, 16, 17, 31, 33, 63, 64, 64, 64, 99], (B, C)).astype(np.int32) if holes else None
    g = _fill(c, C + k, lengths)
    idx, sel = _lists(rng, B, Hr, nQ, C, k, holes)
    q = torch.randn(B, H, nQ * rows, 64, generator=g, device=dev, dtype=_elem(dtype))
    got = gca.cache_xattn(c, q, torch.from_numpy(idx).to(dev), torch.from_numpy(sel).to(dev), causal=bool(lag))
    _check_xattn(c, q, idx, sel, got, rows, lag)


@pytest.mark.parametrize("seed", range(24))
def test_attention_random_problems(dev, seed):
    """Small problems drawn over everything a call may vary in."""
    import torch
    from paper_2410_01651_amd import gca
    rng = np.random.default_rng(1000 + seed)
    pick = lambda *a: a[rng.integers(len(a))]  # noqa: E731
    Hkv, G, B = pick(1, 2, 3), pick(1, 2, 4, 5), pick(1, 2, 3)
    C, k, nQ, rows = pick(1, 4, 30, 90), int(rng.integers(1, 33)), pick(1, 1, 2, 7), pick(1, 2, 5, 16, 31, 64, 70)
    dtype, fmt, obo, lag = pick("bf16", "fp32"), pick("e4m3", "int8"), bool(pick(0, 1)), pick(0, 1)
    c = gca.cache(B, G * Hkv, C, k, Hkv=Hkv, Hr=pick(1, Hkv), D=64, dtype=dtype, format=fmt, off_by_one=obo,
                  attn_scale=pick(None, 0.3, -0.05))
    g = _fill(c, seed, rng.integers(-1, 66, (B, C)).astype(np.int32))
    idx, sel = _lists(rng, B, c.struct.Hr, nQ, C, k, True)
    q = torch.randn(B, G * Hkv, nQ * rows, 64, generator=g, device=dev, dtype=_elem(dtype))
    got = gca.cache_xattn(c, q, torch.from_numpy(idx).to(dev), torch.from_numpy(sel).to(dev), causal=bool(lag))
    _check_xattn(c, q, idx, sel, got, rows, lag)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("scale", [-0.125, 0.0, 3.0])
def test_attention_scales(dev, dtype, scale):
    """A negative scale, none, and one that makes the softmax pick single keys."""
    import torch
    from paper_2410_01651_amd import gca
    rng = np.random.default_rng(3)
    c = gca.cache(1, 2, 6, 4, D=64, dtype=dtype, attn_scale=scale)
    g = _fill(c, 5, np.array([[64, 10, 64, 1, 64, 33]], np.int32))
    idx, sel = _lists(rng, 1, 1, 1, 6, 4, False)
    q = torch.randn(1, 2, 9, 64, generator=g, device=dev, dtype=_elem(dtype))
    got = gca.cache_xattn(c, q, torch.from_numpy(idx).to(dev), torch.from_numpy(sel).to(dev))
    _check_xattn(c, q, idx, sel, got, 9, 0)


def test_attention_odd_entries(dev):
    """Indices outside the cache and entries of free slots are pads; a slot named twice counts twice;
    want_* switches leave the outputs alone."""
    import torch
    from paper_2410_01651_amd import gca
    C, k = 5, 8
    c = gca.cache(1, 1, C, k, D=64)
    g = _fill(c, 8, np.array([[64, 0, 64, 64, -1]], np.int32))
    idx = np.array([[[[3, 2**31 - 1, -2**31, 3, 5, 1, 4, 0], [-1, 5, 1, 4, -7, 9, 1, 1]]]], np.int32)
    sel = np.linspace(-2, 2, 16).reshape(idx.shape).astype(np.float32)
    q = torch.randn(1, 1, 6, 64, generator=g, device=dev, dtype=torch.bfloat16)
    i, s = torch.from_numpy(idx).to(dev), torch.from_numpy(sel).to(dev)
    full = gca.cache_xattn(c, q, i, s)
    ref = _check_xattn(c, q, idx, sel, full, 3, 0)
    assert (ref["w"][0, 0, 0] > 0).tolist() == [True, False, False, True, False, False, False, True]
    assert not host64(full[0])[0, 0, 3:].any()      # the second list names nothing in use
    bare = gca.cache_xattn(c, q, i, s, want_lse=False, want_w=False)
    assert bare[1] is None and bare[2] is None and torch.equal(bare[0], full[0])


@pytest.mark.parametrize("fmt", ["e4m3", "int8"])
@pytest.mark.parametrize("rows", [1, 40])
def test_masked_numbers_stay_out(dev, fmt, rows):
    """Whatever lies behind a chunk's last token, in free slots and in their scales."""
    import torch
    from paper_2410_01651_amd import gca
    c = gca.cache(1, 1, 4, 3, D=64, format=fmt)
    g = _fill(c, 9, np.array([[20, 0, 64, 0]], np.int32))
    q = torch.randn(1, 1, rows, 64, generator=g, device=dev, dtype=torch.bfloat16)
    idx = torch.tensor([[[[0, 1, 2]]]], dtype=torch.int32, device=dev)
    sel = torch.tensor([[[[0.5, 9.0, -0.5]]]], device=dev)
    want = gca.cache_xattn(c, q, idx, sel)
    for t, tail in ((c.k, (0, 0, 0, slice(20, None))), (c.v, (0, 0, 0, slice(None), slice(20, None)))):
        b = t.view(torch.uint8)
        b[tail] = 0x7F        # NaN, or 127
        b[0, 0, 1] = 0xFF
    for s in (c.k_scale, c.v_scale):
        s[0, 0, 1], s[0, 0, 3] = float("nan"), float("inf")
    got = gca.cache_xattn(c, q, idx, sel)
    for x, y in zip(got, want):
        assert torch.equal(x, y)


def test_attention_far_slots(dev):
    """Slots whose tiles lie past 2^32 bytes: the last ones of a 16M-token cache."""
    import torch
    from paper_2410_01651_amd import gca
    C, H, k = 262144, 5, 4
    c = gca.cache(1, H, C, k, D=64)
    small = gca.cache(1, H, k, k, D=64)
    g = _fill(small, 4)
    at = torch.tensor([3, C // 2, C - 2, C - 1], device=dev)
    for x in ("k", "v", "k_scale", "v_scale"):
        t, s = getattr(c, x), getattr(small, x)
        for i, j in enumerate(at.tolist()):
            t[:, :, j] = s[:, :, i]
    c.tokens[:, at] = 64
    q = torch.randn(1, H, 2, 64, generator=g, device=dev, dtype=torch.bfloat16)
    sel = torch.tensor([[[[0.1, -1.0, 0.7, 0.3]]]], device=dev)
    got = gca.cache_xattn(c, q, at.int().view(1, 1, 1, k), sel)
    want = gca.cache_xattn(small, q, torch.arange(k, device=dev, dtype=torch.int32).view(1, 1, 1, k), sel)
    for x, y in zip(got, want):
        assert torch.equal(x, y)


def test_attention_equals_the_uncached_path(dev):
    """Chunks that 8 bits hold exactly: the framework's CAUSAL attention on the same keys and values."""
    import torch
    from paper_2410_01651_amd import gca
    B, H, nC, k = 1, 4, 40, 8
    g = torch.Generator(device=dev).manual_seed(2)
    num = lambda: torch.randint(-14, 15, (B, H, nC * 64, 64), generator=g, device=dev).bfloat16() / 8  # noqa: E731
    kk, vv = num(), num()
    q = torch.randn(B, H, nC * 64, 64, generator=g, device=dev, dtype=torch.bfloat16)
    lq, lk = (torch.randn(B, 1, nC, 64, generator=g, device=dev, dtype=torch.bfloat16) for _ in range(2))
    ref = gca.forward(gca.problem(B, H, nC, k, D=64), lq, lk, q, kk, vv)
    c = gca.cache(B, H, nC, k, D=64)
    gca.cache_store(c, kk, vv, lk, torch.arange(nC, device=dev, dtype=torch.int32).view(B, nC))
    out, lse, w = gca.cache_xattn(c, q, ref["idx"], ref["sel"], causal=True)
    # bf16 against fp16 probabilities, each output rounded once
    lim = 2.0**-7 * float(ref["out"].abs().max())
    assert float((out.float() - ref["out"].float()).abs().max()) <= lim
    fin = torch.isfinite(ref["lse"])
    assert torch.equal(fin, torch.isfinite(lse)) and float((lse - ref["lse"])[fin].abs().max()) <= 1e-5
    assert float((w - ref["w"]).abs().max()) <= 1e-6


# ------------------------------------------------------------------- store ----

STORE = [
    # B, Hkv, Hr, C, n, D, dtype, format
    (1, 1, 1, 1, 1, 64, "bf16", "e4m3"),
    (2, 3, 1, 9, 4, 192, "bf16", "int8"),
    (3, 2, 2, 7, 7, 64, "fp32", "e4m3"),
    (2, 2, 2, 150, 140, 1024, "fp32", "int8"),
]


def _check_tile(n, s, x, fmt):
    """A stored tile against its fp64 quantisation: e4m3 exactly; int8 scales to 2 u, numbers to the
    nearer integer but where the quotient lies within 4 u of a half."""
    want, scale = oc.quantise(x, fmt)
    if fmt == "e4m3":
        np.testing.assert_array_equal(s, scale)
        np.testing.assert_array_equal(n, want)
        return
    assert np.isnan(s) == np.isnan(scale) and (np.isnan(s) or abs(s - scale) <= 2 * U * scale)
    fin = np.abs(x[np.isfinite(x)])
    y = np.clip(np.where(np.isnan(x), 0, x) / (max(fin.max() if fin.size else 0, 2.0**-100) / 127.0), -127, 127)
    ok = ~np.isnan(x)
    assert (np.abs(n - y)[ok] <= 0.5 + 127 * 4 * U).all()


@pytest.mark.parametrize("B,Hkv,Hr,C,n,D,dtype,fmt", STORE)
@pytest.mark.parametrize("ragged", [False, True])
def test_store(dev, B, Hkv, Hr, C, n, D, dtype, fmt, ragged):
    import torch
    from paper_2410_01651_amd import gca
    rng = np.random.default_rng(n + D)
    c = gca.cache(B, 2 * Hkv, C, 4, Hkv=Hkv, Hr=Hr, D=D, dtype=dtype, format=fmt)
    g = _fill(c, 3, rng.integers(0, 65, (B, C)).astype(np.int32))
    c.lmk.normal_(generator=g)
    before = {x: getattr(c, x).clone() for x in c.NAMES}
    elem = _elem(dtype)
    k, v = (torch.randn(B, Hkv, n * 64, 64, generator=g, device=dev, dtype=elem) *
            torch.exp(3 * torch.randn(B, Hkv, n, 1, generator=g, device=dev)).repeat_interleave(64, 2).to(elem)
            for _ in range(2))
    lmk = torch.randn(B, Hr, n, D, generator=g, device=dev, dtype=elem)
    slots = np.stack([rng.permutation(C)[:n] for _ in range(B)]).astype(np.int32)
    lengths = np.full(B, n * 64, np.int32)
    if ragged:
        if n > 3:
            slots[0, 2], slots[-1, 0] = -1, C          # skipped
            slots[-1, 1] = slots[-1, 3]                # named twice: the later chunk
        lengths = np.array([n * 64 - 1, 0, 65])[:B].astype(np.int32) if B > 1 else np.array([7], np.int32)
    gca.cache_store(c, k, v, lmk, torch.from_numpy(slots).to(dev), torch.from_numpy(lengths).to(dev) if ragged else None)
    num = {"k": _values(c.k), "v": _values(c.v)}
    new = {"k": host64(k), "v": host64(v)}
    put = {}                                            # (b, slot) -> chunk
    for b in range(B):
        for i in range(n):
            if 0 <= slots[b, i] < C and lengths[b] > 64 * i:
                put[b, slots[b, i]] = i
    for b in range(B):
        for j in range(C):
            i = put.get((b, j))
            if i is None:                               # left as it was, to the last byte
                for x in ("k", "v", "k_scale", "v_scale", "lmk"):
                    assert torch.equal(getattr(c, x)[b, :, j].contiguous().view(torch.uint8),
                                       before[x][b, :, j].contiguous().view(torch.uint8)), (x, b, j)
                assert c.tokens[b, j] == before["tokens"][b, j]
                continue
            t = min(64, int(lengths[b]) - 64 * i)
            assert int(c.tokens[b, j]) == t and torch.equal(c.lmk[b, :, j], lmk[b, :, i])
            for h in range(Hkv):
                for x in ("k", "v"):
                    tile = new[x][b, h, 64 * i:64 * i + 64].copy()
                    tile[t:] = 0
                    got = num[x][b, h, j] if x == "k" else num[x][b, h, j].T
                    _check_tile(got, float(getattr(c, x + "_scale")[b, h, j]), tile, fmt)
    for x in ("mass", "number", "next"):
        assert torch.equal(getattr(c, x), before[x])


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("fmt", ["e4m3", "int8"])
def test_store_extremes(dev, dtype, fmt):
    """Zeros, the least and largest magnitudes, the e4m3 scale's borders, infinities and NaN."""
    import torch
    from paper_2410_01651_amd import gca
    rng = np.random.default_rng(1)
    tiles = []
    for top in (0.0, 448.0, 450.0, 1.75, 1.765625, 1.0, 2.0**-126, 2.0**-133, 3.3e38):
        x = np.clip(rng.standard_normal((64, 64)), -4, 4) / 4 * top
        x[5, 9] = -top
        tiles.append(x)
    for odd in (np.inf, -np.inf, np.nan):
        x = rng.standard_normal((64, 64))
        x[63, 0], x[0, 63] = odd, odd
        tiles.append(x)
    tiles.append(np.full((64, 64), np.nan))
    tiles.append(np.full((64, 64), np.inf))
    n = len(tiles)
    k = torch.from_numpy(np.stack(tiles).reshape(1, 1, n * 64, 64)).to(_elem(dtype)).to(dev)
    c = gca.cache(1, 1, n, 4, D=64, dtype=dtype, format=fmt)
    slots = torch.arange(n, device=dev, dtype=torch.int32).view(1, n)
    gca.cache_store(c, k, k, None, slots)
    x = k.double().cpu().numpy().reshape(n, 64, 64)
    for i in range(n):
        for t, s in ((_values(c.k)[0, 0, i], c.k_scale), (_values(c.v)[0, 0, i].T, c.v_scale)):
            _check_tile(t, float(s[0, 0, i]), x[i], fmt)
    # the same chunks behind a shorter length: nothing past it counts
    short = torch.tensor([(n - 3) * 64 + 1], dtype=torch.int32, device=dev)
    gca.cache_store(c, k.flip(2).contiguous(), k, None, slots, lengths=short)
    assert c.tokens[0].tolist() == [64] * (n - 3) + [1, 64, 64]


# ------------------------------------------------------------------ select ----

SELECT = [
    # B, Hkv, Hr, C, k, D, dtype, share of slots in use
    (1, 1, 1, 1, 1, 64, "bf16", 1.0),
    (1, 1, 1, 1, 8, 64, "bf16", 0.0),          # nothing in use
    (2, 3, 3, 7, 8, 128, "fp32", 0.5),         # fewer candidates than entries
    (3, 2, 1, 1000, 8, 1024, "bf16", 0.7),
    (2, 2, 2, 333, 16, 512, "bf16", 0.9),      # the query in registers
    (1, 1, 1, 5000, 32, 64, "fp32", 0.3),
    (1, 1, 1, 70000, 5, 512, "bf16", 0.99),    # more keys than the lanes keep
    (300, 1, 1, 600, 3, 64, "bf16", 0.6),      # one workgroup scans a row
    (1, 1, 1, 40000, 32, 64, "bf16", 0.9),     # a thousand lists to merge
    (2, 2, 2, 20000, 16, 64, "fp32", 0.02),    # most of them empty
    (1, 1, 1, 3000, 17, 128, "bf16", 0.8),
    (2, 1, 1, 200, 4, 8192, "fp32", 0.5),
]


def _landmarks(rng, B, Hr, C, D, dtype, tokens, k, scale):
    """Landmarks whose k-th and next scores are apart by more than fp32 sums can be off: D u times the
    sum of the products' magnitudes (at most 0.7 D / sqrt(D) here) is below 1e-3 for D = 8192."""
    import torch
    rnd = lambda *s: torch.from_numpy(rng.standard_normal(s).astype(np.float32)).to(_elem(dtype))  # noqa: E731
    lk = rnd(B, Hr, C, D)
    lq = rnd(B, Hr, 1, D)
    x = lk.double().numpy()
    for b in range(B):
        for h in range(Hr):
            for _ in range(50):
                s = np.sort(scale * (x[b, h] @ lq[b, h, 0].double().numpy())[tokens[b] > 0])[::-1]
                if len(s) <= k or s[k - 1] - s[k] > 1e-3:
                    break
                lq[b, h, 0] = rnd(D)
    return lq, lk


@pytest.mark.parametrize("B,Hkv,Hr,C,k,D,dtype,share", SELECT)
def test_select(dev, B, Hkv, Hr, C, k, D, dtype, share):
    import torch
    from paper_2410_01651_amd import gca
    rng = np.random.default_rng(C + D)
    scale = 1.0 / np.sqrt(D)
    tokens = np.where(rng.random((B, C)) < share, rng.integers(1, 65, (B, C)), -rng.integers(0, 2, (B, C))).astype(np.int32)
    lq, lk = _landmarks(rng, B, Hr, C, D, dtype, tokens, k, scale)
    c = gca.cache(B, Hkv, C, k, Hr=Hr, D=D, dtype=dtype)
    c.lmk.copy_(lk)
    c.tokens.copy_(torch.from_numpy(tokens))
    c.lmk[torch.from_numpy(tokens).to(dev)[:, None, :].expand(B, Hr, C) <= 0] = float("nan")   # free: whatever is there
    idx, sel, w = gca.cache_select(c, lq.to(dev))
    ri, rs, rw = oc.select(lq.double().numpy(), lk.double().numpy(), tokens, k, scale)
    np.testing.assert_array_equal(idx.cpu().numpy(), ri)
    x, f = host64(sel), np.isfinite(rs)
    assert np.array_equal(f, np.isfinite(x)) and (x[~f] == -np.inf).all()
    mag = scale * np.sqrt(D) * np.sqrt(D) * 2     # above the sum of the products' magnitudes (mean 0.64 D)
    err = (D + 2) * U * mag
    assert (np.abs(x[f] - rs[f]) <= err).all()
    assert (np.abs(host64(w) - rw) <= (4 * err + 64 * U) * rw).all()


@pytest.mark.parametrize("C,k,D,dtype", [(1, 1, 64, "bf16"), (7, 8, 192, "fp32"), (8, 32, 320, "bf16"), (9, 3, 1024, "bf16"),
                                         (64, 8, 576, "bf16"), (65, 32, 256, "fp32"), (129, 8, 2048, "bf16"),
                                         (255, 16, 64, "fp32"), (256, 32, 1024, "bf16"), (256, 8, 768, "fp32"),
                                         (257, 8, 128, "bf16"), (250, 8, 2048, "bf16"), (20, 8, 8192, "fp32")])
def test_select_small_caches(dev, C, k, D, dtype):
    """Both sides of the borders of the form for small caches (256 slots, 768 KiB of landmarks per row)."""
    test_select(dev, 3, 2, 2, C, k, D, dtype, 0.8)


@pytest.mark.parametrize("C", [30, 200])
def test_select_small_caches_ties(dev, C):
    """Ties go to the lower slot; scores that are not finite are no candidates; an empty cache has none."""
    import torch
    from paper_2410_01651_amd import gca
    g = torch.Generator(device=dev).manual_seed(C)
    D, k = 192, 6
    c = gca.cache(2, 1, C, k, D=D)
    c.lmk.copy_(torch.randn(c.lmk.shape, generator=g, device=dev) * 0.1)
    lq = torch.randn(2, 1, 1, D, generator=g, device=dev, dtype=torch.bfloat16)
    same = [3, 4, 11, 12, 17, C - 3, C - 2]
    for j in same:
        c.lmk[:, 0, j] = lq[:, 0, 0]                                   # the best of all, seven times
    c.lmk[0, 0, 5, 0], c.lmk[0, 0, 6, 191], c.lmk[0, 0, 7] = float("nan"), float("inf"), float("-inf")
    c.tokens.fill_(64)
    idx, sel, w = gca.cache_select(c, lq)
    assert idx[:, 0, 0].tolist() == [same[:6]] * 2 and torch.equal(sel, sel[..., :1].expand_as(sel))
    assert float((w - 1 / 6).abs().max()) <= 4 * U / 6                 # exp(0) = 1, a sum of six, one division
    c.tokens[0, 4], c.tokens[1] = 0, -1
    idx, sel, w = gca.cache_select(c, lq)
    assert idx[0, 0, 0].tolist() == [3, 11, 12, 17, C - 3, C - 2]
    assert (idx[1] == -1).all() and (sel[1] == float("-inf")).all() and (w[1] == 0).all()


def test_select_equals_the_decode_path(dev):
    """A full cache retrieves what gca_forward in DECODE mode does; ties go to the lower slot, and
    landmarks whose scores are not finite are not candidates."""
    import torch
    from paper_2410_01651_amd import gca
    B, H, C, k, D = 2, 2, 900, 8, 256
    g = torch.Generator(device=dev).manual_seed(1)
    lq = torch.randn(B, 1, 1, D, generator=g, device=dev, dtype=torch.bfloat16)
    c = gca.cache(B, H, C, k, D=D)
    c.lmk.copy_(torch.randn(c.lmk.shape, generator=g, device=dev))
    c.lmk[0, 0, 500:600] = c.lmk[0, 0, 100:200]                       # a hundred ties
    c.lmk[0, 0, 500] = c.lmk[0, 0, 100] = lq[0, 0, 0]                 # and the best of all
    c.lmk[1, 0, 7] = float("nan")
    c.lmk[1, 0, 8] = float("inf")
    c.tokens.fill_(64)
    q = torch.zeros(B, H, 64, 64, device=dev, dtype=torch.bfloat16)
    kv = torch.zeros(B, H, C * 64, 64, device=dev, dtype=torch.bfloat16)
    ref = gca.forward(gca.problem(B, H, C, k, D=D, mode="decode"), lq, c.lmk, q, kv, kv)
    idx, sel, w = gca.cache_select(c, lq)
    assert torch.equal(idx, ref["idx"]) and torch.equal(sel, ref["sel"]) and torch.equal(w, ref["w"])
    assert 100 in idx[0].flatten().tolist()
    c.tokens[0, 100] = 0
    idx, _, w = gca.cache_select(c, lq, want_w=False)
    assert 100 not in idx[0].flatten().tolist() and 500 in idx[0].flatten().tolist() and w is None


# ------------------------------------------------------------------- evict ----

EVICT = [
    # B, Hr, C, k, nQ, n, decay, keep_first, keep_last
    (1, 1, 1, 1, 1, 1, 1.0, 0, 0),
    (1, 1, 1, 1, 0, 1, 1.0, 0, 1),                # the only chunk stays
    (3, 2, 50, 4, 3, 5, 0.5, 2, 4),
    (2, 1, 256, 8, 1, 256, 0.9, 1, 2),            # every slot that may go
    (2, 1, 2049, 8, 40, 700, 0.0, 5, 5),          # the masses forgotten
    (1, 3, 8191, 8, 5, 1, 0.99, 0, 0),
    (2, 1, 8192, 32, 100, 33, 1.0, 0, 64),
    (2, 1, 8193, 8, 7, 9, 0.75, 3, 0),            # a second tile of one slot
    (1, 1, 30000, 16, 300, 20000, 0.5, 0, 0),     # more than two tiles hold
    (1, 1, 20000, 8, 2, 0, 0.25, 0, 0),           # masses only
]


def _evict_state(rng, c, kind):
    B, C = c.struct.B, int(c.struct.capacity)
    tokens = np.where(rng.random((B, C)) < 0.1, -rng.integers(0, 2, (B, C)), rng.integers(1, 65, (B, C))).astype(np.int32)
    if kind == "ties":
        mass = rng.integers(0, 3, (B, C)).astype(np.float32)
    elif kind == "wide":     # magnitudes from denormal to 1e30, and what ranks as 0
        mass = np.exp(rng.uniform(-95, 69, (B, C))).astype(np.float32)
        mass.reshape(-1)[::7] = 0
        mass.reshape(-1)[1::11] = np.inf
        mass.reshape(-1)[2::13] = -1.0
    else:
        mass = rng.gamma(1.0, 1.0, (B, C)).astype(np.float32)
    number = np.stack([rng.permutation(C) for _ in range(B)]).astype(np.int32)
    nxt = np.full(B, C, np.int32) + rng.integers(0, 3, B).astype(np.int32)
    import torch
    for name, a in (("tokens", tokens), ("mass", mass), ("number", number), ("next", nxt)):
        getattr(c, name).copy_(torch.from_numpy(a))
    return tokens, mass, number, nxt


@pytest.mark.parametrize("B,Hr,C,k,nQ,n,decay,keep_first,keep_last", EVICT)
@pytest.mark.parametrize("kind", ["ties", "wide", "plain"])
def test_evict(dev, B, Hr, C, k, nQ, n, decay, keep_first, keep_last, kind):
    import torch
    from paper_2410_01651_amd import gca
    rng = np.random.default_rng(C + n)
    c = gca.cache(B, Hr, C, k, Hr=Hr, D=64)
    state = _evict_state(rng, c, kind)
    idx = w = ti = tw = want = None
    if nQ:
        idx, sel = _lists(rng, B, Hr, nQ, C, k, True)
        w = np.where(idx >= 0, rng.random(idx.shape), 0).astype(np.float32)
        flat_i, flat_w = idx.reshape(-1), w.reshape(-1)
        flat_i[::9], flat_i[1::17] = C + 3, flat_i[0]             # outside; the same slot again and again
        flat_w[2::5], flat_w[3::31] = -0.5, np.nan
        ti, tw = torch.from_numpy(idx).to(dev), torch.from_numpy(w).to(dev)
    if kind == "plain" and n:
        want = rng.integers(-1, n + 3, B).astype(np.int32)
    slots = gca.cache_evict(c, n, ti, tw, decay=decay, keep_first=keep_first, keep_last=keep_last,
                            want=torch.from_numpy(want).to(dev) if want is not None else None)
    rt, rm, rn, rx, rs = oc.evict(*state, n, idx, w, decay, keep_first, keep_last, want)
    # the masses are one fp64 fma and one rounding away from exact integers: equal to the last bit,
    # but where the fp64 product and sum, rounded apart in the oracle, meet a border of fp32
    m = c.mass.cpu().numpy()
    np.testing.assert_array_equal(slots.cpu().numpy(), rs)
    np.testing.assert_array_equal(c.tokens.cpu().numpy(), rt)
    np.testing.assert_array_equal(c.number.cpu().numpy(), rn)
    np.testing.assert_array_equal(c.next.cpu().numpy(), rx)
    assert np.array_equal(np.isfinite(m), np.isfinite(rm))
    f = np.isfinite(rm)
    assert (np.abs(m[f].astype(np.float64) - rm[f]) <= 2 * U * np.abs(rm[f])).all()


def test_evict_sum_does_not_depend_on_the_order(dev):
    """The same entries in another order give the same bits."""
    import torch
    from paper_2410_01651_amd import gca
    g = torch.Generator(device=dev).manual_seed(6)
    idx = torch.randint(0, 40, (1, 1, 5000, 8), generator=g, device=dev, dtype=torch.int32)
    w = torch.rand(idx.shape, generator=g, device=dev) ** 8
    got = []
    for p in (torch.arange(5000, device=dev), torch.randperm(5000, generator=g, device=dev)):
        c = gca.cache(1, 1, 40, 8, D=64)
        c.tokens.fill_(64)
        gca.cache_evict(c, 0, idx[:, :, p].contiguous(), w[:, :, p].contiguous())
        got.append(c.mass.clone())
    assert torch.equal(*got)
    exact = torch.zeros(40, dtype=torch.float64, device=dev).index_add_(0, idx.flatten().long(), w.flatten().double())
    assert float((got[0][0].double() - exact).abs().max()) <= float(exact.max()) * U * 1.01


@pytest.mark.parametrize("C", [6, 9000])
def test_evict_long_lists(dev, C):
    """Sums that pass 2^16: 2^16 + 11 weights of one, of more and at random for the same few slots (the
    batches of eight entries and what is left behind them), then the same and 5,000 more."""
    import torch
    from paper_2410_01651_amd import gca
    rng = np.random.default_rng(C)
    for entries in (65547, 70551):
        c = gca.cache(1, 3, C, 1, Hr=3, D=64)
        c.tokens.fill_(64)
        c.mass.fill_(0.375)
        state = tuple(x.cpu().numpy() for x in (c.tokens, c.mass, c.number, c.next))
        idx = np.full((1, 3, entries // 3, 1), C - 2, np.int32)
        w = np.ones(idx.shape, np.float32)
        idx[0, 0, ::5], w[0, 0, ::5] = 1, rng.random(w[0, 0, ::5].shape)
        w[0, 1, ::7] = 40000.0                       # (counts as 1)
        gca.cache_evict(c, 0, torch.from_numpy(idx).to(dev), torch.from_numpy(w).to(dev), decay=0.5)
        want = oc.evict(*state, 0, idx, w, 0.5)[1]
        assert want.max() > 60000
        # as in test_evict: a rounding of the oracle's sum in fp64, and of the result to fp32
        assert (np.abs(c.mass.cpu().numpy().astype(np.float64) - want) <= 2 * U * want).all()


@pytest.mark.parametrize("n,last", [(300, 300), (512, 500), (600, 600), (1200, 1111)])
def test_store_names_a_slot_again_far_behind(dev, n, last):
    """The last chunk with tokens of those that name a slot is stored, however far behind the others."""
    import torch
    from paper_2410_01651_amd import gca
    g = torch.Generator(device=dev).manual_seed(n)
    c = gca.cache(1, 1, n, 4, D=64)
    k = torch.randn(1, 1, n * 64, 64, generator=g, device=dev, dtype=torch.bfloat16)
    lmk = torch.randn(1, 1, n, 64, generator=g, device=dev, dtype=torch.bfloat16)
    slots = np.random.default_rng(n).permutation(n).astype(np.int32)
    for at, of in ((64, 0), (65, 1), (last * 9 // 10, 2), (last - 1, 3), (last - 1, last // 2), (290, 289)):
        slots[at] = slots[of]
    lengths = torch.tensor([64 * last], device=dev, dtype=torch.int32)
    gca.cache_store(c, k, k, lmk, torch.from_numpy(slots[None]).to(dev), lengths)
    holds = {}
    for i in range(last):
        holds[slots[i]] = i
    one = gca.cache(1, 1, n, 4, D=64)                # every chunk in the slot of its number
    gca.cache_store(one, k, k, lmk, torch.arange(n, device=dev, dtype=torch.int32)[None].contiguous())
    at = torch.tensor(list(holds), device=dev)
    of = torch.tensor(list(holds.values()), device=dev)
    for name in ("k", "v"):
        a, b = getattr(c, name).view(torch.uint8), getattr(one, name).view(torch.uint8)
        assert torch.equal(a[0, 0, at], b[0, 0, of])
    assert torch.equal(c.k_scale[0, 0, at], one.k_scale[0, 0, of]) and torch.equal(c.lmk[0, 0, at], one.lmk[0, 0, of])
    assert int((c.tokens > 0).sum()) == len(holds)


@pytest.mark.parametrize("fmt,dt", [("e4m3", "bf16"), ("int8", "fp32")])
def test_store_long_is_store_in_pieces(dev, fmt, dt):
    """One call of 700 chunks (captured and replayed with other slots, too) leaves what two calls of 350
    leave: slots named twice and outside the cache, sequences that end early, late or have nothing."""
    import torch
    from paper_2410_01651_amd import gca
    rng = np.random.default_rng(7)
    B, H, Hr, n, C = 4, 2, 2, 700, 900
    g = torch.Generator(device=dev).manual_seed(8)
    one, two = (gca.cache(B, H, C, 4, Hr=Hr, D=64, format=fmt, dtype=dt) for _ in range(2))
    for c in (one, two):
        c.tokens.fill_(3)
    k, v = (torch.randn(B, H, n * 64, 64, generator=g, device=dev).to(one.elem) for _ in range(2))
    lmk = torch.randn(B, Hr, n, 64, generator=g, device=dev).to(one.elem)
    half = lambda x, i: x.view(B, x.shape[1], 2, -1, 64)[:, :, i].contiguous()  # noqa: E731
    pieces = [(half(k, i), half(v, i), half(lmk, i)) for i in range(2)]
    slots = torch.zeros(B, n, dtype=torch.int32, device=dev)
    lengths = torch.tensor([0, 64 * 400 + 5, 64 * n, 64 * n + 999], dtype=torch.int32, device=dev)
    st = torch.cuda.Stream()
    gr = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(gr, stream=st):
        gca.cache_store(one, k, v, lmk, slots, lengths=lengths)
    for turn in range(4):
        slots.copy_(torch.from_numpy(rng.integers(-5, C + 5, (B, n)).astype(np.int32)))
        torch.cuda.synchronize()
        if turn == 0:
            gca.cache_store(one, k, v, lmk, slots, lengths=lengths)
        else:
            gr.replay()
        for i, piece in enumerate(pieces):
            gca.cache_store(two, *piece, slots[:, 350 * i:350 * (i + 1)].contiguous(),
                            lengths=(lengths - 64 * 350 * i).clamp(0, 64 * 350 + (999 if i else 0)))
        torch.cuda.synchronize()
        for x in one.NAMES:
            assert torch.equal(getattr(one, x).view(torch.uint8), getattr(two, x).view(torch.uint8)), (turn, x)


# ----------------------------------------------------------------- together ----

def _serve(gca, c, xs, rows, ws, st=None):
    """One chunk of every sequence: select, attend, evict, store.  The chunks themselves are
    written behind the eviction that makes room for them."""
    idx, sel, w = gca.cache_select(c, xs["lmk_q"], ws=ws["select"], stream=st)
    out, lse, _ = gca.cache_xattn(c, xs["q"], idx, sel, want_w=False, stream=st)
    slots = gca.cache_evict(c, 1, idx, w, decay=0.75, keep_first=1, keep_last=2, ws=ws["evict"], stream=st)
    gca.cache_store(c, xs["k"], xs["v"], xs["lmk"], slots, lengths=xs["lengths"], stream=st)
    return idx, sel, w, out, lse, slots


def _turn_inputs(torch, g, dev, dt, B, H, Hkv, Hr, D, rows):
    r = lambda *s: torch.randn(*s, generator=g, device=dev, dtype=dt)  # noqa: E731
    return dict(lmk_q=r(B, Hr, 1, D), q=r(B, H, rows, 64), k=r(B, Hkv, 64, 64), v=r(B, Hkv, 64, 64), lmk=r(B, Hr, 1, D),
                lengths=torch.randint(1, 65, (B,), generator=g, device=dev, dtype=torch.int32))


def _workspaces(gca, c):
    return dict(select=gca.cache_workspace(c, gca.CACHE_SELECT)[0], evict=gca.cache_workspace(c, gca.CACHE_EVICT, 1)[0])


@pytest.mark.parametrize("dtype,fmt,Hr,rows", [("bf16", "e4m3", 1, 64), ("fp32", "int8", 2, 1), ("bf16", "int8", 2, 3)])
def test_serving_loop(dev, dtype, fmt, Hr, rows):
    """Twenty chunks through caches of nine slots that start empty: every step against the oracle,
    run on the state that the device held before it."""
    import torch
    from paper_2410_01651_amd import gca
    B, H, Hkv, C, k, D = 2, 4, 2, 9, 4, 128
    c = gca.cache(B, H, C, k, Hkv=Hkv, Hr=Hr, D=D, dtype=dtype, format=fmt)
    ws = _workspaces(gca, c)
    g = torch.Generator(device=dev).manual_seed(11)
    for step in range(20):
        xs = _turn_inputs(torch, g, dev, _elem(dtype), B, H, Hkv, Hr, D, rows)
        was = {x: getattr(c, x).clone() for x in c.NAMES}
        idx, sel, w, out, lse, slots = _serve(gca, c, xs, rows, ws)
        ti, ts, tw = idx.cpu().numpy(), sel.cpu().numpy(), w.cpu().numpy()
        tokens = was["tokens"].cpu().numpy()
        ri, rs, _ = oc.select(host64(xs["lmk_q"]), host64(was["lmk"]), tokens, k, D**-0.5)
        np.testing.assert_array_equal(ti, ri)
        old = gca.cache(B, H, C, k, Hkv=Hkv, Hr=Hr, D=D, dtype=dtype, format=fmt, tensors=was)
        _check_xattn(old, xs["q"], ti, ts, (out, lse, w), rows, 0)
        rt, rm, rn, rx, rsl = oc.evict(tokens, was["mass"].cpu().numpy(), was["number"].cpu().numpy(),
                                       was["next"].cpu().numpy(), 1, ti, tw, 0.75, 1, 2)
        np.testing.assert_array_equal(slots.cpu().numpy(), rsl)
        np.testing.assert_array_equal(c.number.cpu().numpy(), rn)
        np.testing.assert_array_equal(c.next.cpu().numpy(), rx)
        for b in range(B):
            rt[b, rsl[b, 0]] = int(xs["lengths"][b])
        np.testing.assert_array_equal(c.tokens.cpu().numpy(), rt)
        assert (rsl >= 0).all() and (step >= C or rsl[0, 0] == step)     # empty slots in order, then evictions
    assert (c.number.cpu().numpy().min(axis=1) == 0).all()               # the first chunk was kept


def test_serving_step_in_a_graph(dev):
    """Two captured serving steps over two caches, replayed in turn with eager steps between, on
    their own stream: the same state and outputs as eager steps alone."""
    import torch
    from paper_2410_01651_amd import gca
    B, H, C, k, D = 3, 2, 8300, 8, 64          # two tiles of slots: the eviction needs its workspace
    st = torch.cuda.Stream()
    g = torch.Generator(device=dev).manual_seed(4)
    pairs = []
    for seed in range(2):
        made = []
        for _ in range(2):
            c = gca.cache(B, H, C, k, D=D)
            _fill(c, seed)
            c.lmk.copy_(torch.randn(c.lmk.shape, generator=torch.Generator(device=dev).manual_seed(seed), device=dev))
            c.number.copy_(torch.arange(C, device=dev, dtype=torch.int32))
            c.next.fill_(C)
            made.append((c, _workspaces(gca, c)))
        pairs.append((made, _turn_inputs(torch, g, dev, torch.bfloat16, B, H, H, 1, D, 1)))
    torch.cuda.synchronize()
    graphs = []
    for ((c, ws), _), xs in pairs:
        gr = torch.cuda.CUDAGraph()
        with torch.cuda.graph(gr, stream=st):
            res = _serve(gca, c, xs, 1, ws)
        graphs.append((gr, res))
    for turn in range(4):
        for (((c, _), (e, ws)), xs), (gr, res) in zip(pairs, graphs):
            new = _turn_inputs(torch, g, dev, torch.bfloat16, B, H, H, 1, D, 1)
            for x in xs:
                xs[x].copy_(new[x])
            torch.cuda.synchronize()
            gr.replay()
            want = _serve(gca, e, xs, 1, ws)
            torch.cuda.synchronize()
            for a, b in zip(res, want):
                assert torch.equal(a, b), turn
            for x in c.NAMES:
                assert torch.equal(getattr(c, x).view(torch.uint8), getattr(e, x).view(torch.uint8)), (turn, x)


def test_streams_side_by_side(dev):
    """Serving steps of two caches on two streams at once give what they give alone."""
    import torch
    from paper_2410_01651_amd import gca
    B, H, C, k, D = 4, 4, 500, 8, 256
    runs = []
    for _ in range(2):
        caches, sts = [], [torch.cuda.Stream() for _ in range(2)]
        for seed in range(2):
            c = gca.cache(B, H, C, k, D=D)
            _fill(c, seed)
            c.lmk.copy_(torch.randn(c.lmk.shape, generator=torch.Generator(device=dev).manual_seed(seed), device=dev))
            g = torch.Generator(device=dev).manual_seed(seed)
            caches.append((c, _workspaces(gca, c), _turn_inputs(torch, g, dev, torch.bfloat16, B, H, H, 1, D, 64)))
        torch.cuda.synchronize()
        outs = []
        for _turn in range(3):
            for (c, ws, xs), st in zip(caches, sts):
                outs.append(_serve(gca, c, xs, 64, ws, st))
                if not runs:
                    torch.cuda.synchronize()
        torch.cuda.synchronize()
        runs.append((outs, caches))
    for a, b in zip(*(r[0] for r in runs)):
        for x, y in zip(a, b):
            assert torch.equal(x, y)
    for (a, _, _), (b, _, _) in zip(*(r[1] for r in runs)):
        for x in a.NAMES:
            assert torch.equal(getattr(a, x).view(torch.uint8), getattr(b, x).view(torch.uint8))


def test_binding_refusals(dev):
    """Wrong shapes, types, strides and devices are refused before the library is called."""
    import torch
    from paper_2410_01651_amd import gca
    c = gca.cache(2, 4, 10, 3, Hkv=2, D=64)
    bf, f32, i32 = torch.bfloat16, torch.float32, torch.int32
    z = lambda *s, d=bf, on=dev: torch.zeros(*s, dtype=d, device=on)  # noqa: E731
    idx, sel = z(2, 1, 1, 3, d=i32), z(2, 1, 1, 3, d=f32)
    bad_q = [z(2, 4, 2, 64, d=f32), z(2, 2, 2, 64), z(2, 4, 2, 32), z(2, 4, 2, 64, on="cpu"), z(2, 4, 0, 64),
             z(2, 4, 64, 2).transpose(-1, -2), z(4, 2, 64)]
    for q in bad_q:
        with pytest.raises(ValueError):
            gca.cache_xattn(c, q, idx, sel)
    q = z(2, 4, 3, 64)
    for i, s in ((z(2, 1, 2, 3, d=i32), z(2, 1, 2, 3, d=f32)), (idx.long(), sel), (idx, sel.double()), (idx[..., :2], sel),
                 (idx, z(2, 2, 1, 3, d=f32))):
        with pytest.raises(ValueError):
            gca.cache_xattn(c, q, i, s)
    k, lmk, slots = z(2, 2, 128, 64), z(2, 1, 2, 64), z(2, 2, d=i32)
    for a in ((k.float(), k, lmk, slots), (k, z(2, 4, 128, 64), lmk, slots), (k, k, z(2, 1, 1, 64), slots),
              (k, k, lmk, slots.long()), (k, k, lmk, z(2, 3, d=i32)), (k, k, lmk, z(2, d=i32)),
              (z(2, 128, 2, 64).transpose(1, 2), k, lmk, slots)):
        with pytest.raises(ValueError):
            gca.cache_store(c, *a)
    with pytest.raises(gca.GcaError):
        gca.cache_store(c, z(2, 2, 0, 64), z(2, 2, 0, 64), None, z(2, 0, d=i32))
    with pytest.raises(ValueError):
        gca.cache_store(c, k, k, lmk, slots, lengths=z(3, d=i32))
    with pytest.raises(ValueError):
        gca.cache_select(c, z(2, 1, 2, 64))
    with pytest.raises(gca.GcaError, match="workspace"):
        gca.cache_select(c, z(2, 1, 1, 64), ws=z(16, d=torch.uint8))
    for kw in (dict(n=11), dict(n=-1), dict(n=1, decay=2.0), dict(n=1, idx=idx)):
        with pytest.raises((gca.GcaError, RuntimeError)):
            gca.cache_evict(c, **kw)
    with pytest.raises(ValueError):
        gca.cache_evict(c, 1, idx, sel, want=z(1, d=i32))
