"""GPU parity of the token window and of the verification of drafts against their oracle
(oracle/window.py), at the sizes, masks and values where an operator can go wrong.

Tolerances, in units of u = 2^-24 (half an fp32 step, relative).  A score is a sum of 64 exact products
in fp32, off by at most 66 u `dot`, and a bias formed in four roundings of terms of at most `bias`
(8 u `bias` with their sums).  An exponential is off by the errors of its score and of the maximum, and
by 4 u; as the running maximum grows sums are rescaled once per tile, each time by an
exponential of 4 u whose arguments add up to no more than the scores' range (2 `dot` + `bias`, at
2 u).  Sums over `seen` keys in fp32 are off by at most `seen` u.  So a row's weights are off by
rel = 4 (66 u dot + 8 u bias) + 4 u (2 dot + bias) + (2 seen + 8 tiles + 64) u, relatively, to which the rounding of the
probabilities adds 2^-11 (bf16 tensors: one fp16 term) or 2^-22 (fp32: two), both of sum p |v| (`mag`), and
the output's own rounding 2^-8 (bf16) or u of its value.  Below 2^-14 fp16 has steps of 2^-24: a scaled
probability (at most 2^15) is then off by up to 2^-25 whatever its size, 2^-40 of the block's largest value scale (within its
octave: twice) per unit of a number (`num`).  Blocks of 64 rows hold 2^-9 times a number times its scale, brought to at
most 2^15, in fp16: a value is then off by up to 2^-25 of that, 2^-31 of the largest scale's octave, 2^-30 of the scale,
and so is an output, a mean of values by weights of at most 1 together (`held`).  The verification and what is stored are exact."""

import numpy as np
import pytest

from _helpers import ensure_built, host64
from oracle import cache as oc
from oracle import window as ow

pytestmark = pytest.mark.gpu
U = 2.0**-24


@pytest.fixture(scope="module")
def dev():
    torch = pytest.importorskip("torch")
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    ensure_built()
    return torch.device("cuda:0")


@pytest.fixture(scope="module")
def gca():
    from paper_2410_01651_amd import gca as g
    return g


def _values(t):
    import torch
    if t.dtype == torch.int8:
        return t.cpu().numpy().astype(np.float64)
    return oc.e4m3_values()[t.view(torch.uint8).cpu().numpy()]


def _state(w):
    return dict(k=_values(w.k), v=_values(w.v), k_scale=host64(w.k_scale), v_scale=host64(w.v_scale),
                length=w.length.cpu().numpy().astype(np.int64))


def _fill(w, seed, length):
    """Random numbers and scales in every row, and lengths."""
    import torch
    g = torch.Generator(device=w.device).manual_seed(seed)
    for t in (w.k, w.v):
        x = torch.randint(-127, 128, t.shape, generator=g, device=w.device, dtype=torch.int8)
        if t.dtype != torch.int8:     # any code but NaN
            x = torch.where((x & 0x7F) == 0x7F, x & ~1, x)
        t.view(torch.int8).copy_(x)
    for s in (w.k_scale, w.v_scale):
        x = 2.0**-5 * torch.exp(torch.randn(s.shape, generator=g, device=w.device))
        s.copy_(x if w.k.dtype == torch.int8 else torch.exp2(torch.round(torch.log2(x)) - 1))
    w.length.copy_(torch.as_tensor(np.asarray(length), dtype=torch.int32))
    return g


def _elem(dtype):
    import torch
    return torch.bfloat16 if dtype == "bf16" else torch.float32


def _check_attn(w, q, got, parents=None, lengths=None, slopes=None, held=0.0):
    s, st = w.struct, _state(w)
    out, lse = got
    host = lambda t: None if t is None else t.cpu().numpy()  # noqa: E731
    ref = ow.attn(host64(q), st["k"], st["v"], st["k_scale"], st["v_scale"], st["length"], host(lengths), host(parents),
                  None if slopes is None else host64(slopes), s.window, s.attn_scale, bool(s.off_by_one))
    bf16 = s.dtype == 1
    score = 66 * U * ref["dot"] + 8 * U * ref["bias"]
    rel = 4 * score + 4 * U * (2 * ref["dot"] + ref["bias"]) + (2 * ref["seen"] + 8 * (ref["seen"] / 64 + 2) + 64) * U
    bound = (rel[..., None] + (2.0**-11 if bf16 else 2.0**-22)) * ref["mag"] + (2.0**-8 if bf16 else U) * np.abs(ref["out"])
    bound += 2.0**-40 * ref["num"] + 2.0**-30 * held
    err = np.abs(host64(out) - ref["out"])
    assert (err <= bound * (1 + 2.0**-7) + 1e-30).all(), float((err / (bound + 1e-300)).max())
    if lse is not None:
        x, f = host64(lse), np.isfinite(ref["lse"])
        assert np.array_equal(f, np.isfinite(x)) and (x[~f] == -np.inf).all()
        lim = rel + 16 * U * (1 + np.abs(np.where(f, ref["lse"], 0.0)))
        assert (np.abs(np.where(f, x - np.where(f, ref["lse"], 0.0), 0.0)) <= lim).all()
    return ref


ATTN = [
    # B, H, Hkv, C, window, T, tree, dtype, format, obo, slopes, length
    (1, 1, 1, 64, 0, 1, False, "bf16", "e4m3", False, False, [1]),            # one of everything
    (1, 1, 1, 64, 64, 1, False, "fp32", "int8", True, True, [1]),
    (1, 2, 1, 64, 1, 1, False, "bf16", "int8", False, True, [500]),           # a window of itself
    (3, 4, 2, 128, 0, 1, False, "bf16", "e4m3", False, True, [1, 64, 65]),    # ends of a tile
    (3, 4, 2, 128, 100, 1, False, "fp32", "e4m3", True, True, [63, 128, 1000]),
    (2, 6, 2, 192, 130, 7, False, "bf16", "int8", False, True, [7, 400]),     # 21 rows: nothing before, and a full ring
    (2, 6, 2, 192, 130, 7, True, "fp32", "int8", True, True, [7, 400]),
    (1, 16, 1, 320, 300, 1, False, "bf16", "e4m3", True, False, [299]),       # 16 rows
    (1, 17, 1, 320, 300, 1, False, "bf16", "e4m3", False, True, [301]),       # 17 rows
    (1, 33, 1, 320, 0, 1, False, "bf16", "int8", False, True, [320]),         # 33 rows, full
    (1, 40, 1, 320, 0, 1, False, "fp32", "e4m3", False, True, [320]),
    (2, 2, 2, 128, 64, 64, True, "bf16", "e4m3", False, True, [64, 777]),     # 64 nodes
    (2, 4, 2, 192, 5, 64, True, "fp32", "e4m3", False, True, [70, 900]),      # a window shorter than the tree is deep
    (2, 4, 2, 256, 0, 33, True, "bf16", "int8", True, True, [33, 250]),
    (1, 2, 1, 512, 0, 65, False, "bf16", "e4m3", False, True, [500]),         # chains that straddle blocks of rows
    (1, 3, 3, 640, 100, 200, False, "bf16", "e4m3", True, True, [1000]),
    (2, 3, 1, 640, 70, 129, False, "fp32", "int8", False, True, [129, 4097]),
    (1, 2, 2, 768, 256, 513, False, "bf16", "int8", False, False, [513]),     # window + T - 1 = C
    (1, 1, 1, 4096, 0, 1, False, "bf16", "e4m3", False, True, [4001]),        # split over workgroups
    (1, 2, 1, 4096, 0, 3, True, "fp32", "int8", True, True, [4096]),
    (1, 2, 2, 4096, 0, 64, False, "bf16", "e4m3", True, True, [3000]),
    (1, 1, 1, 8192, 8000, 20, True, "bf16", "int8", False, True, [123457]),
    (2, 8, 8, 64, 0, 5, False, "bf16", "e4m3", False, False, [66, 200]),      # tokens past the capacity
]


def _tree(rng, B, T, kind):
    par = np.full((B, T), -1, np.int32)
    for b in range(B):
        for i in range(1, T):
            par[b, i] = i - 1 if kind == "deep" else rng.integers(max(0, i - 5), i) if kind == "random" else rng.integers(-3, T + 3)
    return par


@pytest.mark.parametrize("case", ATTN, ids=lambda c: "-".join(str(x) for x in c[:9]))
def test_attn(dev, gca, case):
    import torch
    B, H, Hkv, C, window, T, tree, dtype, fmt, obo, slopes, length = case
    w = gca.window(B, H, C, window=window, Hkv=Hkv, dtype=dtype, format=fmt, off_by_one=obo, device=dev)
    g = _fill(w, 7, length)
    rng = np.random.default_rng(C + T)
    q = torch.randn(B, H, T, 64, generator=g, device=dev).to(_elem(dtype))
    sl = torch.exp2(-torch.arange(1, H + 1, device=dev, dtype=torch.float32) / H * 8) if slopes else None
    lengths = None
    if min(length) >= T and B > 1:
        lengths = torch.tensor([T] + [max(0, T - 2)] * (B - 1), dtype=torch.int32, device=dev)
    for kind in (("random", "deep", "wild") if tree else (None,)):
        par = torch.from_numpy(_tree(rng, B, T, kind)).to(dev) if tree else None
        got = gca.window_attn(w, q, parents=par, lengths=lengths, slopes=sl)
        _check_attn(w, q, got, par, lengths, sl)
    if slopes:  # without them too
        got = gca.window_attn(w, q, parents=par, lengths=lengths)
        _check_attn(w, q, got, par, lengths)


def test_attn_random(dev, gca):
    import torch
    rng = np.random.default_rng(5)
    for seed in range(40):
        Hkv = int(rng.integers(1, 5))
        G = int(rng.choice([1, 1, 2, 3, 8]))
        B, T = int(rng.integers(1, 4)), int(rng.choice([1, 2, 5, 17, 40, 64, 90, 150]))
        window = int(rng.choice([0, 0, 1, 30, 64, 200, 511]))
        length = [int(T + rng.integers(0, 700)) for _ in range(B)]
        C = -(-((window + T) if window else max(length)) // 64) * 64 + 64 * int(rng.integers(0, 3))
        dtype, fmt = str(rng.choice(["bf16", "fp32"])), str(rng.choice(["e4m3", "int8"]))
        w = gca.window(B, Hkv * G, C, window=window, Hkv=Hkv, dtype=dtype, format=fmt, off_by_one=bool(rng.integers(2)),
                       attn_scale=float(rng.choice([0.125, -0.3, 1.0, 0.0])), device=dev)
        print("random", seed, B, Hkv, G, T, window, C, dtype, fmt, flush=True)
        g = _fill(w, seed, length)
        q = torch.randn(B, Hkv * G, T, 64, generator=g, device=dev).to(_elem(dtype))
        par = torch.from_numpy(_tree(rng, B, T, "random")).to(dev) if T <= 64 and rng.integers(2) else None
        lengths = torch.from_numpy(rng.integers(0, T + 1, B).astype(np.int32)).to(dev) if rng.integers(2) else None
        sl = torch.randn(Hkv * G, generator=g, device=dev) * 0.1 if rng.integers(2) else None
        _check_attn(w, q, gca.window_attn(w, q, parents=par, lengths=lengths, slopes=sl), par, lengths, sl)


def _same(w, ref, fmt):
    """A window's tensors against the oracle's: numbers exactly, scales to a division's rounding (int8)."""
    st = _state(w)
    for x in ("k", "v"):
        assert np.array_equal(st[x], ref[x], equal_nan=True), x
    for x in ("k_scale", "v_scale"):
        nan = np.isnan(ref[x])
        assert np.array_equal(nan, np.isnan(st[x]))
        assert (np.abs(st[x] - ref[x])[~nan] <= (U * ref[x][~nan] if fmt == "int8" else 0.0)).all(), x
    assert np.array_equal(st["length"], ref["length"])
    assert not w.ticket.any()


def _int8_ties(x):
    """fp32 data whose scaled values are no near-ties, so that a rounding of the factor 127 / max does not
    show: 127 x / max is off by at most 2 u of 127."""
    y = np.abs(x) * (127.0 / np.abs(x).max(axis=-1, keepdims=True))
    return np.abs(y - np.floor(y) - 0.5) < 127 * 4 * U


APPEND = [
    # B, Hkv, C, window, T, dtype, format, length, lengths
    (1, 1, 64, 0, 1, "bf16", "e4m3", [0], None),
    (2, 3, 64, 64, 1, "fp32", "int8", [63, 64], None),
    (2, 3, 128, 100, 1, "bf16", "int8", [127, 1000001], None),
    (3, 2, 192, 64, 70, "bf16", "e4m3", [0, 5, 191], [70, 0, 33]),
    (3, 2, 192, 64, 64, "fp32", "e4m3", [64, 1, 63], [64, 65, -4]),          # counts out of range are clipped
    (2, 2, 128, 64, 300, "bf16", "e4m3", [0, 77], None),                       # more than the ring holds
    (2, 2, 128, 0, 300, "fp32", "int8", [0, 77], None),                        # more than there is room for
    (1, 2, 128, 0, 5, "bf16", "e4m3", [126], None),
    (1, 2, 128, 0, 5, "bf16", "int8", [128], None),
    (1, 16, 1024, 512, 700, "bf16", "e4m3", [900], None),                      # many workgroups
    (5, 4, 256, 100, 100, "bf16", "e4m3", [0, 3, 64, 255, 9000], [100, 0, 1, 64, 99]),  # over all sequences' tiles
    (5, 4, 256, 0, 100, "fp32", "int8", [0, 156, 157, 255, 9000], None),
    (3, 4, 128, 64, 1000, "fp32", "e4m3", [1, 0, 63], [0, 0, 0]),
    (64, 2, 192, 64, 190, "bf16", "int8", list(range(0, 640, 10)), list(range(-1, 191, 3))),
    (3, 16, 1024, 512, 3000, "bf16", "e4m3", [0, 70, 1023], [3000, 1500, 17]),
    (65, 2, 128, 64, 70, "bf16", "e4m3", list(range(65)), None),               # more sequences than lanes
    (65, 2, 128, 64, 140, "bf16", "e4m3", list(range(65)), None),
    (5, 4, 256, 100, 140, "bf16", "e4m3", [0, 3, 64, 255, 9000], [140, 0, 1, 64, 99]),
    (5, 4, 256, 0, 150, "fp32", "int8", [0, 106, 107, 255, 9000], None),
    (3, 2, 192, 64, 129, "bf16", "e4m3", [0, 5, 191], [129, 0, 33]),
    (2, 3, 128, 100, 128, "bf16", "int8", [127, 1000001], None),
    (1, 2, 64, 64, 128, "fp32", "e4m3", [3], None),                            # twice what the ring holds
]


@pytest.mark.parametrize("case", APPEND, ids=lambda c: "-".join(str(x) for x in c[:7]))
def test_append(dev, gca, case):
    import torch
    B, Hkv, C, window, T, dtype, fmt, length, lengths = case
    w = gca.window(B, Hkv, C, window=window, dtype=dtype, format=fmt, device=dev)
    g = _fill(w, 3, length)
    ref = _state(w)
    for rep in range(2):
        k, v = (torch.randn(B, Hkv, T, 64, generator=g, device=dev).to(_elem(dtype)) for _ in range(2))
        for x in (k, v):
            x.mul_(torch.exp2(torch.randint(-20, 20, (B, Hkv, T, 1), generator=g, device=dev).float()).to(x.dtype))
            if fmt == "int8":
                x[torch.from_numpy(_int8_ties(host64(x))).to(dev)] = 0.0
        n = None if lengths is None else torch.tensor(lengths, dtype=torch.int32, device=dev)
        gca.window_append(w, k, v, lengths=n)
        ow.append(ref, host64(k), host64(v), lengths, fmt, window)
        _same(w, ref, fmt)


def test_append_special_values(dev, gca):
    """Rows of zeros, of the smallest and largest numbers, infinities and NaN, alone and together."""
    import torch
    inf, nan = float("inf"), float("nan")
    rows = [[0.0], [2.0**-126], [1e-38, -1e-38], [3e38, -3e38, 1.0], [inf, 1.0, -2.0], [-inf], [nan], [nan, 5.0, inf], [448.0], [448.1],
            [449.0, -0.25], [480.0, 1.0], [464.0], [1.0, -0.0]]
    for dtype in ("fp32", "bf16"):
        for fmt in ("e4m3", "int8"):
            w = gca.window(1, 1, 64, window=64, dtype=dtype, format=fmt, device=dev)
            ref = _state(w)
            x = torch.zeros(1, 1, len(rows), 64, device=dev)
            for i, r in enumerate(rows):
                x[0, 0, i, 7:7 + len(r)] = torch.tensor(r, device=dev)
            x = x.to(_elem(dtype))
            y = x.flip(-1).contiguous()
            gca.window_append(w, x, y)
            ow.append(ref, host64(x), host64(y), None, fmt, 64)
            st = _state(w)
            for name in ("k_scale", "v_scale"):
                a, b = st[name], ref[name]
                assert np.array_equal(np.isnan(a), np.isnan(b))
                assert (np.abs(a - b)[~np.isnan(b)] <= 2 * U * b[~np.isnan(b)] + 1e-45).all()
            assert np.array_equal(st["v"], ref["v"], equal_nan=True)
            bad = np.isnan(ref["k"]).any(axis=-1)
            assert np.array_equal(st["k"][~bad], ref["k"][~bad])
            assert np.isfinite(st["v"]).all()


@pytest.mark.parametrize("window,C,fmt", [(0, 128, "e4m3"), (64, 128, "int8"), (100, 192, "e4m3"), (0, 64, "int8")])
def test_keep(dev, gca, window, C, fmt):
    import torch
    rng = np.random.default_rng(C)
    B, Hkv, T = 9, 3, 27
    w = gca.window(B, Hkv * 2, C, window=window, Hkv=Hkv, format=fmt, device=dev)
    for n in (0, 1, 5, 27, 64):
        _fill(w, n, [T, 27 + 30, 64, 65, 100, 128, 5, 0, 60 + 27] if window == 0 else [T, 57, 200, 999, 129, 128, 64, 63, 12345])
        ref = _state(w)
        path = np.full((B, n), -1, np.int32)
        for b in range(B):
            m = min(n, int(rng.integers(0, T + 1)))
            path[b, :m] = np.sort(rng.choice(T, m, replace=False))
        if n >= 5:
            path[1, :3] = [0, 0, 1]         # twice the same
            path[2, :3] = [4, 2, 9]         # descending
            path[3, :3] = [1, 40, 50]       # behind the tokens
            path[4, :3] = [-1, 3, 4]        # nothing first
        lengths = torch.tensor([T, 3, T, T, T, 0, T, -1, 99], dtype=torch.int32, device=dev)
        gca.window_keep(w, T, torch.from_numpy(path).to(dev), lengths=lengths)
        ow.keep(ref, path, lengths.cpu().numpy(), T, window)
        _same(w, ref, "e4m3")


def test_keep_ends_where_a_token_was_not_kept(dev, gca):
    """As the oracle's: in a window of 64 rows, tokens from position 64 on have none."""
    import torch
    for path in ([0, 2, 3, 5], [0, 1, 2, 3, 5], [4], [0, 1, 2, 3, 4, 5], [5]):
        w = gca.window(3, 2, 64, device=dev)
        _fill(w, 9, [66, 60, 70])
        ref = _state(w)
        p = np.array([path] * 3, np.int32)
        gca.window_keep(w, 6, torch.from_numpy(p).to(dev))
        ow.keep(ref, p, None, 6, 0)
        _same(w, ref, "e4m3")


def _drafts(rng, B, T, V, kind, with_q):
    p = rng.standard_normal((B, T, V)) * 2
    q = p + rng.standard_normal((B, T, V)) * (0.5 if kind != "far" else 4.0)
    p, q = (np.exp(x - x.max(-1, keepdims=True)) for x in (p, q))
    p, q = ((x / x.sum(-1, keepdims=True)).astype(np.float32) for x in (p, q))
    par = _tree(rng, B, T, "random") if kind != "wild" else _tree(rng, B, T, "wild")
    tok = np.zeros((B, T), np.int32)
    for b in range(B):
        for i in range(T):
            a = max(0, min(T - 1, par[b, i]))
            tok[b, i] = rng.choice(V, p=q[b, a].astype(np.float64) / q[b, a].astype(np.float64).sum())
    u = rng.random((B, T)).astype(np.float32)
    return p, (q if with_q else None), par, tok, u


@pytest.mark.parametrize("B,T,V,kind,with_q", [
    (1, 1, 1, "chain", False), (1, 1, 7, "chain", True), (3, 5, 33, "chain", True), (3, 5, 33, "chain", False), (17, 2, 300, "far", True),
    (5, 64, 40, "tree", True), (5, 64, 40, "tree", False), (6, 20, 4099, "tree", True), (6, 20, 4099, "far", True), (6, 20, 5000, "far", False),
    (7, 30, 64, "wild", True), (7, 30, 64, "wild", False), (2, 9, 50000, "tree", True), (2, 3, 262145, "far", True), (300, 4, 1000, "tree", True),
    (1, 2, 524288, "tree", False)])
def test_verify(dev, gca, B, T, V, kind, with_q):
    import torch
    rng = np.random.default_rng(B * T + V)
    for rep in range(3):
        p, q, par, tok, u = _drafts(rng, B, T, V, kind, with_q)
        if kind == "chain":
            par = None
        lengths = rng.integers(0, T + 2, B).astype(np.int32) if rep == 2 else None
        if kind == "wild":
            tok[rng.random(tok.shape) < 0.2] = -5
            tok[rng.random(tok.shape) < 0.2] = V
            u[rng.random(u.shape) < 0.1] = 1.0
            u[rng.random(u.shape) < 0.1] = 0.0
            u[rng.random(u.shape) < 0.1] = np.nan
        up = lambda x: None if x is None else torch.from_numpy(x).to(dev)  # noqa: E731
        got = gca.verify(up(p), up(tok), up(u), q=up(q), parents=up(par), lengths=up(lengths))
        want = ow.verify(p, tok, u, q, par, lengths)
        for x, y, name in zip(got, want, ("path", "count", "next")):
            assert np.array_equal(x.cpu().numpy(), y), name


def test_verify_odd_probabilities(dev, gca):
    """NaN, negative, large and vanishing probabilities; p equal to q, so that rejection leaves nothing; tokens named
    twice; one-hot targets (greedy)."""
    import torch
    rng = np.random.default_rng(1)
    B, T, V = 8, 12, 1500
    for with_q in (False, True):
        p, q, par, tok, u = _drafts(rng, B, T, V, "tree", with_q)
        p[0, :, ::3] = np.nan
        p[1, :, ::2] = -1.0
        p[2] = 1e30
        p[3] = 0.0
        p[4] = 2.0**-60
        tok[5] = tok[5, 1]
        p[6] = 0.0
        p[6, :, 77] = 1.0
        tok[6, ::2] = 77
        if with_q:
            q[0, :, ::5] = np.inf
            q[1, :, ::7] = np.nan
            q[7] = p[7]
            u[7] = np.float32(1 - 2.0**-24)
            q[5] = 0.0
        up = lambda x: None if x is None else torch.from_numpy(x).to(dev)  # noqa: E731
        got = gca.verify(up(p), up(tok), up(u), q=up(q), parents=up(par))
        want = ow.verify(p, tok, u, q, par)
        for x, y, name in zip(got, want, ("path", "count", "next")):
            assert np.array_equal(x.cpu().numpy(), y), name
        assert (got[2][3] == -1).item() and (got[2][4] == -1).item()


@pytest.mark.parametrize("with_q", [False, True])
def test_verify_of_the_largest_sum(dev, gca, with_q):
    """2^19 probabilities of 1 are 2^63 in whole multiples of 2^-44.  (With a first draft that q does not have, and so
    is accepted, or with drafts that leave p as it is: their tokens are no tokens.)"""
    import torch
    B, T, V = 3, 3, 1 << 19
    p = np.ones((B, T, V), np.float32)
    q = np.zeros((B, T, V), np.float32) if with_q else None
    tok = np.array([[0, -1, V], [0, 5, -1], [0, V - 1, 7]], np.int32)
    par = np.array([[-1, 0, 0]] * B, np.int32)
    u = np.array([[0.75, 0.5, 0.5], [0.0, 0.25, 0.5], [1 - 2.0**-24, 0.9, 0.9]], np.float32)
    up = lambda x: None if x is None else torch.from_numpy(x).to(dev)  # noqa: E731
    got = gca.verify(up(p), up(tok), up(u), q=up(q), parents=up(par))
    want = ow.verify(p, tok, u, q, par)
    assert want[2][0] == 3 << 17
    for x, y, name in zip(got, want, ("path", "count", "next")):
        assert np.array_equal(x.cpu().numpy(), y), name
