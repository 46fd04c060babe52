"""The token window and the verification of drafts as programs use them: whole steps, graphs, other streams,
odd values in places that a row does not see, long windows, refusals of the binding."""

import numpy as np
import pytest

import test_gpu_window as tw
from _helpers import ensure_built, host64
from oracle import window as ow

pytestmark = pytest.mark.gpu


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


# B, H, Hkv, C, T, tree, dtype, format, lengths: windows without an end, whose sequences differ in length (one
# workgroup per row block and several; heads that do not fill the XCDs; none, one, all tokens)
UNEQUAL = [
    (2, 2, 1, 4096, 1, False, "bf16", "e4m3", [1, 4096]),
    (5, 8, 2, 4096, 1, False, "bf16", "int8", [4096, 3, 700, 64, 2000]),
    (3, 6, 3, 2048, 20, True, "fp32", "e4m3", [20, 2048, 1111]),
    (64, 4, 4, 1024, 9, True, "bf16", "e4m3", None),
    (33, 8, 1, 1088, 5, False, "fp32", "int8", None),
    (16, 8, 8, 2048, 1, False, "bf16", "e4m3", None),
    (9, 32, 2, 1024, 40, True, "bf16", "e4m3", None),
    (65, 1, 1, 1024, 1, False, "bf16", "e4m3", None),      # more sequences than lanes
    (4, 2, 2, 8192, 70, False, "bf16", "e4m3", [70, 8192, 5000, 200]),
    (2, 1, 1, 16384, 200, False, "bf16", "e4m3", [16384, 201]),  # more row blocks than tickets
]


@pytest.mark.parametrize("case", UNEQUAL, ids=lambda c: "-".join(str(x) for x in c[:8]))
def test_attn_of_unequal_sequences(dev, gca, case):
    import torch
    B, H, Hkv, C, T, tree, dtype, fmt, length = case
    rng = np.random.default_rng(B + C)
    if length is None:
        length = [int(x) for x in rng.integers(T, C + 1, B)]
        length[B // 2] = T
    w = gca.window(B, H, C, Hkv=Hkv, dtype=dtype, format=fmt, device=dev)
    g = tw._fill(w, 11, length)
    q = torch.randn(B, H, T, 64, generator=g, device=dev).to(tw._elem(dtype))
    par = torch.from_numpy(tw._tree(rng, B, T, "random")).to(dev) if tree else None
    sl = torch.rand(H, generator=g, device=dev) * 0.05
    ws = gca.window_workspace(w, T)[0].fill_(255)    # whatever it holds
    for rep in range(2):
        got = gca.window_attn(w, q, parents=par, slopes=sl, ws=ws)
        tw._check_attn(w, q, got, par, None, sl)
    assert not w.ticket.any()


@pytest.mark.parametrize("B,T,G,C,window,fmt", [
    (3, 64, 8, 1024, 0, "int8"), (3, 33, 2, 1024, 0, "e4m3"), (3, 70, 3, 1024, 0, "e4m3"), (4, 1, 8, 1024, 0, "e4m3"), (4, 5, 8, 1024, 0, "int8"),
    (5, 20, 3, 2048, 0, "e4m3"), (3, 130, 1, 1024, 0, "e4m3"), (2, 5, 3, 512, 0, "e4m3"), (3, 64, 8, 1024, 900, "int8"), (4, 9, 4, 1024, 500, "e4m3"),
    (1, 64, 4, 4096, 0, "e4m3"), (70, 40, 2, 1024, 0, "e4m3"), (4, 64, 4, 512, 0, "e4m3"), (128, 64, 8, 128, 64, "e4m3")])
def test_every_row_is_written(dev, gca, B, T, G, C, window, fmt):
    """Whatever part of the rows has tokens (none of a sequence's, or of all, among them): out and lse hold NaN before."""
    import torch
    Hkv = 2
    rng = np.random.default_rng(T + G)
    w = gca.window(B, Hkv * G, C, window=window, Hkv=Hkv, format=fmt, device=dev)
    g = tw._fill(w, 3, [int(x) for x in rng.integers(T, C + 1, B)])
    q = torch.randn(B, Hkv * G, T, 64, generator=g, device=dev).bfloat16()
    some = rng.integers(0, T + 1, B)
    some[B // 2] = 0
    few = np.full(B, T)
    few[0] = 0
    for n in (some, few, np.zeros(B), np.minimum(1, some), None):
        lengths = None if n is None else torch.from_numpy(n.astype(np.int32)).to(dev)
        for tree in ((False, True) if T <= 64 else (False,)):
            par = torch.from_numpy(tw._tree(rng, B, T, "random")).to(dev) if tree else None
            out = torch.full_like(q, float("nan"))
            lse = torch.full(q.shape[:3], float("nan"), device=dev)
            gca.window_attn(w, q, parents=par, lengths=lengths, out=out, lse=lse)
            at = torch.arange(T, device=dev)[None, None] >= (T if n is None else lengths[:, None, None])
            at = at.expand(B, Hkv * G, T)
            assert (out[at] == 0).all() and (lse[at] == -float("inf")).all()
            assert torch.isfinite(out[~at]).all() and torch.isfinite(lse[~at]).all()
    assert not w.ticket.any()


@pytest.mark.parametrize("dtype,fmt,B,T,G", [("bf16", "e4m3", 2, 9, 1), ("fp32", "int8", 2, 9, 1), ("bf16", "int8", 2, 9, 4),
                                              ("bf16", "e4m3", 16, 64, 4), ("fp32", "e4m3", 2, 33, 2), ("bf16", "e4m3", 1, 1, 1)])
def test_odd_values_that_a_row_does_not_see(dev, gca, dtype, fmt, B, T, G):
    """NaN and infinities among the keys and values of sibling nodes, of tokens behind the window and of
    rows never written have no effect; those that a row sees come out as NaN."""
    import torch
    Hkv = 8
    C, window = 192, 70
    w = gca.window(B, Hkv * G, C, window=window, Hkv=Hkv, dtype=dtype, format=fmt, device=dev)
    for t in (w.k, w.v):
        t.view(torch.uint8).fill_(0x7F)           # never written: NaN numbers, NaN scales
    for t in (w.k_scale, w.v_scale):
        t.fill_(float("nan"))
    g = torch.Generator(device=dev).manual_seed(1)
    rand = lambda *s: torch.randn(*s, generator=g, device=dev).to(tw._elem(dtype))  # noqa: E731
    n0 = 100
    k, v = rand(B, Hkv, n0, 64), rand(B, Hkv, n0, 64)
    k[:, :, 3, 5] = float("nan")                  # behind every row's window
    v[:, :, 4, 5] = float("nan")
    v[:, :, 5, 6] = float("inf")
    gca.window_append(w, k, v)
    k, v = rand(B, Hkv, T, 64), rand(B, Hkv, T, 64)
    bad = T // 2
    if T > 2:
        k[:, :, bad, 1], v[:, :, bad, 2] = float("nan"), float("nan")
    par = np.tile(np.array([-1] + [0] * (T - 1), np.int32), (B, 1))   # siblings, and one child of the bad node
    if T > 2:
        par[:, T - 1] = bad
    par = torch.from_numpy(par).to(dev)
    gca.window_append(w, k, v)
    q = rand(B, Hkv * G, T, 64)
    out, lse = gca.window_attn(w, q, parents=par)
    out, lse = host64(out), host64(lse)
    hit = np.zeros(T, bool)
    if T > 2:
        hit[[bad, T - 1]] = True
    assert np.isnan(out[:, :, hit]).all() and np.isfinite(out[:, :, ~hit]).all() and np.isfinite(lse[:, :, ~hit]).all()
    # the same with ordinary values in those places
    c = gca.window(B, Hkv * G, C, window=window, Hkv=Hkv, dtype=dtype, format=fmt, device=dev)
    for name in ("k", "v", "k_scale", "v_scale", "length"):
        getattr(c, name).view(torch.uint8).copy_(getattr(w, name).view(torch.uint8))
    for name in ("k_scale", "v_scale"):
        getattr(c, name).nan_to_num_(0.5)
    if fmt == "e4m3":     # (int8: every code is a number)
        for name in ("k", "v"):
            x = getattr(c, name).view(torch.uint8)
            x[(x & 0x7F) == 0x7F] = 1
    out2, lse2 = (host64(x) for x in gca.window_attn(c, q, parents=par))
    # The scores are the same.  A sibling's value scale of 1/2 may be the block's largest, by which every row's
    # probabilities are scaled before they are rounded: each side is off by its rounding of them, 2^-11 or 2^-22 of
    # sum p |v|, at most the largest |v|, or 2^-40 of twice that scale per unit of a number (at most 448 of each of C),
    # and by the output's.
    assert np.array_equal(lse[:, :, ~hit], lse2[:, :, ~hit])
    top = float(max(k.float().nan_to_num(0.0).abs().max(), v.float().nan_to_num(0.0).abs().max(), 8.0)) * 1.0625
    lim = 2 * ((2.0**-11 + 2.0**-8 if dtype == "bf16" else 2.0**-22 + tw.U) * top + 2.0**-40 * 448 * C)
    assert np.abs(out - out2)[:, :, ~hit].max() <= lim


def test_scores_and_scales_at_the_ends_of_their_range(dev, gca):
    """Value scales from 2^-126 to 2^100 in one window, scores of hundreds, slopes that leave one token."""
    import torch
    for dtype in ("bf16", "fp32"):
        for fmt in ("e4m3", "int8"):
            for H, T in ((1, 1), (2, 20), (40, 64)):
                w = gca.window(2, H, 640, window=500, dtype=dtype, format=fmt, device=dev)
                g = tw._fill(w, 5, [640, 90])
                e = torch.randint(-126, 100, w.v_scale.shape, generator=g, device=dev).float()
                w.v_scale.copy_(torch.exp2(e))
                w.k_scale.mul_(64.0 if fmt == "e4m3" else 3.0)
                q = torch.randn(2, H, T, 64, generator=g, device=dev).to(tw._elem(dtype))
                sl = torch.logspace(-3, 2, H, device=dev)
                tw._check_attn(w, q, gca.window_attn(w, q, slopes=sl, lengths=torch.tensor([T, T], dtype=torch.int32, device=dev)),
                               None, None, sl)


@pytest.mark.parametrize("T,G,tree", [(1, 33, False), (40, 1, True), (64, 1, False)])
def test_scales_far_apart_in_blocks_of_64_rows(dev, gca, T, G, tree):
    """So many sequences that blocks have 64 rows, and value scales from 2^-20 to 2^20, the largest ones among the
    oldest tokens or the newest; three of the sequences are compared."""
    import torch
    from types import SimpleNamespace
    B, Hkv, C = 256, 8, 128
    w = gca.window(B, Hkv * G, C, Hkv=Hkv, device=dev)
    g = tw._fill(w, 21, [C] * B)
    q = torch.randn(B, Hkv * G, T, 64, generator=g, device=dev).to(torch.bfloat16)
    par = torch.from_numpy(tw._tree(np.random.default_rng(2), B, T, "random")).to(dev) if tree else None
    sl = torch.full((Hkv * G,), 0.5, device=dev)
    for turned in (False, True):
        e = torch.linspace(20, -20, C, device=dev).round()
        w.v_scale.copy_(torch.exp2(e.flip(0) if turned else e))
        out, lse = gca.window_attn(w, q, parents=par, slopes=sl)
        for b in (0, 100, B - 1):
            one = SimpleNamespace(struct=w.struct, **{n: getattr(w, n)[b:b + 1] for n in w.NAMES})
            tw._check_attn(one, q[b:b + 1], (out[b:b + 1], lse[b:b + 1]), None if par is None else par[b:b + 1], None, sl,
                           held=2.0**20)


def _step(gca, w, k, v, q, par, p, qd, tok, u, ws):
    """A step of a serving loop: the drafts join the window, attend, are verified, and the accepted path stays."""
    gca.window_append(w, k, v)
    out, lse = gca.window_attn(w, q, parents=par, ws=ws)
    path, count, nxt = gca.verify(p, tok, u, q=qd, parents=par)
    gca.window_keep(w, q.shape[2], path)
    return out, lse, path, count, nxt


@pytest.mark.parametrize("window,C,fmt,dtype", [(100, 192, "e4m3", "bf16"), (0, 512, "int8", "fp32")])
def test_serving_loop(dev, gca, window, C, fmt, dtype):
    """Prompts of different lengths, then steps with trees of drafts, against the oracle's."""
    import torch
    rng = np.random.default_rng(2)
    B, H, Hkv, T, V = 3, 4, 2, 11, 50
    w = gca.window(B, H, C, window=window, Hkv=Hkv, dtype=dtype, format=fmt, device=dev)
    g = torch.Generator(device=dev).manual_seed(3)
    rand = lambda *s: torch.randn(*s, generator=g, device=dev).to(tw._elem(dtype))  # noqa: E731
    ref = tw._state(w)
    k, v, n = rand(B, Hkv, 90, 64), rand(B, Hkv, 90, 64), torch.tensor([90, 1, 0], dtype=torch.int32, device=dev)
    gca.window_append(w, k, v, lengths=n)
    ow.append(ref, host64(k), host64(v), n.cpu().numpy(), fmt, window)
    q = rand(B, H, 90, 64)
    tw._check_attn(w, q, gca.window_attn(w, q, lengths=n), None, n)
    for step in range(12):
        k, v, q = rand(B, Hkv, T, 64), rand(B, Hkv, T, 64), rand(B, H, T, 64)
        p, qd, par, tok, u = tw._drafts(rng, B, T, V, "tree", step % 2 == 0)
        up = lambda x: None if x is None else torch.from_numpy(x).to(dev)  # noqa: E731
        gca.window_append(w, k, v)
        got = gca.window_attn(w, q, parents=up(par))
        tw._check_attn(w, q, got, up(par))
        path, count, nxt = gca.verify(up(p), up(tok), up(u), q=up(qd), parents=up(par))
        want = ow.verify(p, tok, u, qd, par)
        assert all(np.array_equal(a.cpu().numpy(), b) for a, b in zip((path, count, nxt), want))
        gca.window_keep(w, T, path)
        ow.append(ref, host64(k), host64(v), None, fmt, window)
        ow.keep(ref, want[0], None, T, window)
        assert np.array_equal(w.length.cpu().numpy(), ref["length"])
    st = tw._state(w)
    for b in range(B):
        for pos in range(max(0, int(ref["length"][b]) - (window or C)), int(ref["length"][b])):
            r = ow.row_of(pos, C, window)
            got = st["k"][b, :, r] * st["k_scale"][b, :, r, None], st["v"][b, :, r // 64, :, r % 64] * st["v_scale"][b, :, r, None]
            wish = ref["k"][b, :, r] * ref["k_scale"][b, :, r, None], ref["v"][b, :, r // 64, :, r % 64] * ref["v_scale"][b, :, r, None]
            for x, y in zip(got, wish):   # (int8: a near-tie may round the other way)
                lim = 0.0 if fmt == "e4m3" else 1.01 * np.abs(y).max(axis=-1, keepdims=True) / 127
                assert (np.abs(x - y) <= lim).all()


def test_pieces_of_a_prompt_equal_one_call(dev, gca):
    """A prompt appended and attended to in pieces gives what one call gives, bit for bit where the
    tiles are cut alike, and within the rounding of its parts everywhere."""
    import torch
    B, H, L, window, C = 2, 2, 700, 200, 1024
    g = torch.Generator(device=dev).manual_seed(9)
    k, v, q = (torch.randn(B, H, L, 64, generator=g, device=dev).bfloat16() for _ in range(3))
    one = gca.window(B, H, C, window=window, device=dev)
    gca.window_append(one, k, v)
    whole, _ = gca.window_attn(one, q)
    tw._check_attn(one, q, (whole, None))
    two = gca.window(B, H, C, window=window, device=dev)
    at = 0
    for n in (1, 63, 64, 100, 7, 465):
        part = lambda x: x[:, :, at:at + n].contiguous()  # noqa: E731
        gca.window_append(two, part(k), part(v))
        out, _ = gca.window_attn(two, part(q))
        tw._check_attn(two, part(q), (out, None))
        at += n
    assert at == L
    for name in ("k", "v", "k_scale", "v_scale", "length"):
        assert torch.equal(getattr(one, name).view(torch.uint8), getattr(two, name).view(torch.uint8)), name


def test_graph_of_a_step(dev, gca):
    """A step captured into a graph and replayed, with eager work between, equals eager steps bit for bit."""
    import torch
    rng = np.random.default_rng(4)
    B, H, Hkv, C, T, V = 4, 8, 2, 4096, 7, 5000
    p, qd, par, tok, u = tw._drafts(rng, B, T, V, "tree", True)
    up = lambda x: torch.from_numpy(x).to(dev)  # noqa: E731
    p, qd, par, tok, u = up(p), up(qd), up(par), up(tok), up(u)
    wins = [gca.window(B, H, C, Hkv=Hkv, device=dev) for _ in range(2)]
    for w in wins:
        g = tw._fill(w, 8, [3000, 100, 2500, 8])
    k, v, q = (torch.randn(B, h, T, 64, generator=g, device=dev).bfloat16() for h in (Hkv, Hkv, H))
    ws = [gca.window_workspace(w, T)[0] for w in wins]
    vs = gca.verify_workspace(B, T, V)[0]
    torch.cuda.synchronize()

    def step(w, s):
        gca.window_append(w, k, v)
        out, lse = gca.window_attn(w, q, parents=par, ws=s)
        path, count, nxt = gca.verify(p, tok, u, q=qd, parents=par, ws=vs)
        gca.window_keep(w, T, path)
        return out, lse, path, count, nxt

    graph = torch.cuda.CUDAGraph()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        with torch.cuda.graph(graph, stream=side):
            captured = step(wins[0], ws[0])
    torch.cuda.synchronize()
    assert not wins[0].ticket.any()
    for rep in range(5):
        k.normal_(generator=g)
        q.normal_(generator=g)
        u.uniform_(generator=g)
        eager = step(wins[1], ws[1])
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip(captured, eager):
            assert torch.equal(a, b)
        for name in ("k", "v", "k_scale", "v_scale", "length", "ticket"):
            assert torch.equal(getattr(wins[0], name).view(torch.uint8), getattr(wins[1], name).view(torch.uint8)), (rep, name)


def test_other_streams_and_two_windows_at_once(dev, gca):
    import torch
    B, H, C, T = 2, 4, 4096, 3
    g = torch.Generator(device=dev).manual_seed(6)
    wins = [gca.window(B, H, C, device=dev) for _ in range(2)]
    for i, w in enumerate(wins):
        tw._fill(w, 20 + i, [4000, 1500])
    q = [torch.randn(B, H, T, 64, generator=g, device=dev).bfloat16() for _ in wins]
    want = [gca.window_attn(w, x) for w, x in zip(wins, q)]
    streams = [torch.cuda.Stream() for _ in wins]
    torch.cuda.synchronize()
    got = [[], []]
    for rep in range(20):
        for i, (w, x, s) in enumerate(zip(wins, q, streams)):
            got[i].append(gca.window_attn(w, x, stream=s))
    torch.cuda.synchronize()
    for i in range(2):
        for out, lse in got[i]:
            assert torch.equal(out, want[i][0]) and torch.equal(lse, want[i][1])
    # an append, an attention and a roll-back ordered on a stream of their own
    before = [t.clone() for t in (wins[0].k_scale, wins[0].length)]
    k = torch.randn(B, H, T, 64, generator=g, device=dev).bfloat16()
    none = torch.empty(B, 0, dtype=torch.int32, device=dev)
    torch.cuda.synchronize()
    gca.window_append(wins[0], k, k, stream=streams[0])
    gca.window_keep(wins[0], T, none, stream=streams[0])
    torch.cuda.synchronize()
    assert torch.equal(wins[0].length, before[1])


def test_long_window_passes_32_bits(dev, gca):
    """Rows whose bytes lie past 2^32 from the tensors' start."""
    import torch
    B, H, C = 2, 36, 1 << 20        # 2 x 36 x 2^20 x 64 bytes = 4.8 GB each
    if torch.cuda.mem_get_info(dev)[0] < 24 << 30:
        pytest.skip("not enough free memory")
    w = gca.window(B, H, C, device=dev)
    w.length.fill_(C - 130)
    g = torch.Generator(device=dev).manual_seed(1)
    k, v = (torch.randn(B, H, 130, 64, generator=g, device=dev).bfloat16() for _ in range(2))
    gca.window_append(w, k, v)
    assert (w.length == C).all()
    assert w.k_scale[:, :, C - 130:].all() and not w.k_scale[:, :, :C - 130].any()
    q = torch.randn(B, H, 1, 64, generator=g, device=dev).bfloat16()
    sl = torch.full((H,), 4.0, device=dev)      # (zeros further back weigh nothing)
    out, lse = gca.window_attn(w, q, slopes=sl)
    r = slice(C - 130, C)
    last = host64(w.v.view(torch.uint8)[-1, -1, C // 64 - 3:].view(w.v.dtype).float().transpose(1, 2).reshape(-1, 64)[-130:])
    kk = host64(w.k.view(torch.uint8)[-1, -1, r].view(w.k.dtype).float()) * host64(w.k_scale[-1, -1, r])[:, None]
    s = kk @ host64(q[-1, -1, 0]) / 8 + 4.0 * np.arange(-129, 1)
    e = np.exp(s - s.max())
    ref = (e / e.sum()) @ (last * host64(w.v_scale[-1, -1, r])[:, None])
    assert np.abs(host64(out[-1, -1, 0]) - ref).max() <= (2.0**-8 + 2.0**-10) * np.abs(ref).max() + 2.0**-11 * np.abs(last).max()


def test_binding_refuses(dev, gca):
    import torch
    w = gca.window(2, 4, 128, window=100, Hkv=2, device=dev)
    q = torch.zeros(2, 4, 3, 64, dtype=torch.bfloat16, device=dev)
    k = torch.zeros(2, 2, 3, 64, dtype=torch.bfloat16, device=dev)
    i32 = lambda *s: torch.zeros(*s, dtype=torch.int32, device=dev)  # noqa: E731
    for call, word in (
            (lambda: gca.window_append(w, k.float(), k), "k must be"), (lambda: gca.window_append(w, k, k[:, :1]), "v must"),
            (lambda: gca.window_append(w, k, k.transpose(1, 2).contiguous().transpose(1, 2)), "contiguous"),
            (lambda: gca.window_append(w, k[0], k), "shape"), (lambda: gca.window_append(w, k, k, lengths=i32(3)), "lengths"),
            (lambda: gca.window_attn(w, q[:, :2]), "q must"), (lambda: gca.window_attn(w, q, parents=i32(2, 4)), "parents"),
            (lambda: gca.window_attn(w, q, slopes=torch.zeros(2, device=dev)), "slopes"), (lambda: gca.window_attn(w, q.cpu()), "device"),
            (lambda: gca.window_attn(w, q, out=q.float()), "out"), (lambda: gca.window_attn(w, q, lse=torch.zeros(2, 4, device=dev)), "lse"),
            (lambda: gca.window_keep(w, 3, i32(2)), "path"), (lambda: gca.window_keep(w, 3, i32(2, 3).long()), "path"),
            (lambda: gca.verify(torch.zeros(2, 3, device=dev), i32(2, 3), torch.zeros(2, 3, device=dev)), "shape"),
            (lambda: gca.verify(torch.zeros(2, 3, 5, device=dev), i32(2, 2), torch.zeros(2, 3, device=dev)), "tokens"),
            (lambda: gca.verify(torch.zeros(2, 3, 5, device=dev), i32(2, 3), torch.zeros(2, 3, device=dev), q=torch.zeros(2, 3, 4, device=dev)), "q must"),
            (lambda: gca.window(2, 4, 128, tensors=dict(length=torch.zeros(2, dtype=torch.int64, device=dev))), "length")):
        with pytest.raises(ValueError, match=word):
            call()
    for call, status in (
            (lambda: gca.window_attn(w, torch.zeros(2, 4, 30, 64, dtype=torch.bfloat16, device=dev)), gca.GCA_ERR_INVALID),
            (lambda: gca.window_attn(gca.window(1, 1, 128, device=dev), torch.zeros(1, 1, 65, 64, dtype=torch.bfloat16, device=dev),
                                     parents=i32(1, 65)), gca.GCA_ERR_UNSUPPORTED),
            (lambda: gca.window_append(gca.window(1, 1, 100, device=dev), k[:1, :1], k[:1, :1]), gca.GCA_ERR_UNSUPPORTED),
            (lambda: gca.window_keep(w, 3, i32(2, 65)), gca.GCA_ERR_UNSUPPORTED),
            (lambda: gca.verify(torch.zeros(1, 65, 5, device=dev), i32(1, 65), torch.zeros(1, 65, device=dev)), gca.GCA_ERR_UNSUPPORTED)):
        with pytest.raises(gca.GcaError) as e:
            call()
        assert e.value.status == status
    assert not w.length.any()
