"""What a row of the window attention does not see: tokens behind it, other branches of a tree, tokens before its
window.  A value's scale there may be any number.  Rows go in blocks of 16, 32 or 64, which round their
probabilities (and, of 64 rows, their values) relative to the largest value scale that a row of the block sees; a
token that none of them sees is to leave every bit of the block's results as it is.

Tolerances: those of test_gpu_window.py, with the largest value scale taken over what the rows of a block see
instead of over what any new token sees."""

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


def _star(T, first):
    """Nodes up to `first` are a chain, the others children of the root."""
    return [-1] + [i - 1 if i < first else 0 for i in range(1, T)]


# B, H, Hkv, C, window, T, parents, dtype, format, base, far (position of the token with the large scale), heads and
# rows of blocks that do not see it
UNSEEN = [
    (128, 8, 8, 256, 0, 128, None, "bf16", "e4m3", 32, 120, slice(None), slice(0, 64)),       # 64 rows: a later block's token
    (128, 8, 8, 256, 100, 128, None, "bf16", "e4m3", 1056, 1144, slice(None), slice(0, 64)),  # in a ring
    (1, 2, 2, 128, 0, 64, None, "bf16", "e4m3", 10, 50, slice(None), slice(0, 32)),           # 32 rows
    (1, 2, 2, 128, 60, 64, None, "bf16", "int8", 10, 50, slice(None), slice(0, 32)),
    (2, 2, 1, 128, 0, 64, None, "fp32", "e4m3", 10, 50, slice(None), slice(0, 32)),
    (2, 2, 1, 1024, 0, 64, None, "fp32", "int8", 900, 941, slice(None), slice(0, 32)),        # several waves; workgroups by lengths
    (1, 1, 1, 128, 0, 40, _star(40, 8), "bf16", "e4m3", 20, 25, slice(None), slice(32, 40)),  # a node of another branch
    (1, 1, 1, 128, 0, 40, _star(40, 8), "fp32", "int8", 20, 55, slice(None), slice(0, 32)),   # a later block's node
    (1, 4, 2, 128, 0, 20, _star(20, 8), "bf16", "int8", 20, 25, slice(1, None, 2), slice(12, 20)),  # a group's rows as one list
    (128, 16, 8, 128, 0, 40, _star(40, 8), "bf16", "e4m3", 20, 25, slice(1, None, 2), slice(24, 40)),  # of 64 rows
    (1, 1, 1, 128, 70, 40, _star(40, 40), "bf16", "e4m3", 110, 70, slice(None), slice(32, 40)),  # before the deep nodes' window
    (1, 1, 1, 128, 3, 40, _star(40, 40), "fp32", "e4m3", 20, 45, slice(None), slice(32, 40)),    # an ancestor too far up
]


@pytest.mark.parametrize("case", UNSEEN, ids=lambda c: "-".join(str(x) for x in (*c[:6], "tree" if c[6] else "chain", *c[7:11])))
def test_scales_that_a_block_does_not_see(dev, gca, case):
    import torch
    B, H, Hkv, C, window, T, parents, dtype, fmt, base, far, heads, rows = case
    w = gca.window(B, H, C, window=window, Hkv=Hkv, dtype=dtype, format=fmt, device=dev)
    g = tw._fill(w, 31, [base + T] * B)
    q = torch.randn(B, H, T, 64, generator=g, device=dev).to(tw._elem(dtype))
    sl = torch.full((H,), 0.01, device=dev)
    par = None if parents is None else torch.tensor([parents] * B, dtype=torch.int32, device=dev)
    run = lambda: [x[:, heads, rows].clone() for x in gca.window_attn(w, q, parents=par, slopes=sl)]  # noqa: E731
    out, lse = run()
    assert torch.isfinite(out).all() and torch.isfinite(lse).all()
    for scale in (2.0**60, 2.0**-60, float("nan")):
        w.v_scale[:, :, far % C] = scale
        out2, lse2 = run()
        assert torch.equal(lse, lse2), scale
        assert torch.equal(out, out2), (scale, float((out - out2).abs().max()))


def _seen_scale(w, T, n, parents, b):
    """[H, T]: the largest value scale that a row of row i's block sees, for sequence b, and the blocks' height."""
    s, st = w.struct, tw._state(w)
    G, C = s.H // s.Hkv, s.capacity
    many = s.B * s.Hkv * (G * (-(-T // 64)) if T >= 64 else -(-G * T // 64)) >= 2048
    height = 16 if G * T <= 16 else 64 if s.dtype == 1 and s.format == 0 and many else 32
    vis = ow.visible(int(st["length"][b]), n, C, s.window, parents)
    nu = np.zeros((s.H, T))
    for j in range(s.Hkv):
        if T >= height:
            blocks = [[(g, t) for t in range(t0, min(t0 + height, T))] for g in range(G) for t0 in range(0, T, height)]
        else:
            rows = [(g, t) for g in range(G) for t in range(n)]
            blocks = [rows[m:m + height] for m in range(0, len(rows), height)]
        for blk in blocks:
            seen = [vis[t][0] for g, t in blk if t < n]
            top = max((st["v_scale"][b, j, x].max() for x in seen if len(x)), default=0.0)
            for g, t in blk:
                nu[j * G + g, t] = top
    return nu, height


@pytest.mark.parametrize("B,Hkv,G,C,window,T,tree,dtype,fmt", [
    (2, 1, 2, 640, 0, 150, False, "bf16", "e4m3"), (2, 1, 2, 640, 100, 150, False, "fp32", "int8"),
    (128, 8, 1, 256, 0, 130, False, "bf16", "e4m3"), (128, 8, 1, 256, 70, 130, False, "bf16", "e4m3"),
    (3, 2, 3, 192, 0, 25, True, "bf16", "e4m3"), (3, 2, 3, 192, 30, 25, True, "fp32", "e4m3"),
    (3, 2, 2, 192, 9, 45, True, "bf16", "int8"), (128, 8, 2, 128, 0, 40, True, "bf16", "e4m3"),
    (3, 1, 3, 1024, 0, 40, False, "bf16", "int8"), (3, 1, 3, 1024, 0, 25, True, "fp32", "e4m3")])
def test_rounding_goes_by_what_a_block_sees(dev, gca, B, Hkv, G, C, window, T, tree, dtype, fmt):
    """Value scales from 2^-60 to 2^60 at random; and growing with the position, so that each token's is above
    those before it."""
    import torch
    w = gca.window(B, Hkv * G, C, window=window, Hkv=Hkv, dtype=dtype, format=fmt, device=dev)
    length = [min(C, T + 37 * b + 5) for b in range(B)]
    g = tw._fill(w, 17, length)
    q = torch.randn(B, Hkv * G, T, 64, generator=g, device=dev).to(tw._elem(dtype))
    par = torch.from_numpy(tw._tree(np.random.default_rng(T), B, T, "random")).to(dev) if tree else None
    counts = np.array([T if b % 2 == 0 else T - 3 for b in range(B)], np.int32)
    lengths = torch.from_numpy(counts).to(dev)
    for growing in (False, True):
        e = torch.randint(-60, 61, w.v_scale.shape, generator=g, device=dev).float()
        if growing:
            e = torch.linspace(-60, 60, C, device=dev).round().expand(w.v_scale.shape)
        w.v_scale.copy_(torch.exp2(e))
        out, lse = gca.window_attn(w, q, parents=par, lengths=lengths)
        st = tw._state(w)
        for b in (0, 1, B - 1):
            one = lambda x: None if x is None else host64(x[b:b + 1])  # noqa: E731
            pb = None if par is None else par[b:b + 1].cpu().numpy()
            ref = ow.attn(one(q), *(st[x][b:b + 1] for x in ("k", "v", "k_scale", "v_scale", "length")), counts[b:b + 1], pb, None,
                          window, 0.125, False)
            nu, height = _seen_scale(w, T, int(counts[b]), None if pb is None else pb[0], b)
            bf16, U = dtype == "bf16", tw.U
            rel = 4 * 66 * U * ref["dot"] + 8 * U * ref["dot"] + (2 * ref["seen"] + 8 * (ref["seen"] / 64 + 2) + 64) * U
            bound = (rel[..., None] + (2.0**-11 if bf16 else 2.0**-22)) * ref["mag"] + (2.0**-8 if bf16 else U) * np.abs(ref["out"])
            # sum |number|, from the oracle's term for the largest scale that any row sees
            num = np.abs(st["v"][b]).sum(axis=(1, 3))        # [Hkv, 64], of all rows: at least what a row sees
            bound += 2.0**-39 * nu[None, :, :, None] * np.repeat(num, G, axis=0)[None, :, None, :]
            if height == 64:
                bound += 2.0**-30 * nu[None, :, :, None]
            err = np.abs(one(out) - ref["out"])
            assert (err <= bound * (1 + 2.0**-7) + 1e-30).all(), (b, growing, float((err / (bound + 1e-300)).max()))
            f = np.isfinite(ref["lse"])
            assert np.array_equal(f, np.isfinite(one(lse)))
            assert (np.abs(one(lse)[f] - ref["lse"][f]) <= rel[f] + 16 * U * (1 + np.abs(ref["lse"][f]))).all()
