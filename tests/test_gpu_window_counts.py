"""The window attention where workgroups are dealt out by the sequences' lengths (no window's end, 2 to 64 sequences,
1,024 rows and more) with counts of tokens, and queries that hold NaN or infinities.  Tolerances: those of
test_gpu_window.py."""

import numpy as np
import pytest

import test_gpu_window as tw
from _helpers import ensure_built

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


@pytest.mark.parametrize("B,Hkv,G,C,T,tree,dtype,fmt", [
    (2, 1, 2, 4096, 1, False, "bf16", "e4m3"),
    (5, 2, 4, 4096, 3, False, "bf16", "int8"),       # rows of all heads in one block
    (3, 3, 2, 2048, 20, True, "fp32", "e4m3"),       # a group's rows as one list of several blocks
    (3, 1, 8, 1024, 9, True, "bf16", "e4m3"),
    (64, 4, 1, 1024, 9, True, "bf16", "e4m3"),       # a sequence for every lane
    (33, 1, 8, 1088, 5, False, "fp32", "int8"),
    (9, 2, 16, 1024, 40, True, "bf16", "e4m3"),      # head by head, two blocks each
    (2, 1, 4, 8192, 64, True, "bf16", "int8"),
    (4, 2, 1, 8192, 70, False, "bf16", "e4m3"),
    (3, 2, 3, 1024, 33, False, "fp32", "e4m3"),
])
def test_counts_where_workgroups_go_by_lengths(dev, gca, B, Hkv, G, C, T, tree, dtype, fmt):
    import torch
    rng = np.random.default_rng(B * C + T)
    H = Hkv * G
    length = rng.integers(T, C + 1, B)
    length[0], length[B // 2] = C, T
    w = gca.window(B, H, C, Hkv=Hkv, dtype=dtype, format=fmt, device=dev)
    g = tw._fill(w, 23, [int(x) for x in length])
    q = torch.randn(B, H, T, 64, generator=g, device=dev).to(tw._elem(dtype))
    par = torch.from_numpy(tw._tree(rng, B, T, "random")).to(dev) if tree else None
    sl = torch.rand(H, generator=g, device=dev) * 0.05
    ws = gca.window_workspace(w, T)[0].fill_(255)
    some = rng.integers(0, T + 1, B)
    some[B // 2] = 0
    last = np.zeros(B)
    last[-1] = 1
    for n in (some, last, np.minimum(some, 1), rng.integers(-2, T + 3, B)):
        lengths = torch.from_numpy(n.astype(np.int32)).to(dev)
        out = torch.full_like(q, float("nan"))
        lse = torch.full((B, H, T), float("nan"), device=dev)
        got = gca.window_attn(w, q, parents=par, lengths=lengths, slopes=sl, out=out, lse=lse, ws=ws)
        tw._check_attn(w, q, got, par, lengths, sl)
    assert not w.ticket.any()


@pytest.mark.parametrize("B,Hkv,G,C,window,T,tree,dtype,fmt", [
    (2, 2, 1, 192, 100, 1, False, "bf16", "e4m3"), (2, 2, 4, 192, 0, 9, True, "bf16", "int8"), (2, 1, 1, 192, 70, 40, False, "fp32", "e4m3"),
    (3, 1, 2, 4096, 0, 5, True, "bf16", "e4m3"), (3, 1, 2, 4096, 0, 5, False, "fp32", "int8"), (128, 8, 1, 192, 60, 128, False, "bf16", "e4m3")])
def test_queries_with_nan_and_infinities(dev, gca, B, Hkv, G, C, window, T, tree, dtype, fmt):
    """A row with a NaN or an infinity in its query comes out as NaN, or as one that sees nothing where all its
    scores are -inf; no other row's bits change."""
    import torch
    inf, nan = float("inf"), float("nan")
    H = Hkv * G
    for obo in (False, True):
        w = gca.window(B, H, C, window=window, Hkv=Hkv, dtype=dtype, format=fmt, off_by_one=obo, device=dev)
        g = tw._fill(w, 29, [C - 7] * B)
        # column 3 of all keys is above zero: an infinity there makes all of a row's scores +inf or -inf
        k = w.k.view(torch.int8)
        k[..., 3] = (k[..., 3] & 0x7F).clamp(1, 0x7E)
        q = torch.randn(B, H, T, 64, generator=g, device=dev).to(tw._elem(dtype))
        par = torch.from_numpy(tw._tree(np.random.default_rng(3), B, T, "random")).to(dev) if tree else None
        out, lse = gca.window_attn(w, q, parents=par)
        assert torch.isfinite(out).all()
        b, h, t = B - 1, H - 1, T // 2
        for x in (nan, inf, -inf):
            bad = q.clone()
            bad[b, h, t, 3] = x
            out2, lse2 = gca.window_attn(w, bad, parents=par)
            row, row_lse = out2[b, h, t].clone(), float(lse2[b, h, t])
            if x == -inf and dtype == "bf16":     # (fp32 queries come in terms whose later ones are inf - inf)
                assert (row == 0).all() and row_lse == -inf
            else:
                assert torch.isnan(row).all() and np.isnan(row_lse), x
            out2[b, h, t], lse2[b, h, t] = out[b, h, t], lse[b, h, t]
            assert torch.equal(out, out2) and torch.equal(lse, lse2), x
