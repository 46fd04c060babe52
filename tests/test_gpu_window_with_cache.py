"""A layer's serving step with both halves of its attention: drafted tokens join the token window, attend to it and to
the retrieved chunks, are verified, and the accepted ones stay; a chunk that they complete, in the middle of a step's
path or at its end, is stored in the chunk cache, where the next steps retrieve it.

Every operator is compared with its oracle on the state that the device holds (tolerances: test_gpu_window.py,
test_gpu_cache.py).  Both stores hold the same tokens: a number is off by half a step, 2^-4 of its value or 2^-10
of its scale (e4m3), or 1/2 of its scale (int8), so a chunk's numbers and the window's differ by the two sums."""

import numpy as np
import pytest

import test_gpu_cache as tc
import test_gpu_window as tw
from _helpers import ensure_built, host64
from oracle import cache as oc
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


def _off(n, scale, fmt):
    """What numbers times their scale may be off by from what was stored."""
    return 0.5 * scale + 2.0**-20 if fmt == "int8" else np.maximum(2.0**-4 * np.abs(n) * scale, 2.0**-10 * scale) * 1.07


@pytest.mark.parametrize("dtype,fmt,window", [("bf16", "e4m3", 100), ("fp32", "int8", 70), ("bf16", "int8", 100)])
def test_steps(dev, gca, dtype, fmt, window):
    import torch
    rng = np.random.default_rng(window)
    B, H, Hkv, C, T, V, slots, topk, D = 3, 4, 2, 256, 14, 12, 3, 2, 64
    w = gca.window(B, H, C, window=window, Hkv=Hkv, dtype=dtype, format=fmt, device=dev)
    c = gca.cache(B, H, slots, topk, Hkv=Hkv, D=D, dtype=dtype, format=fmt, device=dev)
    g = torch.Generator(device=dev).manual_seed(7)
    rand = lambda *s: torch.randn(*s, generator=g, device=dev).to(tw._elem(dtype))  # noqa: E731
    up = lambda x: torch.from_numpy(x).to(dev)  # noqa: E731
    sl = torch.exp2(-torch.arange(1, H + 1, device=dev, dtype=torch.float32))
    text = [([], []) for _ in range(B)]      # the accepted tokens' keys and values [Hkv, 64]
    stored = np.zeros(B, np.int64)           # chunks that went to the cache
    idx, sel, fw = gca.cache_select(c, rand(B, 1, 1, D))
    inside = at_end = 0
    for step in range(64):
        k, v, q = rand(B, Hkv, T, 64), rand(B, Hkv, T, 64), rand(B, H, T, 64)
        p, qd, par, tok, u = tw._drafts(rng, B, T, V, "tree", False)
        p = p * 0.3 + 0.7 / V                # (paths of some length)
        tok[:, 1:] = np.take_along_axis(p.argmax(-1), np.maximum(par, 0), 1)[:, 1:]
        u *= 0.12
        par, tok = np.ascontiguousarray(par), np.ascontiguousarray(tok)
        gca.window_append(w, k, v)
        got = gca.window_attn(w, q, parents=up(par), slopes=sl)
        tw._check_attn(w, q, got, up(par), None, sl)
        out, lse, weights = gca.cache_xattn(c, q, idx, sel)
        tc._check_xattn(c, q, idx.cpu().numpy(), sel.cpu().numpy(), (out, lse, weights), T, 0)
        path, count, nxt = gca.verify(up(p.astype(np.float32)), up(tok), up(u), parents=up(par))
        want = ow.verify(p.astype(np.float32), tok, u, None, par)
        assert all(np.array_equal(a.cpu().numpy(), b) for a, b in zip((path, count, nxt), want))
        gca.window_keep(w, T, path)
        kept = want[0]
        full = np.zeros(B, np.int32)
        for b in range(B):
            m = int(want[1][b])
            for i in kept[b, :m]:
                text[b][0].append(k[b, :, i])
                text[b][1].append(v[b, :, i])
            n = len(text[b][0])
            full[b] = n // 64 > stored[b]
            inside += int(full[b] and n % 64 > 0)
            at_end += int(full[b] and n % 64 == 0)
        assert w.length.cpu().tolist() == [len(x[0]) for x in text]
        if not full.any():
            continue
        chunk = [torch.zeros(B, Hkv, 64, 64, dtype=tw._elem(dtype), device=dev) for _ in range(2)]
        for b in np.nonzero(full)[0]:
            for x, y in zip(chunk, text[b]):
                x[b] = torch.stack(y[64 * stored[b]:64 * stored[b] + 64], dim=1)
        at = gca.cache_evict(c, 1, idx, fw, decay=0.5, keep_last=1, want=up(full))
        gca.cache_store(c, *chunk, rand(B, 1, 1, D), at, lengths=up(64 * full))
        at = at.cpu().numpy()
        st, held = tw._state(w), dict(k=tc._values(c.k), v=tc._values(c.v), k_scale=host64(c.k_scale), v_scale=host64(c.v_scale))
        for b in np.nonzero(full)[0]:
            s, rows = int(at[b, 0]), np.arange(64 * stored[b], 64 * stored[b] + 64) % C
            assert 0 <= s < slots and int(c.tokens[b, s]) == 64
            for name in ("k", "v"):
                n1, s1 = held[name][b, :, s], held[name + "_scale"][b, :, s, None, None]
                n2, s2 = st[name][b], st[name + "_scale"][b][:, rows, None]
                if name == "v":
                    n1, n2 = n1.transpose(0, 2, 1), n2.transpose(0, 1, 3, 2).reshape(Hkv, C, 64)
                n2 = n2[:, rows]
                x = host64(chunk[name == "v"][b])
                assert (np.abs(n1 * s1 - x) <= _off(n1, s1, fmt)).all() and (np.abs(n2 * s2 - x) <= _off(n2, s2, fmt)).all(), (step, name)
            stored[b] += 1
        idx, sel, fw = gca.cache_select(c, rand(B, 1, 1, D))
        assert (idx.cpu().numpy() >= 0).sum(axis=(1, 2, 3)).tolist() == [min(int(n), slots, topk) for n in stored]
    assert inside > 0 and at_end > 0 and stored.max() > slots, (inside, at_end, stored)   # (an eviction too)
