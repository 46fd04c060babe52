"""Pins of the token window's oracle: closed forms, library routines, and the property that the
verification exists for, that accepted and drawn tokens are distributed as the target's own."""

import itertools

import numpy as np
import pytest

from oracle import window as ow


def _window(rng, B, Hkv, C):
    return dict(k=rng.integers(-9, 9, (B, Hkv, C, 64)).astype(float), v=rng.integers(-9, 9, (B, Hkv, C // 64, 64, 64)).astype(float),
                k_scale=rng.random((B, Hkv, C)) / 8, v_scale=rng.random((B, Hkv, C)), length=np.zeros(B, np.int64))


@pytest.mark.parametrize("window,off_by_one", [(0, False), (0, True), (40, False), (40, True)])
def test_chain_is_masked_softmax_attention(window, off_by_one):
    torch = pytest.importorskip("torch")
    rng = np.random.default_rng(window)
    B, H, Hkv, C, T = 2, 4, 2, 128, 9
    w = _window(rng, B, Hkv, C)
    length = np.array([T + 3, 100])
    q = rng.standard_normal((B, H, T, 64))
    slopes = np.array([0.5, 0.25, 0.0, 0.1])
    r = ow.attn(q, w["k"], w["v"], w["k_scale"], w["v_scale"], length, None, None, slopes, window, 0.125, off_by_one)
    for b, h in itertools.product(range(B), range(H)):
        j, L = h // 2, int(length[b])
        k = torch.from_numpy(w["k"][b, j] * w["k_scale"][b, j][:, None])[:L]
        v = torch.from_numpy(w["v"][b, j].transpose(0, 2, 1).reshape(C, 64) * w["v_scale"][b, j][:, None])[:L]
        i, p = torch.arange(L - T, L)[:, None], torch.arange(L)
        s = torch.from_numpy(q[b, h]) @ k.T / 8 + float(slopes[h]) * (p - i)
        s = s.masked_fill((p > i) | ((p <= i - window) if window else (p < 0)), -torch.inf)
        if off_by_one:
            s = torch.cat([s, torch.zeros(T, 1, dtype=s.dtype)], dim=1)
        assert np.allclose(r["lse"][b, h], torch.logsumexp(s, 1).numpy())
        assert np.allclose(r["out"][b, h], (torch.softmax(s, 1)[:, :L] @ v).numpy())


def test_tree_rows_equal_the_chains_of_their_paths():
    """Node i of a tree attends as the last token of a chain of its ancestors does."""
    rng = np.random.default_rng(3)
    H, C, T, L = 2, 128, 7, 50
    w = _window(rng, 1, H, C)
    parents = np.array([[-1, 0, 0, 1, 1, 2, 4]])
    q = rng.standard_normal((1, H, T, 64))
    slopes = np.array([0.3, 0.1])
    for window in (0, 20, 3):
        args = lambda x, qq, n, par: ow.attn(qq, x["k"], x["v"], x["k_scale"], x["v_scale"], np.array([L + n]), None, par, slopes,  # noqa: E731
                                             window, 0.125, False)
        tree = args(w, q, T, parents)
        for i in range(T):
            up, a = [i], i
            while parents[0, a] >= 0:
                a = parents[0, a]
                up.insert(0, a)
            x = {n: y.copy() for n, y in w.items()}
            x["length"][:] = L + T
            ow.keep(x, np.array([up]), None, T, window)
            assert x["length"][0] == L + len(up)
            one = args(x, np.ascontiguousarray(q[:, :, up]), len(up), None)
            assert np.allclose(one["out"][:, :, -1], tree["out"][:, :, i]) and np.allclose(one["lse"][:, :, -1], tree["lse"][:, :, i])


def test_append_wraps_and_keeps_the_last():
    w = _window(np.random.default_rng(0), 1, 1, 64)
    x = np.arange(1, 101, dtype=float)[None, None, :, None] * np.ones(64)
    ow.append(w, x, x, None, "e4m3", 64)
    assert w["length"][0] == 100
    for p in range(36, 100):   # token p is p + 1 throughout: a power of two times an e4m3 number, rounded
        got = w["k"][0, 0, p % 64] * w["k_scale"][0, 0, p % 64]
        assert (np.abs(got - (p + 1)) <= (p + 1) * 2.0**-4).all()
        assert (w["v"][0, 0, 0, :, p % 64] == w["k"][0, 0, p % 64]).all()


def test_keep_ends_where_a_token_was_not_kept():
    """C = 64 and 60 tokens before: tokens 4 and on of the new ones have no rows."""
    for path, m in (([0, 2, 3, 5], 3), ([0, 1, 2, 3, 5], 5), ([4], 0), ([0, 1, 2, 3, 4, 5], 6)):
        w = _window(np.random.default_rng(1), 1, 1, 64)
        w["length"][:] = 66
        old = w["k"].copy()
        ow.keep(w, np.array([path]), None, 6, 0)
        assert w["length"][0] == 60 + m
        for i in range(min(m, 4)):
            assert (w["k"][0, 0, 60 + i] == old[0, 0, 60 + path[i]]).all()


@pytest.mark.parametrize("children,drawn", [(1, True), (2, True), (3, True), (1, False), (2, False)])
def test_verified_tokens_follow_the_target(children, drawn):
    """The token behind the root, accepted or drawn, has probability p[0] whatever the draft's q: in n
    random runs its share is off by at most 5 standard deviations, 5 / (2 sqrt n)."""
    rng = np.random.default_rng(children)
    V, n, T = 4, 20000, 1 + children
    p0, q0 = (rng.dirichlet(np.ones(V)).astype(np.float32) for _ in range(2))
    tokens = rng.choice(V, (n, T), p=q0 / q0.astype(np.float64).sum()).astype(np.int32)
    p, q = (np.broadcast_to(x, (n, T, V)) for x in (p0, q0))
    parents = np.tile(np.array([-1] + [0] * children, np.int32), (n, 1))
    path, count, nxt = ow.verify(p, tokens, rng.random((n, T)).astype(np.float32), q if drawn else None, parents)
    first = np.where(count > 1, np.take_along_axis(tokens, np.maximum(path[:, 1:2], 0), 1)[:, 0], nxt)
    assert np.abs(np.bincount(first, minlength=V) / n - p0).max() <= 2.5 / np.sqrt(n)


def test_verify_closed_forms():
    V = 4
    eye = np.eye(V, dtype=np.float32)
    u = np.full((1, 4), 0.7, np.float32)
    # greedy: one-hot targets accept exactly the drafts that agree, and name the next token
    p = eye[[2, 1, 3, 0]][None]
    assert [x.tolist() for x in ow.verify(p, np.array([[0, 2, 1, 0]]), u)] == [[[0, 1, 2, -1]], [3], [3]]
    assert [x.tolist() for x in ow.verify(p, np.array([[0, 2, 1, 3]]), u)] == [[[0, 1, 2, 3]], [4], [0]]
    assert [x.tolist() for x in ow.verify(p, np.array([[0, 1, 1, 3]]), u)] == [[[0, -1, -1, -1]], [1], [2]]
    # nodes behind the sequence's own are not tested; no nodes, no token
    assert [x.tolist() for x in ow.verify(p, np.array([[0, 2, 1, 3]]), u, lengths=[2])] == [[[0, 1, -1, -1]], [2], [1]]
    assert [x.tolist() for x in ow.verify(p, np.array([[0, 2, 1, 3]]), u, lengths=[0])] == [[[-1] * 4], [0], [-1]]
    # the draw goes by partial sums, and by what rejection leaves
    half = np.array([[[0.5, 0.0, 0.25, 0.25]] * 2], np.float32)
    draw = lambda x, tok=3, q=None: ow.verify(half, np.array([[0, tok]]), np.array([[x, 0.99]], np.float32), q)[2][0]  # noqa: E731
    assert [draw(x) for x in (0.0, 0.66, 0.67, 0.99)] == [0, 0, 2, 2]
    assert [draw(x, tok=1) for x in (0.49, 0.5, 0.74, 0.75)] == [0, 2, 2, 3]
    q = np.array([[[0.25, 0.0, 0.0, 0.75]] * 2], np.float32)     # leaves 1/4, 0, 1/4, 0
    assert [draw(x, 3, q) for x in (0.49, 0.51)] == [0, 2]
    # nothing left: of p itself
    assert draw(0.9, 3, half * 0 + 1.0) == 3
    # the largest sum, 2^19 ones in whole multiples of 2^-44: 2^63
    ones = np.ones((1, 1, 1 << 19), np.float32)
    assert ow.verify(ones, np.array([[0]]), np.array([[0.75]], np.float32))[2].tolist() == [3 << 17]
