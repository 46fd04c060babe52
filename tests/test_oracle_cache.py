"""Pins of the chunk cache's oracle: every e4m3 code, rounding by hand, agreement with the
uncached oracle where the cache holds its chunks exactly, and eviction by brute force."""

import itertools

import numpy as np
import pytest

import _helpers  # noqa: F401
from oracle import cache as oc, gca as og


def test_e4m3_codes_round_to_themselves_and_halves_to_even():
    v = oc.e4m3_values()
    fin = v[np.isfinite(v)]
    assert fin.max() == 448.0 and np.sum(np.isnan(v)) == 2 and fin[fin > 0].min() == 2.0**-9
    np.testing.assert_array_equal(oc.e4m3_round(fin), fin)
    pos = np.sort(np.unique(fin[fin >= 0]))
    mid = (pos[:-1] + pos[1:]) / 2
    codes = np.arange(len(pos))            # consecutive codes are consecutive values
    even = np.where(codes[:-1] % 2 == 0, pos[:-1], pos[1:])
    np.testing.assert_array_equal(oc.e4m3_round(mid), even)
    np.testing.assert_array_equal(oc.e4m3_round(np.nextafter(mid, 0)), pos[:-1])
    np.testing.assert_array_equal(oc.e4m3_round(np.nextafter(mid, 999)), pos[1:])


@pytest.mark.parametrize("top,scale", [(448.0, 1.0), (448.25, 2.0), (1.75, 2.0**-8), (1.0, 2.0**-8), (1.76, 2.0**-7),
                                       (0.0, 2.0**-126), (2.0**-130, 2.0**-126), (3.0e38, 2.0**120)])
def test_e4m3_scale(top, scale):
    x = np.zeros((64, 64))
    x[3, 5] = -top
    n, s = oc.quantise(x, "e4m3")
    assert s == scale and abs(n).max() <= 448.0


def test_int8_numbers():
    x = np.zeros((64, 64))
    x[0, :4] = 127.0, 2.5, -3.5, np.inf
    n, s = oc.quantise(x, "int8")
    assert s == 1.0 and n[0, :4].tolist() == [127, 2, -4, 127]
    x[1, 0] = np.nan
    assert np.isnan(oc.quantise(x, "int8")[1])


@pytest.mark.parametrize("off_by_one", [False, True])
def test_attention_agrees_with_the_uncached_oracle(off_by_one):
    """Integer keys and values are held exactly: CAUSAL attention over the cache is the oracle's."""
    rng = np.random.default_rng(5)
    B, H, nC, k = 1, 2, 6, 3
    q = rng.standard_normal((B, H, nC * 64, 64))
    kk, vv = (rng.integers(-127, 128, (B, H, nC * 64, 64)).astype(np.float64) / 64 for _ in range(2))
    lq, lk = rng.standard_normal((2, B, 1, nC, 64))
    pp = dict(S=64, topk=k, score_scale=0.125, attn_scale=0.125, mode="causal", off_by_one=off_by_one, Sq=64)
    ref = og.forward(pp, lq, lk, q, kk, vv)
    tiles = lambda x: 64 * x.reshape(B, H, nC, 64, 64)  # noqa: E731
    r = oc.xattn(q, ref["idx"], ref["sel"], tiles(kk), tiles(vv).swapaxes(-1, -2), np.full((B, H, nC), 1 / 64),
                 np.full((B, H, nC), 1 / 64), np.full((B, nC), 64), 0.125, 64, lag=1, off_by_one=off_by_one)
    np.testing.assert_allclose(r["out"], ref["out"], atol=1e-12)
    np.testing.assert_allclose(r["w"], ref["w"], atol=1e-14)
    f = np.isfinite(ref["lse"])
    assert np.array_equal(f, np.isfinite(r["lse"]))
    np.testing.assert_allclose(r["lse"][f], ref["lse"][f], atol=1e-12)


def test_eviction_by_brute_force():
    """The slots taken are the only set whose members all rank before the others."""
    rng = np.random.default_rng(1)
    for _ in range(50):
        C, n = int(rng.integers(1, 8)), int(rng.integers(0, 5))
        n = min(n, C)
        tokens = rng.integers(0, 3, (1, C))
        mass = np.where(tokens > 0, rng.integers(0, 3, (1, C)), 0).astype(np.float32)
        number = rng.permutation(C)[None]
        t, m, num, nxt, slots = oc.evict(tokens, mass, number, np.array([C]), n, keep_first=1, keep_last=2)
        may = [j for j in range(C) if tokens[0, j] == 0 or 1 <= number[0, j] < C - 2]
        order = lambda j: (tokens[0, j] > 0, mass[0, j], j)  # noqa: E731
        want = min(n, len(may))
        sets = [s for s in itertools.combinations(may, want)
                if all(order(a) < order(b) for a in s for b in may if b not in s)]
        assert len(sets) == 1 and slots[0, :want].tolist() == list(sets[0]) and (slots[0, want:] == -1).all()
        assert nxt[0] == C + n and (t[0, list(sets[0])] == 0).all()
        assert num[0, list(sets[0])].tolist() == list(range(C, C + want))
