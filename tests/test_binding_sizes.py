"""Sizes that do not fit the C structs are refused by the binding (ctypes takes them modulo a power of two)."""

import pytest

from _helpers import ensure_built


@pytest.fixture(scope="module")
def gca():
    ensure_built()
    from paper_2410_01651_amd import gca as g
    return g


@pytest.mark.parametrize("field,value", [
    ("window", (1 << 32) + 100), ("window", 1 << 31), ("window", -(1 << 31) - 1), ("B", (1 << 32) + 2), ("H", (1 << 32) + 4), ("Hkv", (1 << 32) + 2),
    ("capacity", (1 << 64) + 128)])
def test_window(gca, field, value):
    sizes = dict(B=2, H=4, Hkv=2, capacity=128, window=100)
    sizes[field] = value
    with pytest.raises(ValueError, match=rf"{field} = {value} does not fit"):
        gca.window(**sizes)


@pytest.mark.parametrize("field,value", [("topk", (1 << 32) + 4), ("B", (1 << 32) + 2), ("Hr", (1 << 32) + 1), ("D", (1 << 32) + 64),
                                         ("capacity", (1 << 64) + 128)])
def test_cache(gca, field, value):
    sizes = dict(B=2, H=4, Hkv=2, capacity=128, topk=4, Hr=1, D=64)
    sizes[field] = value
    with pytest.raises(ValueError, match=rf"{field} = {value} does not fit"):
        gca.cache(**sizes)


@pytest.mark.parametrize("field,value", [("topk", (1 << 32) + 4), ("B", (1 << 32) + 2), ("n_chunks", (1 << 64) + 8), ("S", (1 << 32) + 64)])
def test_problem(gca, field, value):
    sizes = dict(B=2, H=4, n_chunks=8, topk=4)
    sizes[field] = value
    with pytest.raises(ValueError, match=rf"{field} = {value} does not fit"):
        gca.problem(**sizes)


def test_seeds_are_taken_modulo_64_bits(gca):
    assert gca.problem(2, 4, 8, 4, gumbel_seed=-1).gumbel_seed == (1 << 64) - 1


def test_tokens_kept(gca):
    """Refused before the window or the path is looked at for anything but its shape."""
    torch = pytest.importorskip("torch")
    for T in (1 << 63, (1 << 64) + 3, -(1 << 64) + 3):
        with pytest.raises(ValueError, match="does not fit"):
            gca.window_keep(type("W", (), dict(torch=torch, dims=(2, 4, 2)))(), T, torch.zeros(2, 3, dtype=torch.int32))
