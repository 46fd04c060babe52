"""int8 numbers of the token window where entries are ties or next to one: an entry times 127 over its token's largest
magnitude is then off a half by the rounding of that factor at most.  It is the magnitude's reciprocal times 127,
each rounded to fp32, here as in the chunk cache, so both stores, and elementary fp32 operations, give the same numbers."""

import numpy as np
import pytest

from _helpers import ensure_built, host64

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


def _numbers(x):
    """By numpy, in fp32 (its operations round to nearest)."""
    x = host64(x).astype(np.float32)
    top = np.maximum(np.abs(x).max(axis=-1, keepdims=True), np.float32(2.0**-100))
    return np.rint(x * ((np.float32(1) / top) * np.float32(127)))


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("B,Hkv,C,window,T", [(7, 3, 64, 64, 1), (3, 2, 512, 300, 100), (2, 4, 2048, 512, 1900), (3, 2, 2048, 0, 700)])
def test_numbers_are_elementary_ones(dev, gca, dtype, B, Hkv, C, window, T):
    import torch
    w = gca.window(B, Hkv, C, window=window, dtype=dtype, format="int8", device=dev)
    g = torch.Generator(device=dev).manual_seed(T)
    k, v = (torch.randn(B, Hkv, T, 64, generator=g, device=dev) for _ in range(2))
    for x in (k, v):     # entries that are odd halves of 127ths of their token's largest, and those next to them
        at = torch.randint(0, 127, x.shape, generator=g, device=dev)
        top = x.abs().amax(dim=-1, keepdim=True).bfloat16().float()
        tie = (2 * at + 1) * top / 254
        x[:, :, ::2, 1:] = torch.where(at[:, :, ::2, 1:] % 3 == 0, tie[:, :, ::2, 1:], x[:, :, ::2, 1:])
        x[:, :, ::2, :1] = top[:, :, ::2]
    k, v = (x.to(w.elem) for x in (k, v))
    gca.window_append(w, k, v)
    rows = torch.arange(T, device=dev)
    assert np.array_equal(w.k[:, :, rows].cpu().numpy(), _numbers(k))
    got = w.v.transpose(-1, -2).reshape(B, Hkv, C, 64)[:, :, rows]
    assert np.array_equal(got.cpu().numpy(), _numbers(v))


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_both_stores_hold_the_same_numbers(dev, gca, dtype):
    """A chunk whose tokens have the same largest magnitude has the window's scales."""
    import torch
    B, Hkv = 16, 4
    w = gca.window(B, Hkv, 128, window=65, dtype=dtype, format="int8", device=dev)
    c = gca.cache(B, Hkv, 2, 1, D=64, dtype=dtype, format="int8", device=dev)
    g = torch.Generator(device=dev).manual_seed(1)
    k, v = (torch.randn(B, Hkv, 64, 64, generator=g, device=dev).to(w.elem) for _ in range(2))
    for x in (k, v):
        x.clamp_(-2.0, 2.0)
        x[..., 5] = torch.rand(B, Hkv, 1, generator=g, device=dev).to(x.dtype) + 2.0
    gca.window_append(w, k, v)
    gca.cache_store(c, k, v, None, torch.zeros(B, 1, dtype=torch.int32, device=dev))
    assert torch.equal(w.k[:, :, :64], c.k[:, :, 0])
    assert torch.equal(w.v[:, :, 0], c.v[:, :, 0])
