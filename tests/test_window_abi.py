"""The token window's and the verification's part of the C ABI on the host: struct layout, workspace
sizes, and calls that are refused before anything is launched (no call here reaches a kernel)."""

import ctypes
import math

import pytest

from _helpers import ensure_built


@pytest.fixture(scope="module")
def gca():
    ensure_built()
    from paper_2410_01651_amd import gca as g
    g.lib()
    return g


FAKE = 1 << 20   # aligned, never dereferenced
P = ctypes.c_void_p


def _window(gca, **kw):
    f = dict(B=2, H=8, Hkv=4, d=64, capacity=1024, window=512, attn_scale=0.125, off_by_one=0, dtype=gca.GCA_BF16,
             format=gca.GCA_E4M3, flags=0, k=FAKE, v=FAKE, k_scale=FAKE, v_scale=FAKE, length=FAKE, ticket=FAKE)
    f.update(kw)
    return gca.WindowStruct(**f)


def _append(gca, w, T=3, **kw):
    a = dict(k=FAKE, v=FAKE, lengths=FAKE)
    a.update(kw)
    return gca.lib().gca_window_append(ctypes.byref(w), a["k"], a["v"], a["lengths"], T, None)


def _attn(gca, w, T=3, **kw):
    a = dict(q=FAKE, parents=None, lengths=None, slopes=None, out=FAKE, lse=None, ws=FAKE, nbytes=1 << 30)
    a.update(kw)
    return gca.lib().gca_window_attn(ctypes.byref(w), a["q"], a["parents"], a["lengths"], a["slopes"], a["out"], a["lse"], T,
                                     a["ws"], a["nbytes"], None)


def _keep(gca, w, T=3, n=3, **kw):
    a = dict(path=FAKE, lengths=None)
    a.update(kw)
    return gca.lib().gca_window_keep(ctypes.byref(w), a["path"], n, a["lengths"], T, None)


def _verify(gca, B=2, T=5, V=1000, **kw):
    a = dict(p=FAKE, q=None, tokens=FAKE, parents=None, u=FAKE, lengths=None, path=FAKE, count=FAKE, next=FAKE, ws=FAKE,
             nbytes=1 << 30)
    a.update(kw)
    return gca.lib().gca_verify(B, T, V, a["p"], a["q"], a["tokens"], a["parents"], a["u"], a["lengths"], a["path"], a["count"],
                                a["next"], a["ws"], a["nbytes"], None)


CALLS = (_append, _attn, _keep)


def _msg(gca):
    return gca.lib().gca_last_error().decode()


def test_struct_layout(gca):
    S = gca.WindowStruct
    assert ctypes.sizeof(S) == 96 and S.capacity.offset == 16 and S.flags.offset == 44
    assert S.k.offset == 48 and S.ticket.offset == 88


@pytest.mark.parametrize("field,value,status", [
    ("B", 0, "INVALID"), ("H", 0, "INVALID"), ("Hkv", 0, "INVALID"), ("Hkv", 3, "INVALID"), ("d", 128, "UNSUPPORTED"),
    ("capacity", 0, "INVALID"), ("capacity", 100, "UNSUPPORTED"), ("capacity", (1 << 24) + 64, "UNSUPPORTED"),
    ("window", -1, "INVALID"), ("window", 1025, "INVALID"), ("dtype", 2, "INVALID"), ("format", 2, "INVALID"),
    ("format", -1, "INVALID"), ("off_by_one", 2, "INVALID"), ("flags", 1, "INVALID"), ("attn_scale", math.nan, "INVALID"),
    ("attn_scale", math.inf, "INVALID"), ("attn_scale", 1e-40, "UNSUPPORTED"), ("attn_scale", -(2.0**-65), "UNSUPPORTED"),
    ("B", 1 << 20, "UNSUPPORTED"),
])
def test_malformed_window_is_refused(gca, field, value, status):
    w = _window(gca, **{field: value})
    for call in CALLS:
        assert call(gca, w) == getattr(gca, "GCA_ERR_" + status), _msg(gca)
        assert _msg(gca)
    assert gca.lib().gca_window_workspace_size(ctypes.byref(w), 1) == 0


@pytest.mark.parametrize("call,names", [
    (_append, ("k", "v", "k_scale", "v_scale", "length", "ticket")), (_attn, ("k", "v", "k_scale", "v_scale", "length", "ticket")),
    (_keep, ("k", "v", "k_scale", "v_scale", "length", "ticket"))])
def test_missing_members_are_refused(gca, call, names):
    for name in names:
        assert call(gca, _window(gca, **{name: None})) == gca.GCA_ERR_INVALID
        assert name in _msg(gca)
        assert call(gca, _window(gca, **{name: FAKE + 2})) == gca.GCA_ERR_INVALID


@pytest.mark.parametrize("call,names", [
    (_append, ("k", "v")), (_attn, ("q", "out")), (_keep, ("path",)), (_verify, ("p", "tokens", "u", "path", "count", "next"))])
def test_missing_arguments_are_refused(gca, call, names):
    first = () if call is _verify else (_window(gca),)
    for name in names:
        for bad in (None, FAKE + 2):
            assert call(gca, *first, **{name: bad}) == gca.GCA_ERR_INVALID
            assert name in _msg(gca)


@pytest.mark.parametrize("call,names", [
    (_append, ("lengths",)), (_attn, ("parents", "lengths", "slopes", "lse")), (_keep, ("lengths",)),
    (_verify, ("q", "parents", "lengths"))])
def test_misaligned_optional_arguments_are_refused(gca, call, names):
    first = () if call is _verify else (_window(gca),)
    for name in names:
        assert call(gca, *first, **{name: FAKE + 1}) == gca.GCA_ERR_INVALID
        assert name in _msg(gca)


def test_counts_are_refused(gca):
    w = _window(gca)
    for call in CALLS:
        assert call(gca, w, T=0) == gca.GCA_ERR_INVALID
        assert call(gca, w, T=-5) == gca.GCA_ERR_INVALID
        assert call(gca, w, T=1 << 40) == gca.GCA_ERR_UNSUPPORTED
    # a ring's window has to outlast the new tokens
    assert _attn(gca, w, T=514) == gca.GCA_ERR_INVALID and "capacity" in _msg(gca)
    assert _keep(gca, w, T=1025) == gca.GCA_ERR_INVALID
    assert _keep(gca, w, T=514) == gca.GCA_ERR_INVALID and "capacity" in _msg(gca)
    assert _attn(gca, w, T=65, parents=FAKE) == gca.GCA_ERR_UNSUPPORTED
    assert _keep(gca, w, n=65) == gca.GCA_ERR_UNSUPPORTED
    assert _keep(gca, w, n=-1) == gca.GCA_ERR_INVALID
    for kw, status in ((dict(B=0), "INVALID"), (dict(T=0), "INVALID"), (dict(V=0), "INVALID"), (dict(T=65), "UNSUPPORTED"),
                       (dict(V=(1 << 19) + 1), "UNSUPPORTED"), (dict(B=1 << 40), "UNSUPPORTED")):
        assert _verify(gca, **kw) == getattr(gca, "GCA_ERR_" + status)
        assert gca.lib().gca_verify_workspace_size(*(dict(B=2, T=5, V=1000) | kw).values()) == 0


def test_workspace(gca):
    L = gca.lib()
    for H, Hkv, dtype in ((8, 8, 0), (8, 1, 1), (64, 2, 1), (64, 2, 0)):
        for capacity, window in ((64, 64), (1024, 100), (4096, 0), (1 << 24, 0), (8192, 4000)):
            for B in (1, 7, 100):
                w = _window(gca, B=B, H=H, Hkv=Hkv, dtype=dtype, capacity=capacity, window=window)
                last = 0
                for T in (1, 2, 3, 4, 5, 8, 16, 17, 31, 32, 33, 63, 64, 65, 100, 1000):
                    n = L.gca_window_workspace_size(ctypes.byref(w), T)
                    assert n >= last and n % 256 == 0 and n < 1 << 25
                    last = n
    big = _window(gca, capacity=1 << 20, window=0)
    need = L.gca_window_workspace_size(ctypes.byref(big), 1)
    assert need > 0
    assert _attn(gca, big, T=1, nbytes=need - 1) == gca.GCA_ERR_WORKSPACE
    assert _attn(gca, big, T=1, ws=None) == gca.GCA_ERR_WORKSPACE
    assert _attn(gca, big, T=1, ws=FAKE + 128) != gca.GCA_OK
    need = L.gca_verify_workspace_size(2, 5, 200000)
    assert need > 0 and need % 256 == 0
    assert _verify(gca, V=200000, nbytes=need - 1) == gca.GCA_ERR_WORKSPACE
    assert _verify(gca, V=200000, ws=None) == gca.GCA_ERR_WORKSPACE


def test_a_refused_size_leaves_the_error_as_it_was(gca):
    assert _append(gca, _window(gca, B=0)) != gca.GCA_OK
    before = _msg(gca)
    assert gca.lib().gca_window_workspace_size(None, 1) == 0 and gca.lib().gca_verify_workspace_size(0, 0, 0) == 0
    assert _msg(gca) == before


def test_binding_refuses_host_tensors(gca):
    import torch
    with pytest.raises(ValueError, match="device"):
        gca.window(1, 1, 64, device="cpu")
    with pytest.raises(ValueError, match="device"):
        gca.verify(torch.zeros(1, 1, 5), torch.zeros(1, 1, dtype=torch.int32), torch.zeros(1, 1))
    with pytest.raises(ValueError, match="no tensors"):
        gca.window(1, 1, 64, tensors=dict(x=torch.zeros(1)))
