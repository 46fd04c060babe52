"""The chunk cache's part of the C ABI on the host: struct layout, workspace sizes, and calls
that are refused before anything is launched (no call here reaches a kernel)."""

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


def _cache(gca, **kw):
    f = dict(B=2, H=8, Hkv=4, Hr=1, d=64, S=64, capacity=100, topk=8, D=256, score_scale=0.0625, attn_scale=0.125,
             off_by_one=0, dtype=gca.GCA_BF16, format=gca.GCA_E4M3, flags=0, k=FAKE, v=FAKE, k_scale=FAKE, v_scale=FAKE,
             lmk=FAKE, tokens=FAKE, mass=FAKE, number=FAKE, next=FAKE)
    f.update(kw)
    return gca.CacheStruct(**f)


def _store(gca, c, n=3, **kw):
    a = dict(k=FAKE, v=FAKE, lmk=FAKE, slots=FAKE, lengths=FAKE)
    a.update(kw)
    L = gca.lib()
    return L.gca_cache_store(ctypes.byref(c), a["k"], a["v"], a["lmk"], a["slots"], a["lengths"], n, None)


def _select(gca, c, **kw):
    a = dict(lmk_q=FAKE, idx=FAKE, sel=FAKE, w=None, ws=FAKE, nbytes=1 << 24)
    a.update(kw)
    return gca.lib().gca_cache_select(ctypes.byref(c), a["lmk_q"], a["idx"], a["sel"], a["w"], a["ws"], a["nbytes"], None)


def _xattn(gca, c, nQ=1, rows=1, lag=0, **kw):
    a = dict(q=FAKE, idx=FAKE, sel=FAKE, out=FAKE, lse=None, w=None)
    a.update(kw)
    return gca.lib().gca_cache_xattn(ctypes.byref(c), a["q"], a["idx"], a["sel"], a["out"], a["lse"], a["w"], nQ, rows,
                                     lag, None)


def _evict(gca, c, n=3, nQ=1, decay=1.0, keep_first=0, keep_last=0, **kw):
    a = dict(idx=None, w=None, want=None, slots=FAKE, ws=FAKE, nbytes=1 << 24)
    a.update(kw)
    return gca.lib().gca_cache_evict(ctypes.byref(c), a["idx"], a["w"], nQ, decay, keep_first, keep_last, a["want"],
                                     a["slots"], n, a["ws"], a["nbytes"], None)


CALLS = (_store, _select, _xattn, _evict)


def _msg(gca):
    return gca.lib().gca_last_error().decode()


def test_struct_layout(gca):
    S = gca.CacheStruct
    assert ctypes.sizeof(S) == 136 and S.capacity.offset == 24 and S.flags.offset == 60
    assert S.k.offset == 64 and S.next.offset == 128


@pytest.mark.parametrize("field,value,status", [
    ("B", 0, "INVALID"), ("H", 0, "INVALID"), ("Hkv", 0, "INVALID"), ("Hkv", 3, "INVALID"), ("Hr", 2, "INVALID"),
    ("Hr", 8, "INVALID"), ("d", 128, "UNSUPPORTED"), ("S", 32, "UNSUPPORTED"), ("capacity", 0, "INVALID"),
    ("capacity", 262145, "UNSUPPORTED"), ("topk", 0, "INVALID"), ("topk", 33, "UNSUPPORTED"), ("D", 0, "INVALID"),
    ("D", 96, "UNSUPPORTED"), ("D", 8256, "UNSUPPORTED"), ("dtype", 2, "INVALID"), ("format", 2, "INVALID"),
    ("format", -1, "INVALID"), ("off_by_one", 2, "INVALID"), ("flags", 1, "INVALID"), ("attn_scale", math.nan, "INVALID"),
    ("score_scale", math.inf, "INVALID"), ("B", 1 << 20, "UNSUPPORTED"),
])
def test_malformed_cache_is_refused(gca, field, value, status):
    c = _cache(gca, **{field: value})
    for call in CALLS:
        assert call(gca, c) == getattr(gca, "GCA_ERR_" + status), _msg(gca)
        assert _msg(gca)
    for op in (gca.CACHE_SELECT, gca.CACHE_EVICT):
        assert gca.lib().gca_cache_workspace_size(ctypes.byref(c), op, 1) == 0


@pytest.mark.parametrize("call,names", [
    (_store, ("k", "v", "k_scale", "v_scale", "lmk", "tokens")), (_select, ("lmk", "tokens")),
    (_xattn, ("k", "v", "k_scale", "v_scale", "tokens")), (_evict, ("tokens", "mass", "number", "next"))])
def test_missing_or_misaligned_members(gca, call, names):
    for name in names:
        assert call(gca, _cache(gca, **{name: None})) == gca.GCA_ERR_INVALID and "cache " + name in _msg(gca)
        assert call(gca, _cache(gca, **{name: FAKE + 2})) == gca.GCA_ERR_INVALID and "aligned" in _msg(gca)


@pytest.mark.parametrize("call,names", [(_store, ("k", "v", "slots")), (_select, ("lmk_q", "idx", "sel")),
                                        (_xattn, ("q", "idx", "sel", "out")), (_evict, ("slots",))])
def test_missing_or_misaligned_arguments(gca, call, names):
    for name in names:
        assert call(gca, _cache(gca), **{name: None}) == gca.GCA_ERR_INVALID and name in _msg(gca)
        assert call(gca, _cache(gca), **{name: FAKE + 2}) == gca.GCA_ERR_INVALID and "aligned" in _msg(gca)


def test_ranges(gca):
    c = _cache(gca)
    assert _store(gca, c, n=0) == gca.GCA_ERR_INVALID
    assert _store(gca, c, n=1 << 40) == gca.GCA_ERR_UNSUPPORTED
    for nQ, rows in ((0, 1), (1, 0), (-1, 5)):
        assert _xattn(gca, c, nQ=nQ, rows=rows) == gca.GCA_ERR_INVALID
    for nQ, rows in ((1 << 40, 1), (1, 1 << 40), (1 << 25, 1 << 25), (1 << 62, 1 << 62)):
        assert _xattn(gca, c, nQ=nQ, rows=rows) == gca.GCA_ERR_UNSUPPORTED
    for lag in (-1, 2):
        assert _xattn(gca, c, lag=lag) == gca.GCA_ERR_INVALID
    for kw in (dict(n=-1), dict(n=101), dict(decay=-0.5), dict(decay=1.5), dict(decay=math.nan), dict(keep_first=-1),
               dict(keep_last=-1), dict(idx=FAKE), dict(w=FAKE), dict(idx=FAKE, w=FAKE, nQ=0)):
        assert _evict(gca, c, **kw) == gca.GCA_ERR_INVALID, kw
    assert _evict(gca, c, idx=FAKE, w=FAKE, nQ=1 << 40) == gca.GCA_ERR_UNSUPPORTED


def test_workspaces(gca):
    L = gca.lib()
    size = lambda c, op, n=0: L.gca_cache_workspace_size(ctypes.byref(c), op, n)  # noqa: E731
    c = _cache(gca)
    need = size(c, gca.CACHE_SELECT)
    assert need > 0
    assert _select(gca, c, ws=None, nbytes=0) == gca.GCA_ERR_WORKSPACE
    assert _select(gca, c, nbytes=need - 1) == gca.GCA_ERR_WORKSPACE
    assert _select(gca, c, ws=FAKE + 16, nbytes=need) == gca.GCA_ERR_WORKSPACE
    assert size(c, gca.CACHE_EVICT, 3) == 0 and size(c, 7, 1) == 0 and size(c, gca.OP_FORWARD, 1) == 0
    big = _cache(gca, capacity=100000)
    last = 0
    for n in (1, 2, 100, 8191, 8192, 8193, 100000):
        s = size(big, gca.CACHE_EVICT, n)
        assert s >= last and s > 0
        last = s
    assert size(big, gca.CACHE_EVICT, 0) == size(big, gca.CACHE_EVICT, 100001) == 0
    assert _evict(gca, big, n=5, nbytes=size(big, gca.CACHE_EVICT, 5) - 1) == gca.GCA_ERR_WORKSPACE
    assert L.gca_cache_workspace_size(None, gca.CACHE_SELECT, 0) == 0


def test_workspace_query_keeps_the_last_error(gca):
    c = _cache(gca, topk=0)
    assert _select(gca, c) == gca.GCA_ERR_INVALID
    before = _msg(gca)
    assert gca.lib().gca_cache_workspace_size(ctypes.byref(_cache(gca, B=0)), gca.CACHE_SELECT, 0) == 0
    assert _msg(gca) == before and "topk" in before


def test_binding_refuses_host_caches(gca):
    torch = pytest.importorskip("torch")
    with pytest.raises(ValueError, match="device memory"):
        gca.cache(1, 2, 8, 2, device="cpu")
    with pytest.raises(ValueError, match="no tensors named"):
        gca.cache(1, 2, 8, 2, tensors={"keys": torch.zeros(1)})
    with pytest.raises(ValueError):
        gca.cache(1, 2, 8, 2, tensors={"mass": torch.zeros(1, 8)})   # a host tensor
    with pytest.raises(KeyError):
        gca.cache(1, 2, 8, 2, format="e5m2")
