"""Python binding of libgca (ctypes; argument marshalling only).

Every function here forwards to the C entry point of the same name in
``include/gca.h``: it checks that the tensors are contiguous device tensors of
the expected dtype, allocates the outputs (and workspace) with torch, and passes
raw device pointers plus torch's current HIP stream.  All arithmetic runs in the
library's HIP kernels; nothing here computes.  A missing library raises.
"""

import ctypes
import math
import os
from dataclasses import dataclass

LIB_PATH = os.path.join(os.path.dirname(os.path.abspath(__file__)), "libgca.so")

EXPORTS = (
    "gca_chunk_scores",
    "gca_topk",
    "gca_grouped_xattn_fwd",
    "gca_grouped_xattn_bwd",
    "gca_forward",
    "gca_forward_noalloc",
    "gca_cache_store",
    "gca_cache_select",
    "gca_cache_xattn",
    "gca_cache_evict",
    "gca_cache_workspace_size",
    "gca_workspace_size",
    "gca_status_string",
    "gca_last_error",
    "gca_profile_arm",
    "gca_profile_count",
    "gca_profile_name",
)

GCA_OK, GCA_ERR_INVALID, GCA_ERR_UNSUPPORTED, GCA_ERR_WORKSPACE, GCA_ERR_HIP = range(5)
GCA_FP32, GCA_BF16 = 0, 1
GCA_CAUSAL, GCA_DECODE = 0, 1
FLAG_FUSED_TOPK, FLAG_MATERIALIZE, FLAG_GUMBEL, FLAG_HOST_KV, FLAG_LMK_ROW = 1, 2, 4, 8, 16
OP_FORWARD, OP_BACKWARD = 0, 1
GCA_E4M3, GCA_INT8 = 0, 1
CACHE_SELECT, CACHE_EVICT = 2, 3
NOALLOC_SCRATCH_BYTES = 16 << 20


class Problem(ctypes.Structure):
    """Mirror of ``gca_problem``."""

    _fields_ = [
        ("B", ctypes.c_int32),
        ("H", ctypes.c_int32),
        ("d", ctypes.c_int32),
        ("S", ctypes.c_int32),
        ("n_chunks", ctypes.c_int64),
        ("topk", ctypes.c_int32),
        ("Hr", ctypes.c_int32),
        ("D", ctypes.c_int32),
        ("score_scale", ctypes.c_float),
        ("attn_scale", ctypes.c_float),
        ("off_by_one", ctypes.c_int32),
        ("dtype", ctypes.c_int32),
        ("mode", ctypes.c_int32),
        ("flags", ctypes.c_uint32),
        ("gumbel_seed", ctypes.c_uint64),
    ]

    @property
    def n_query_chunks(self) -> int:
        return self.n_chunks if self.mode == GCA_CAUSAL else 1

    @property
    def query_rows(self) -> int:
        """Query rows per chunk: S, or S + 1 with the LMK row (GCA_FLAG_LMK_ROW)."""
        return self.S + 1 if self.flags & FLAG_LMK_ROW else self.S


class CacheStruct(ctypes.Structure):
    """Mirror of ``gca_cache``."""

    _fields_ = [
        ("B", ctypes.c_int32),
        ("H", ctypes.c_int32),
        ("Hkv", ctypes.c_int32),
        ("Hr", ctypes.c_int32),
        ("d", ctypes.c_int32),
        ("S", ctypes.c_int32),
        ("capacity", ctypes.c_int64),
        ("topk", ctypes.c_int32),
        ("D", ctypes.c_int32),
        ("score_scale", ctypes.c_float),
        ("attn_scale", ctypes.c_float),
        ("off_by_one", ctypes.c_int32),
        ("dtype", ctypes.c_int32),
        ("format", ctypes.c_int32),
        ("flags", ctypes.c_uint32),
        ("k", ctypes.c_void_p),
        ("v", ctypes.c_void_p),
        ("k_scale", ctypes.c_void_p),
        ("v_scale", ctypes.c_void_p),
        ("lmk", ctypes.c_void_p),
        ("tokens", ctypes.c_void_p),
        ("mass", ctypes.c_void_p),
        ("number", ctypes.c_void_p),
        ("next", ctypes.c_void_p),
    ]


class GcaError(RuntimeError):
    def __init__(self, status: int, message: str):
        super().__init__(message)
        self.status = status


_lib = None


def lib():
    """The loaded libgca (raises if it has not been built)."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise RuntimeError(f"libgca is not built ({LIB_PATH} missing); run "
                               "`python -m paper_2410_01651_amd.build`")
        L = ctypes.CDLL(LIB_PATH)
        vp, P = ctypes.c_void_p, ctypes.POINTER(Problem)
        C, i64 = ctypes.POINTER(CacheStruct), ctypes.c_int64
        sig = {
            "gca_chunk_scores": [P, vp, vp, vp, vp],
            "gca_topk": [P, vp, vp, vp, vp],
            "gca_grouped_xattn_fwd": [P, vp, vp, vp, vp, vp, vp, vp, vp, vp],
            "gca_grouped_xattn_bwd": [P, vp, vp, vp, vp, vp, vp, vp, vp, vp, vp, vp, vp, vp, vp, vp,
                                      vp, ctypes.c_size_t, vp],
            "gca_forward": [P, vp, vp, vp, vp, vp, vp, vp, vp, vp, vp, vp, ctypes.c_size_t, vp],
            "gca_forward_noalloc": [P, vp, vp, vp, vp, vp, vp, vp, vp, vp, vp, vp],
            "gca_cache_store": [C, vp, vp, vp, vp, vp, i64, vp],
            "gca_cache_select": [C, vp, vp, vp, vp, vp, ctypes.c_size_t, vp],
            "gca_cache_xattn": [C, vp, vp, vp, vp, vp, vp, i64, i64, ctypes.c_int32, vp],
            "gca_cache_evict": [C, vp, vp, i64, ctypes.c_float, ctypes.c_int32, ctypes.c_int32, vp, vp, i64, vp,
                                ctypes.c_size_t, vp],
        }
        for name, args in sig.items():
            fn = getattr(L, name)
            fn.argtypes = args
            fn.restype = ctypes.c_int
        L.gca_cache_workspace_size.argtypes = [C, ctypes.c_int, i64]
        L.gca_cache_workspace_size.restype = ctypes.c_size_t
        L.gca_workspace_size.argtypes = [P, ctypes.c_int]
        L.gca_workspace_size.restype = ctypes.c_size_t
        L.gca_status_string.argtypes = [ctypes.c_int]
        L.gca_status_string.restype = ctypes.c_char_p
        L.gca_last_error.argtypes = []
        L.gca_last_error.restype = ctypes.c_char_p
        L.gca_profile_arm.argtypes = [ctypes.c_void_p, ctypes.c_int]
        L.gca_profile_arm.restype = None
        L.gca_profile_count.argtypes = []
        L.gca_profile_count.restype = ctypes.c_int
        L.gca_profile_name.argtypes = [ctypes.c_int]
        L.gca_profile_name.restype = ctypes.c_char_p
        _lib = L
    return _lib


def _check(status: int) -> None:
    if status != GCA_OK:
        L = lib()
        raise GcaError(status, f"{L.gca_status_string(status).decode()}: {L.gca_last_error().decode()}")


def problem(B, H, n_chunks, topk, D=None, Hr=1, d=64, S=64, score_scale=None, attn_scale=None,
            off_by_one=False, dtype="bf16", mode="causal", flags=0, gumbel_seed=None,
            lmk_row=False) -> Problem:
    """Build a ``gca_problem``; D defaults to H*d, scales to 1/sqrt(D) and 1/sqrt(d).
    A ``gumbel_seed`` turns on Gumbel top-k selection (GCA_FLAG_GUMBEL);
    ``lmk_row`` gives every query chunk S + 1 rows (GCA_FLAG_LMK_ROW)."""
    D = H * d if D is None else D
    if gumbel_seed is not None:
        flags |= FLAG_GUMBEL
    if lmk_row:
        flags |= FLAG_LMK_ROW
    return Problem(
        B=B, H=H, d=d, S=S, n_chunks=n_chunks, topk=topk, Hr=Hr, D=D,
        score_scale=1.0 / math.sqrt(D) if score_scale is None else score_scale,
        attn_scale=1.0 / math.sqrt(d) if attn_scale is None else attn_scale,
        off_by_one=int(bool(off_by_one)),
        dtype={"fp32": GCA_FP32, "bf16": GCA_BF16}[dtype] if isinstance(dtype, str) else dtype,
        mode={"causal": GCA_CAUSAL, "decode": GCA_DECODE}[mode] if isinstance(mode, str) else mode,
        flags=flags,
        gumbel_seed=0 if gumbel_seed is None else int(gumbel_seed),
    )


# ----------------------------------------------------------- marshalling ----

def _torch():
    import torch
    return torch


def _elem_dtype(p: Problem):
    torch = _torch()
    return torch.bfloat16 if p.dtype == GCA_BF16 else torch.float32


def _ptr(t, name, dtype=None, shape=None, host_ok=False):
    if t is None:
        return None
    # a host tensor (GCA_FLAG_HOST_KV) is checked by the library itself: it must
    # be pinned memory with a device mapping (torch's is_pinned() query costs far
    # more than the call it would guard)
    if not t.is_cuda and not host_ok:
        raise ValueError(f"{name} must be a device tensor")
    if not t.is_contiguous():
        raise ValueError(f"{name} must be contiguous")
    if dtype is not None and t.dtype != dtype:
        raise ValueError(f"{name} must be {dtype}, got {t.dtype}")
    if shape is not None and tuple(t.shape) != tuple(shape):
        raise ValueError(f"{name} must have shape {tuple(shape)}, got {tuple(t.shape)}")
    return ctypes.c_void_p(t.data_ptr())


def _host_kv(p: Problem) -> bool:
    return bool(p.flags & FLAG_HOST_KV)


def _stream(stream):
    torch = _torch()
    if stream is None:
        stream = torch.cuda.current_stream()
    return ctypes.c_void_p(stream.cuda_stream)


def _alloc_on(stream):
    """Context for allocating outputs and workspace that the kernels use on
    `stream`: torch's caching allocator then ties the blocks to that stream, so a
    temporary freed on return is not handed to other streams' work while the
    kernels may still run."""
    import contextlib
    if stream is None:
        return contextlib.nullcontext()
    return _torch().cuda.stream(stream)


@dataclass
class Shapes:
    lmk_q: tuple
    lmk_k: tuple
    q: tuple
    kv: tuple
    rows: tuple     # [B, Hr, nQ, topk]
    scores: tuple   # [B, Hr, nQ, nC]
    lse: tuple      # [B, H, Lq, topk]


def shapes(p: Problem) -> Shapes:
    nQ, nC = p.n_query_chunks, p.n_chunks
    return Shapes(
        lmk_q=(p.B, p.Hr, nQ, p.D), lmk_k=(p.B, p.Hr, nC, p.D),
        q=(p.B, p.H, nQ * p.query_rows, p.d), kv=(p.B, p.H, nC * p.S, p.d),
        rows=(p.B, p.Hr, nQ, p.topk), scores=(p.B, p.Hr, nQ, nC),
        lse=(p.B, p.H, nQ * p.query_rows, p.topk),
    )


def workspace_size(p: Problem, op: int) -> int:
    return int(lib().gca_workspace_size(ctypes.byref(p), op))


def workspace(p: Problem, op: int, device="cuda"):
    torch = _torch()
    n = workspace_size(p, op)
    return torch.empty(max(n, 1), dtype=torch.uint8, device=device), n


# ------------------------------------------------------------ entry points ----

def chunk_scores(p: Problem, lmk_q, lmk_k, scores=None, stream=None):
    torch = _torch()
    sh, dt = shapes(p), _elem_dtype(p)
    with _alloc_on(stream):
        if scores is None:
            scores = torch.empty(sh.scores, dtype=torch.float32, device=lmk_q.device)
    _check(lib().gca_chunk_scores(ctypes.byref(p), _ptr(lmk_q, "lmk_q", dt, sh.lmk_q),
                                  _ptr(lmk_k, "lmk_k", dt, sh.lmk_k),
                                  _ptr(scores, "scores", torch.float32, sh.scores), _stream(stream)))
    return scores


def topk(p: Problem, scores, idx=None, sel=None, stream=None):
    torch = _torch()
    sh = shapes(p)
    with _alloc_on(stream):
        if idx is None:
            idx = torch.empty(sh.rows, dtype=torch.int32, device=scores.device)
        if sel is None:
            sel = torch.empty(sh.rows, dtype=torch.float32, device=scores.device)
    _check(lib().gca_topk(ctypes.byref(p), _ptr(scores, "scores", torch.float32, sh.scores),
                          _ptr(idx, "idx", torch.int32, sh.rows), _ptr(sel, "sel", torch.float32, sh.rows),
                          _stream(stream)))
    return idx, sel


def grouped_xattn_fwd(p: Problem, q, k, v, idx, sel, out=None, lse=None, w=None, want_lse=True,
                      want_w=True, stream=None):
    torch = _torch()
    sh, dt = shapes(p), _elem_dtype(p)
    dev = q.device
    with _alloc_on(stream):
        if out is None:
            out = torch.empty(sh.q, dtype=dt, device=dev)
        if lse is None and want_lse:
            lse = torch.empty(sh.lse, dtype=torch.float32, device=dev)
        if w is None and want_w:
            w = torch.empty(sh.rows, dtype=torch.float32, device=dev)
    _check(lib().gca_grouped_xattn_fwd(
        ctypes.byref(p), _ptr(q, "q", dt, sh.q),
        _ptr(k, "k", dt, sh.kv, _host_kv(p)), _ptr(v, "v", dt, sh.kv, _host_kv(p)),
        _ptr(idx, "idx", torch.int32, sh.rows), _ptr(sel, "sel", torch.float32, sh.rows),
        _ptr(out, "out", dt, sh.q), _ptr(lse, "lse", torch.float32, sh.lse),
        _ptr(w, "w", torch.float32, sh.rows), _stream(stream)))
    return out, lse, w


def grouped_xattn_bwd(p: Problem, q, k, v, idx, sel, lse, dout, lmk_q=None, lmk_k=None,
                      landmark_grads=True, ws=None, grads=None, stream=None):
    """Returns dict dq, dk, dv, dsel and (if landmark_grads) dlmk_q, dlmk_k.
    landmark_grads: True (both), False (neither), or a collection of the names
    "dlmk_q" / "dlmk_k" to request one of them."""
    torch = _torch()
    sh, dt = shapes(p), _elem_dtype(p)
    dev = q.device
    g = dict(grads or {})
    if landmark_grads is True:
        wanted = ("dlmk_q", "dlmk_k")
    elif not landmark_grads:
        wanted = ()
    else:
        wanted = tuple(landmark_grads)
        if not set(wanted) <= {"dlmk_q", "dlmk_k"}:
            raise ValueError(f"landmark_grads names must be dlmk_q / dlmk_k, got {wanted}")
    landmark_grads = bool(wanted)
    with _alloc_on(stream):
        for name, shape, gdt in (("dq", sh.q, dt), ("dk", sh.kv, dt), ("dv", sh.kv, dt),
                                 ("dsel", sh.rows, torch.float32)):
            if name not in g:
                g[name] = torch.empty(shape, dtype=gdt, device=dev)
        for name, shape in (("dlmk_q", sh.lmk_q), ("dlmk_k", sh.lmk_k)):
            if name in wanted and name not in g:
                g[name] = torch.empty(shape, dtype=torch.float32, device=dev)
        if ws is None:
            ws, nbytes = workspace(p, OP_BACKWARD, dev)
        else:
            nbytes = ws.numel()
    _check(lib().gca_grouped_xattn_bwd(
        ctypes.byref(p), _ptr(q, "q", dt, sh.q),
        _ptr(k, "k", dt, sh.kv, _host_kv(p)), _ptr(v, "v", dt, sh.kv, _host_kv(p)),
        _ptr(idx, "idx", torch.int32, sh.rows), _ptr(sel, "sel", torch.float32, sh.rows),
        _ptr(lse, "lse", torch.float32, sh.lse), _ptr(dout, "dout", dt, sh.q),
        _ptr(g["dq"], "dq", dt, sh.q), _ptr(g["dk"], "dk", dt, sh.kv), _ptr(g["dv"], "dv", dt, sh.kv),
        _ptr(g["dsel"], "dsel", torch.float32, sh.rows),
        _ptr(lmk_q, "lmk_q", dt, sh.lmk_q) if landmark_grads else None,
        _ptr(lmk_k, "lmk_k", dt, sh.lmk_k) if landmark_grads else None,
        _ptr(g.get("dlmk_q") if "dlmk_q" in wanted else None, "dlmk_q", torch.float32, sh.lmk_q),
        _ptr(g.get("dlmk_k") if "dlmk_k" in wanted else None, "dlmk_k", torch.float32, sh.lmk_k),
        _ptr(ws, "workspace"), ctypes.c_size_t(nbytes), _stream(stream)))
    return g


def forward(p: Problem, lmk_q, lmk_k, q, k, v, out=None, idx=None, sel=None, lse=None, w=None,
            want_lse=True, want_w=True, ws=None, stream=None):
    """The whole path; returns dict out, idx, sel, lse, w."""
    torch = _torch()
    sh, dt = shapes(p), _elem_dtype(p)
    dev = q.device
    with _alloc_on(stream):
        if out is None:
            out = torch.empty(sh.q, dtype=dt, device=dev)
        if idx is None:
            idx = torch.empty(sh.rows, dtype=torch.int32, device=dev)
        if sel is None:
            sel = torch.empty(sh.rows, dtype=torch.float32, device=dev)
        if lse is None and want_lse:
            lse = torch.empty(sh.lse, dtype=torch.float32, device=dev)
        if w is None and want_w:
            w = torch.empty(sh.rows, dtype=torch.float32, device=dev)
        if ws is None:
            ws, nbytes = workspace(p, OP_FORWARD, dev)
        else:
            nbytes = ws.numel()
    _check(lib().gca_forward(
        ctypes.byref(p), _ptr(lmk_q, "lmk_q", dt, sh.lmk_q), _ptr(lmk_k, "lmk_k", dt, sh.lmk_k),
        _ptr(q, "q", dt, sh.q),
        _ptr(k, "k", dt, sh.kv, _host_kv(p)), _ptr(v, "v", dt, sh.kv, _host_kv(p)),
        _ptr(out, "out", dt, sh.q), _ptr(idx, "idx", torch.int32, sh.rows),
        _ptr(sel, "sel", torch.float32, sh.rows), _ptr(lse, "lse", torch.float32, sh.lse),
        _ptr(w, "w", torch.float32, sh.rows), _ptr(ws, "workspace"), ctypes.c_size_t(nbytes),
        _stream(stream)))
    return {"out": out, "idx": idx, "sel": sel, "lse": lse, "w": w}


def forward_noalloc(p: Problem, lmk_q, lmk_k, q, k, v, out, idx, sel, lse=None, w=None, stream=None):
    """gca_forward_noalloc: the whole forward path into caller-provided outputs,
    with the library's own per-device scratch as workspace (nothing allocated)."""
    torch = _torch()
    sh, dt = shapes(p), _elem_dtype(p)
    _check(lib().gca_forward_noalloc(
        ctypes.byref(p), _ptr(lmk_q, "lmk_q", dt, sh.lmk_q), _ptr(lmk_k, "lmk_k", dt, sh.lmk_k),
        _ptr(q, "q", dt, sh.q),
        _ptr(k, "k", dt, sh.kv, _host_kv(p)), _ptr(v, "v", dt, sh.kv, _host_kv(p)),
        _ptr(out, "out", dt, sh.q), _ptr(idx, "idx", torch.int32, sh.rows),
        _ptr(sel, "sel", torch.float32, sh.rows), _ptr(lse, "lse", torch.float32, sh.lse),
        _ptr(w, "w", torch.float32, sh.rows), _stream(stream)))
    return {"out": out, "idx": idx, "sel": sel, "lse": lse, "w": w}


# -------------------------------------------------------------- chunk cache ----

class Cache:
    """A bounded 8-bit chunk cache (``gca_cache``): its sizes and its device tensors, which
    are the program's own and may be read or, between calls, changed in place:

    * ``k`` [B, Hkv, C, 64 tokens, 64], ``v`` [B, Hkv, C, 64, 64 tokens]: 8-bit numbers
      (``torch.float8_e4m3fn`` or ``torch.int8``), values transposed per chunk;
    * ``k_scale``, ``v_scale`` [B, Hkv, C] fp32: a number stands for itself times these;
    * ``lmk`` [B, Hr, C, D]: landmark keys; ``tokens`` [B, C] int32: 0 = free slot;
    * ``mass`` [B, C] fp32, ``number`` [B, C] int32, ``next`` [B] int32: what eviction goes by.

    To give sequence b's place to another sequence, zero ``tokens[b]``, ``mass[b]`` and
    ``next[b]``."""

    NAMES = ("k", "v", "k_scale", "v_scale", "lmk", "tokens", "mass", "number", "next")

    def __init__(self, struct, tensors, device, index):
        self.torch = torch = _torch()
        self.struct = struct
        self.ref = ctypes.byref(struct)
        self.device = device
        self.index = index    # the device's ordinal
        self.here = _Here(torch, index)
        self.dims = struct.B, struct.H, struct.Hkv, struct.Hr, struct.D, struct.topk
        self.elem = torch.bfloat16 if struct.dtype == GCA_BF16 else torch.float32
        for name in self.NAMES:
            setattr(self, name, tensors[name])


def cache_shapes(B, Hkv, capacity, Hr, D):
    """Shapes of a cache's tensors, by name."""
    return dict(k=(B, Hkv, capacity, 64, 64), v=(B, Hkv, capacity, 64, 64), k_scale=(B, Hkv, capacity),
                v_scale=(B, Hkv, capacity), lmk=(B, Hr, capacity, D), tokens=(B, capacity), mass=(B, capacity),
                number=(B, capacity), next=(B,))


def cache(B, H, capacity, topk, Hkv=None, Hr=1, D=None, score_scale=None, attn_scale=None, off_by_one=False,
          dtype="bf16", format="e4m3", device="cuda", tensors=None) -> Cache:
    """A cache of `capacity` chunks for each of B sequences, all slots free.  Hkv defaults to H, D
    to H * 64, the scales to 1/sqrt(D) and 1/sqrt(64); ``format`` is "e4m3" or "int8".  Members
    named in ``tensors`` are taken as they are instead of allocated."""
    torch = _torch()
    Hkv, D = H if Hkv is None else Hkv, H * 64 if D is None else D
    elem = {"bf16": torch.bfloat16, "fp32": torch.float32}[dtype]
    num = {"e4m3": torch.float8_e4m3fn, "int8": torch.int8}[format]
    types = dict(k=num, v=num, k_scale=torch.float32, v_scale=torch.float32, lmk=elem, tokens=torch.int32,
                 mass=torch.float32, number=torch.int32, next=torch.int32)
    sh = cache_shapes(B, Hkv, capacity, Hr, D)
    given = dict(tensors or {})
    if not set(given) <= set(sh):
        raise ValueError(f"a cache has no tensors named {sorted(set(given) - set(sh))}")
    device = torch.device(device)
    if device.type != "cuda":
        raise ValueError("a cache lives in device memory")
    if device.index is None:
        device = next(iter(given.values())).device if given else torch.device("cuda", torch.cuda.current_device())
    for name, t in given.items():
        _ptr(t, name, types[name], sh[name])
        if t.device != device:
            raise ValueError(f"{name} is on {t.device}, the cache on {device}")
    for name in sh:
        if name not in given:
            given[name] = torch.zeros(sh[name], dtype=types[name], device=device)
    struct = CacheStruct(
        B=B, H=H, Hkv=Hkv, Hr=Hr, d=64, S=64, capacity=capacity, topk=topk, D=D,
        score_scale=1.0 / math.sqrt(D) if score_scale is None else score_scale,
        attn_scale=0.125 if attn_scale is None else attn_scale, off_by_one=int(bool(off_by_one)),
        dtype=GCA_BF16 if dtype == "bf16" else GCA_FP32, format=GCA_E4M3 if format == "e4m3" else GCA_INT8, flags=0,
        **{name: given[name].data_ptr() for name in sh})
    return Cache(struct, given, device, device.index)


def cache_workspace_size(c: Cache, op: int, n: int = 0) -> int:
    return int(lib().gca_cache_workspace_size(c.ref, op, n))


def cache_workspace(c: Cache, op: int, n: int = 0):
    """Workspace of CACHE_SELECT, or of CACHE_EVICT of up to n chunks, on the cache's device."""
    size = cache_workspace_size(c, op, n)
    return _torch().empty(max(size, 1), dtype=_torch().uint8, device=c.device), size


class _Here:
    """Context of a cache's call on the current stream of its device, which is the current one; the
    value is the stream's handle.  (One per cache: it holds nothing of a call.)"""

    __slots__ = ("raw", "index")

    def __init__(self, torch, index):
        self.raw, self.index = torch._C._cuda_getCurrentRawStream, index

    def __enter__(self):
        return self.raw(self.index)

    def __exit__(self, *exc):
        pass


class _There:
    """The same on another stream or another device's: made current while the call allocates and
    launches."""

    def __init__(self, ctx, c: Cache):
        self.ctx, self.c = ctx, c

    def __enter__(self):
        self.ctx.__enter__()
        return self.c.here.__enter__()

    def __exit__(self, *exc):
        self.ctx.__exit__(*exc)


def _at(c: Cache, stream):
    """Context in which a cache's call allocates and launches: on the given stream, or the current
    one of the cache's device."""
    torch = c.torch
    if stream is None:
        if torch._C._cuda_getDevice() == c.index:
            return c.here
        return _There(torch.cuda.device(c.index), c)
    if stream.device != c.device:
        raise ValueError(f"the stream is on {stream.device}, the cache on {c.device}")
    return _There(torch.cuda.stream(stream), c)


def _cache_ptr(c: Cache, t, name, dtype, shape):
    """The address of a tensor of a cache's call (one expression where all is well: these checks are
    a large part of what a call of a few microseconds costs)."""
    if t is None:
        return None
    if t.get_device() == c.index and t.dtype is dtype and t.shape == shape and t.is_contiguous():
        return t.data_ptr()
    if t.device != c.device:
        raise ValueError(f"{name} must be on the cache's device {c.device}, got {t.device}")
    if t.dtype != dtype:
        raise ValueError(f"{name} must be {dtype}, got {t.dtype}")
    if t.shape != shape:
        raise ValueError(f"{name} must have shape {tuple(shape)}, got {tuple(t.shape)}")
    raise ValueError(f"{name} must be contiguous")


def _new(c: Cache, shape, dtype, like=None):
    """A new output and its address (nothing to check); `like`: a tensor of its shape, which is cheaper
    to go by."""
    t = c.torch.empty(shape, dtype=dtype, device=c.device) if like is None else c.torch.empty_like(like, dtype=dtype)
    return t, t.data_ptr()


def cache_store(c: Cache, k, v, lmk, slots, lengths=None, stream=None):
    """gca_cache_store: chunks of k, v [B, Hkv, n * 64, 64] (and their landmark keys lmk
    [B, Hr, n, D], or None) into slots [B, n]; lengths [B]: new tokens of each sequence."""
    i32 = c.torch.int32
    B, _, Hkv, Hr, D, _ = c.dims
    if slots.dim() != 2:
        raise ValueError("slots must have shape (B, n)")
    n = slots.shape[1]
    kv = (B, Hkv, n * 64, 64)
    with _at(c, stream) as st:
        _check(lib().gca_cache_store(c.ref, _cache_ptr(c, k, "k", c.elem, kv), _cache_ptr(c, v, "v", c.elem, kv),
                                     _cache_ptr(c, lmk, "lmk", c.elem, (B, Hr, n, D)),
                                     _cache_ptr(c, slots, "slots", i32, (B, n)),
                                     _cache_ptr(c, lengths, "lengths", i32, (B,)), n, st))


def cache_select(c: Cache, lmk_q, idx=None, sel=None, w=None, want_w=True, ws=None, stream=None):
    """gca_cache_select: the best slots in use for landmark queries lmk_q [B, Hr, 1, D];
    returns idx, sel, w [B, Hr, 1, topk]."""
    i32, f32 = c.torch.int32, c.torch.float32
    B, _, _, Hr, D, K = c.dims
    rows = (B, Hr, 1, K)
    qp, ip = _cache_ptr(c, lmk_q, "lmk_q", c.elem, (B, Hr, 1, D)), _cache_ptr(c, idx, "idx", i32, rows)
    sp, wp = _cache_ptr(c, sel, "sel", f32, rows), _cache_ptr(c, w, "w", f32, rows)
    with _at(c, stream) as st:
        if idx is None:
            idx, ip = _new(c, rows, i32, sel)
        if sel is None:
            sel, sp = _new(c, rows, f32, idx)
        if w is None and want_w:
            w, wp = _new(c, rows, f32, sel)
        if ws is None:
            ws = cache_workspace(c, CACHE_SELECT)[0]
        _check(lib().gca_cache_select(c.ref, qp, ip, sp, wp, _cache_ptr(c, ws, "workspace", c.torch.uint8, ws.shape),
                                      ws.numel(), st))
    return idx, sel, w


def cache_xattn(c: Cache, q, idx, sel, out=None, lse=None, w=None, want_lse=True, want_w=True, causal=False,
                stream=None):
    """gca_cache_xattn: query rows q [B, H, nQ * rows, 64] against the chunks that their group's
    list idx, sel [B, Hr, nQ, topk] names (causal: the list before); returns out, lse, w."""
    i32, f32 = c.torch.int32, c.torch.float32
    B, H, _, Hr, _, K = c.dims
    if q.dim() != 4 or idx.dim() != 4:
        raise ValueError("q must have shape (B, H, nQ * rows, 64) and idx (B, Hr, nQ, topk)")
    nQ, Lq = idx.shape[2], q.shape[2]
    if nQ < 1 or Lq < 1 or Lq % nQ:
        raise ValueError(f"q's {Lq} rows are not a positive multiple of idx's {nQ} lists")
    qs, rows, ls = (B, H, Lq, 64), (B, Hr, nQ, K), (B, H, Lq, K)
    qp, ip = _cache_ptr(c, q, "q", c.elem, qs), _cache_ptr(c, idx, "idx", i32, rows)
    sp, op = _cache_ptr(c, sel, "sel", f32, rows), _cache_ptr(c, out, "out", c.elem, qs)
    lp, wp = _cache_ptr(c, lse, "lse", f32, ls), _cache_ptr(c, w, "w", f32, rows)
    with _at(c, stream) as st:
        if out is None:
            out, op = _new(c, qs, c.elem, q)
        if lse is None and want_lse:
            lse, lp = _new(c, ls, f32)
        if w is None and want_w:
            w, wp = _new(c, rows, f32, sel)
        _check(lib().gca_cache_xattn(c.ref, qp, ip, sp, op, lp, wp, nQ, Lq // nQ, int(bool(causal)), st))
    return out, lse, w


def cache_evict(c: Cache, n, idx=None, w=None, decay=1.0, keep_first=0, keep_last=1, want=None, slots=None, ws=None,
                stream=None):
    """gca_cache_evict: adds the weights w of the lists idx [B, Hr, nQ, topk] to the masses and
    returns slots [B, n] for each sequence's next n chunks (want [B]: the number of chunks that each
    will store, where some have fewer)."""
    i32, f32 = c.torch.int32, c.torch.float32
    B, _, _, Hr, _, K = c.dims
    nQ = 0
    if idx is not None:
        if idx.dim() != 4 or idx.shape[2] < 1:
            raise ValueError("idx must have shape (B, Hr, nQ, topk)")
        nQ = idx.shape[2]
    rows = (B, Hr, nQ, K)
    ip, wp = _cache_ptr(c, idx, "idx", i32, rows), _cache_ptr(c, w, "w", f32, rows)
    want_p, sp = _cache_ptr(c, want, "want", i32, (B,)), _cache_ptr(c, slots, "slots", i32, (B, n))
    with _at(c, stream) as st:
        if slots is None:
            slots, sp = _new(c, (B, n), i32)
        if ws is None:
            ws = cache_workspace(c, CACHE_EVICT, n)[0]
        _check(lib().gca_cache_evict(c.ref, ip, wp, nQ, decay, keep_first, keep_last, want_p, sp if n else None, n,
                                     _cache_ptr(c, ws, "workspace", c.torch.uint8, ws.shape), ws.numel(), st))
    return slots


# ---------------------------------------------------------------- profiling ----

def profile_arm(event_array, capacity: int) -> None:
    """Arm the per-kernel event hook with a ctypes array of hipEvent_t (None disarms)."""
    lib().gca_profile_arm(event_array, capacity if event_array is not None else 0)


def profile_record():
    """Kernel names preceding each recorded event since arming."""
    L = lib()
    return [L.gca_profile_name(i).decode() for i in range(L.gca_profile_count())]
