"""Thin ctypes binding of include/unison_kv.h (argument marshalling only).

The operators of one serving step over a paged KV cache: ``attend``,
``verify``, ``observe``, ``commit`` and ``evict``.  ``Cache`` and ``Tree`` hold
the descriptions that a serving program keeps; the calls take the step's
tensors.  Every computation runs in libunison.so's CUDA kernels; calls are
queued on the current (or the given) stream and synchronise nothing.
"""
from __future__ import annotations

import ctypes as C
import threading

import torch

from . import binding

MAX_TOKENS = 64  # new tokens of one session in one call
DTYPE = {torch.bfloat16: 0, torch.float16: 1, torch.float32: 2}


class KvCache(C.Structure):
    _fields_ = [(f, C.c_void_p) for f in ("k", "v", "mass", "pos", "page_table", "length", "next_pos", "status")] + \
        [(f, C.c_int64) for f in ("k_page", "k_head", "k_slot", "v_page", "v_head", "v_slot", "m_page", "m_head",
                                  "m_slot")] + \
        [(f, C.c_int32) for f in ("n_seqs", "max_pages", "n_pages", "page_size", "n_heads", "head_dim", "dtype",
                                  "reserved")]


class KvTree(C.Structure):
    _fields_ = [(f, C.c_void_p) for f in ("offsets", "mask", "parent")] + \
        [(f, C.c_int32) for f in ("n_seqs", "n_tokens", "max_tokens", "reserved")]


class KvStep(C.Structure):
    _fields_ = [(f, C.c_void_p) for f in ("q", "k_new", "v_new", "out", "lse", "mass_new")] + \
        [(f, C.c_int64) for f in ("q_token", "q_head", "k_token", "k_head", "v_token", "v_head", "out_token",
                                  "out_head")] + [("n_q_heads", C.c_int32), ("scale", C.c_float)]


class KvPath(C.Structure):
    _fields_ = [("path", C.c_void_p), ("n_path", C.c_void_p), ("path_stride", C.c_int64)]


class KvVerify(C.Structure):
    _fields_ = [("p", C.c_void_p), ("q", C.c_void_p), ("p_row", C.c_int64), ("q_row", C.c_int64)] + \
        [(f, C.c_void_p) for f in ("token", "u", "u_sample", "path", "n_path", "next_token")] + \
        [("path_stride", C.c_int64), ("vocab", C.c_int32), ("dtype", C.c_int32)]


# Every symbol include/unison_kv.h declares (checked by the ABI tests).
EXPORTS = ["unison_kv_attend_workspace", "unison_kv_attend", "unison_kv_observe", "unison_kv_commit",
           "unison_kv_evict_workspace", "unison_kv_evict", "unison_kv_verify"]

_lock = threading.Lock()
_lib = None


def lib():
    """libunison.so with the signatures of include/unison_kv.h."""
    global _lib
    if _lib is None:
        L = binding.lib()
        with _lock:
            P = C.POINTER
            L.unison_kv_attend_workspace.argtypes = [P(KvCache), P(KvTree), C.c_int]
            L.unison_kv_attend_workspace.restype = C.c_uint64
            L.unison_kv_attend.argtypes = [P(KvCache), P(KvTree), P(KvStep), C.c_void_p, C.c_uint64, C.c_void_p]
            L.unison_kv_observe.argtypes = [P(KvCache), P(KvTree), P(KvStep), P(KvPath), C.c_void_p]
            L.unison_kv_commit.argtypes = L.unison_kv_observe.argtypes
            L.unison_kv_evict_workspace.argtypes = [P(KvCache)]
            L.unison_kv_evict_workspace.restype = C.c_uint64
            L.unison_kv_evict.argtypes = [P(KvCache), P(KvCache), C.c_void_p, C.c_int32, C.c_int32, C.c_void_p,
                                          C.c_uint64, C.c_void_p]
            L.unison_kv_verify.argtypes = [P(KvTree), P(KvVerify), C.c_void_p]
            _lib = L
    return _lib


def _need(ok, what):
    if not ok:
        raise ValueError(what)


def _dense(x, dtype, shape, what):
    if x is not None:
        _need(x.dtype == dtype and tuple(x.shape) == shape and x.is_contiguous(),
              f"{what}: a contiguous {dtype} tensor of shape {shape} is wanted")
        return x.data_ptr()
    return None


class Cache:
    """The paged KV cache of a batch of sessions (one layer).

    k, v: [page, head, slot, head_dim], bfloat16 or float16, the last axis
    contiguous, the others of any stride (a pool that is stored as [page, slot,
    head, head_dim] is passed as its permuted view).  page_table: int32
    [session, page], -1 where there is none; length: int32 [session] slots in
    use; mass (float32) and pos (int32): [page, head, slot], of the same
    strides; next_pos: int32 [session]; status: int32 [session], where device
    values out of range are reported.  The tensors stay the caller's and are
    changed in place.
    """

    def __init__(self, k, v, page_table, length, mass=None, pos=None, next_pos=None, status=None):
        _need(k.dim() == 4 and k.shape == v.shape, "k, v: [page, head, slot, head_dim] of the same shape")
        _need(k.dtype == v.dtype and k.dtype in (torch.bfloat16, torch.float16), "k, v: bfloat16 or float16")
        _need(k.stride(3) == 1 and v.stride(3) == 1, "k, v: the last axis is contiguous")
        _need(page_table.dim() == 2, "page_table: [session, page]")
        n, pages = page_table.shape
        marks = [x for x in (mass, pos) if x is not None]
        for x, dt in ((mass, torch.float32), (pos, torch.int32)):
            _need(x is None or (x.dtype == dt and x.shape == k.shape[:3]), "mass float32, pos int32: [page, head, slot]")
        _need(len(marks) < 2 or mass.stride() == pos.stride(), "mass and pos: the same strides")
        m = marks[0].stride() if marks else (0, 0, 0)
        ptr = lambda x: None if x is None else x.data_ptr()  # noqa: E731
        self.tensors = (k, v, page_table, length, mass, pos, next_pos, status)  # kept while the pointers are used
        self.k, self.v, self.page_table, self.length, self.mass, self.pos, self.next_pos, self.status = self.tensors
        self.dtype, self.device, self.n_seqs = k.dtype, k.device, n
        self.n_heads, self.head_dim = k.shape[1], k.shape[3]
        self.struct = KvCache(
            k.data_ptr(), v.data_ptr(), ptr(mass), ptr(pos), _dense(page_table, torch.int32, (n, pages), "page_table"),
            _dense(length, torch.int32, (n,), "length"), _dense(next_pos, torch.int32, (n,), "next_pos"),
            _dense(status, torch.int32, (n,), "status"), *k.stride()[:3], *v.stride()[:3], *m, n, pages, k.shape[0],
            k.shape[2], k.shape[1], k.shape[3], DTYPE[k.dtype], 0)
        self.ref = C.byref(self.struct)


class Tree:
    """The new tokens of a step: session b owns tokens offsets[b] ..
    offsets[b+1]-1 (int32 tensor of n_seqs + 1), at most max_tokens of them.
    mask: int64 [token], bit j of a node's word if it sees node j of its
    session (None: a chain); parent: int32 [token], read by ``verify``."""

    def __init__(self, offsets, max_tokens, mask=None, parent=None, n_tokens=None):
        n = n_tokens
        for x in (mask, parent):
            n = x.shape[0] if n is None and x is not None else n
        _need(n is not None, "n_tokens is wanted where neither mask nor parent tells it")
        self.tensors = (offsets, mask, parent)
        self.n_seqs, self.n_tokens, self.max_tokens = offsets.shape[0] - 1, n, max_tokens
        self.struct = KvTree(_dense(offsets, torch.int32, (self.n_seqs + 1,), "offsets"),
                             _dense(mask, torch.int64, (n,), "mask"), _dense(parent, torch.int32, (n,), "parent"),
                             self.n_seqs, n, max_tokens, 0)
        self.ref = C.byref(self.struct)


def _step(cache, tree, q, k_new, v_new, out, lse, mass_new, scale):
    """The C struct of a step's tensors, each [token, head, head_dim] with a contiguous last axis."""
    args, strides = [], []
    for x, heads in ((q, None), (k_new, cache.n_heads), (v_new, cache.n_heads), (out, None)):
        if x is None:
            args.append(None)
            strides += (0, 0)
            continue
        s, t = x.shape, x.stride()
        if x.dtype != cache.dtype or len(s) != 3 or s[0] != tree.n_tokens or s[2] != cache.head_dim or t[2] != 1 or \
                (heads is not None and s[1] != heads):
            raise ValueError("step tensors: [token, head, head_dim] of the cache's type and sizes, last axis contiguous")
        args.append(x.data_ptr())
        strides += t[:2]
    return KvStep(*args, None if lse is None else lse.data_ptr(), None if mass_new is None else mass_new.data_ptr(),
                  *strides, 0 if q is None else q.shape[1], cache.head_dim ** -0.5 if scale is None else scale)


def _path(tree, path, n_path):
    if path is None:
        return None
    _need(path.dtype == torch.int32 and path.dim() == 2 and path.shape[0] == tree.n_seqs and path.stride(1) == 1 and
          path.shape[1] >= tree.max_tokens, "path: int32 [session, max_tokens]")
    return C.byref(KvPath(path.data_ptr(), _dense(n_path, torch.int32, (tree.n_seqs,), "n_path"), path.stride(0)))


class _On:
    """Allocations of a call belong to the stream that it is queued on."""

    def __init__(self, stream):
        self.given = stream
        self.handle = binding._stream_handle(stream)
        self.context = None

    def __enter__(self):
        if self.given is not None and hasattr(self.given, "cuda_stream"):
            self.context = torch.cuda.stream(self.given)
            self.context.__enter__()
        return self.handle

    def __exit__(self, *e):
        if self.context is not None:
            self.context.__exit__(*e)


def attend(cache: Cache, tree: Tree, q, k_new, v_new, scale=None, out=None, lse=None, workspace=None, stream=None):
    """unison_kv_attend: (out [token, q head, head_dim], lse float32 [token, q
    head]).  scale defaults to head_dim ** -0.5; workspace: a uint8 tensor of
    at least ``attend_workspace`` bytes, else one is allocated."""
    with _On(stream) as handle:
        out = torch.empty_like(q) if out is None else out
        lse = torch.empty(q.shape[:2], dtype=torch.float32, device=q.device) if lse is None else lse
        _need(out.shape == q.shape, "out: the shape of q")
        _dense(lse, torch.float32, tuple(q.shape[:2]), "lse")
        step = _step(cache, tree, q, k_new, v_new, out, lse, None, scale)
        if workspace is None:
            workspace = torch.empty(attend_workspace(cache, tree, q.shape[1]), dtype=torch.uint8, device=q.device)
        binding._check("unison_kv_attend", lib().unison_kv_attend(
            cache.ref, tree.ref, C.byref(step), workspace.data_ptr(), workspace.numel(), handle))
    return out, lse


def attend_workspace(cache: Cache, tree: Tree, n_q_heads: int) -> int:
    return int(lib().unison_kv_attend_workspace(cache.ref, tree.ref, n_q_heads))


def observe(cache: Cache, tree: Tree, q, lse, k_new, scale=None, path=None, n_path=None, mass_new=None, stream=None):
    """unison_kv_observe: adds to cache.mass; returns mass_new, float32 [token,
    head], the weight of the new tokens themselves."""
    with _On(stream) as handle:
        mass_new = torch.empty((tree.n_tokens, cache.n_heads), dtype=torch.float32, device=q.device) \
            if mass_new is None else mass_new
        _dense(mass_new, torch.float32, (tree.n_tokens, cache.n_heads), "mass_new")
        _dense(lse, torch.float32, tuple(q.shape[:2]), "lse")
        step = _step(cache, tree, q, k_new, None, None, lse, mass_new, scale)
        binding._check("unison_kv_observe", lib().unison_kv_observe(
            cache.ref, tree.ref, C.byref(step), _path(tree, path, n_path), handle))
    return mass_new


def commit(cache: Cache, tree: Tree, k_new, v_new, mass_new=None, path=None, n_path=None, stream=None) -> None:
    """unison_kv_commit: the accepted tokens go into the pages, length and
    next_pos grow.  Without path every new token is accepted."""
    _dense(mass_new, torch.float32, (tree.n_tokens, cache.n_heads), "mass_new")
    step = _step(cache, tree, None, k_new, v_new, None, None, mass_new, 0.0)
    binding._check("unison_kv_commit", lib().unison_kv_commit(
        cache.ref, tree.ref, C.byref(step), _path(tree, path, n_path), binding._stream_handle(stream)))


def evict_workspace(cache: Cache) -> int:
    return int(lib().unison_kv_evict_workspace(cache.ref))


def evict(cache: Cache, keep, sink=0, recent=0, into: Cache | None = None, workspace=None, stream=None) -> None:
    """unison_kv_evict: at most keep[b] (int32 tensor) slots of each session
    stay, in place or, with ``into``, in another cache."""
    _dense(keep, torch.int32, (cache.n_seqs,), "keep")
    with _On(stream) as handle:
        if workspace is None:
            workspace = torch.empty(evict_workspace(cache), dtype=torch.uint8, device=cache.device)
        binding._check("unison_kv_evict", lib().unison_kv_evict(
            cache.ref, None if into is None else into.ref, keep.data_ptr(), sink, recent, workspace.data_ptr(),
            workspace.numel(), handle))


def verify(tree: Tree, token, p, q, u, u_sample, path=None, n_path=None, next_token=None, stream=None):
    """unison_kv_verify: (path [session, max_tokens], n_path [session],
    next_token [session]), all int32.  p, q: [token, vocab] probabilities of
    one type (q None: certain drafts); token int32 [token]; u float32 [token];
    u_sample float32 [session]."""
    n, t = tree.n_seqs, tree.max_tokens
    for x in (p, q):
        _need(x is None or (x.dim() == 2 and x.dtype == p.dtype and x.dtype in DTYPE and x.stride(1) == 1 and
                            x.shape == (tree.n_tokens, p.shape[1])), "p, q: [token, vocab] of one type")
    with _On(stream) as handle:
        new = lambda *s: torch.empty(s, dtype=torch.int32, device=p.device)  # noqa: E731
        path = new(n, t) if path is None else path
        n_path = new(n) if n_path is None else n_path
        next_token = new(n) if next_token is None else next_token
        _need(path.dtype == torch.int32 and path.dim() == 2 and path.shape[0] == n and path.shape[1] >= t and
              path.stride(1) == 1, "path: int32 [session, max_tokens]")
        args = KvVerify(
            p.data_ptr(), None if q is None else q.data_ptr(), p.stride(0), 0 if q is None else q.stride(0),
            _dense(token, torch.int32, (tree.n_tokens,), "token"), _dense(u, torch.float32, (tree.n_tokens,), "u"),
            _dense(u_sample, torch.float32, (n,), "u_sample"), path.data_ptr(),
            _dense(n_path, torch.int32, (n,), "n_path"), _dense(next_token, torch.int32, (n,), "next_token"),
            path.stride(0), p.shape[1], DTYPE[p.dtype])
        binding._check("unison_kv_verify", lib().unison_kv_verify(tree.ref, C.byref(args), handle))
    return path, n_path, next_token
