"""Thin ctypes binding of include/unison_kv.h (argument marshalling only).

The operators of one serving step over a paged KV cache: ``attend``,
``verify``, ``observe``, ``commit`` and ``evict``.  ``Cache`` and ``Tree`` hold
the descriptions that a serving program keeps; the calls take the step's
tensors.  Every computation runs in libunison.so's CUDA kernels; calls are
queued on the current (or the given) stream and synchronise nothing.
"""
from __future__ import annotations

import ctypes as C
import struct
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
            A, B = C.c_void_p, C.c_char_p  # a struct's address, a packed struct
            L.unison_kv_attend_workspace.argtypes = [A, A, C.c_int]
            L.unison_kv_attend_workspace.restype = C.c_uint64
            L.unison_kv_attend.argtypes = [A, A, B, A, C.c_uint64, A]
            L.unison_kv_observe.argtypes = [A, A, B, B, A]
            L.unison_kv_commit.argtypes = L.unison_kv_observe.argtypes
            L.unison_kv_evict_workspace.argtypes = [A]
            L.unison_kv_evict_workspace.restype = C.c_uint64
            L.unison_kv_evict.argtypes = [A, A, A, C.c_int32, C.c_int32, A, C.c_uint64, A]
            L.unison_kv_verify.argtypes = [A, B, A]
            _lib = L
    return _lib


def _need(ok, what):
    if not ok:
        raise ValueError(what)


def _dense(x, dtype, shape, what, device):
    if x is None or x.dtype is not dtype or x.shape != shape or not x.is_contiguous() or x.device != device:
        raise ValueError(f"{what}: a contiguous {dtype} tensor of shape {shape} on {device} is wanted")
    return x.data_ptr()


def _given(x, *wanted):
    """The same of a tensor that may be left out."""
    return None if x is None else _dense(x, *wanted)


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
        device = k.device
        _need(v.device == device, "k, v: on one device")
        _need(k.stride(3) == 1 and v.stride(3) == 1, "k, v: the last axis is contiguous")
        _need(page_table.dim() == 2, "page_table: [session, page]")
        n, pages = page_table.shape
        marks = [x for x in (mass, pos) if x is not None]
        for x, dt in ((mass, torch.float32), (pos, torch.int32)):
            _need(x is None or (x.dtype == dt and x.shape == k.shape[:3] and x.device == device),
                  "mass float32, pos int32: [page, head, slot], on the device of k")
        _need(len(marks) < 2 or mass.stride() == pos.stride(), "mass and pos: the same strides")
        m = marks[0].stride() if marks else (0, 0, 0)
        ptr = lambda x: None if x is None else x.data_ptr()  # noqa: E731
        self.tensors = (k, v, page_table, length, mass, pos, next_pos, status)  # kept while the pointers are used
        self.k, self.v, self.page_table, self.length, self.mass, self.pos, self.next_pos, self.status = self.tensors
        self.dtype, self.device, self.n_seqs, self.on_gpu = k.dtype, k.device, n, k.is_cuda
        self.n_heads, self.head_dim = k.shape[1], k.shape[3]
        self.struct = KvCache(
            k.data_ptr(), v.data_ptr(), ptr(mass), ptr(pos),
            _dense(page_table, torch.int32, (n, pages), "page_table", device),
            _dense(length, torch.int32, (n,), "length", device),
            _given(next_pos, torch.int32, (n,), "next_pos", device),
            _given(status, torch.int32, (n,), "status", device), *k.stride()[:3], *v.stride()[:3], *m, n, pages,
            k.shape[0], k.shape[2], k.shape[1], k.shape[3], DTYPE[k.dtype], 0)
        self.address = C.addressof(self.struct)
        self.scale = self.head_dim ** -0.5
        self.sizes = {}    # bytes of workspace, by the call's sizes
        self.scratch = {}  # workspaces, by stream


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
        self.device = offsets.device
        self.struct = KvTree(_dense(offsets, torch.int32, (self.n_seqs + 1,), "offsets", self.device),
                             _given(mask, torch.int64, (n,), "mask", self.device),
                             _given(parent, torch.int32, (n,), "parent", self.device), self.n_seqs, n, max_tokens, 0)
        self.address = C.addressof(self.struct)


# One packed unison_kv_step, unison_kv_path and unison_kv_verify_args: a call
# passes the bytes, which ctypes hands over without a copy or a conversion per
# field.
_STEP = struct.Struct("=6Q8qif")
_PATH = struct.Struct("=2Qq")
_VERIFY = struct.Struct("=2Q2q6Qq2i")
assert (_STEP.size, _PATH.size, _VERIFY.size) == (C.sizeof(KvStep), C.sizeof(KvPath), C.sizeof(KvVerify))
_NO_STRIDES = (0, 0, 0)


def _rows(cache, x, n, heads):
    """(pointer, strides) of a step's tensor [n, heads, head_dim] of the cache's type, its last axis contiguous."""
    s = x.stride()
    if x.dtype is not cache.dtype or x.shape != (n, heads, cache.head_dim) or s[2] != 1 or x.device != cache.device:
        raise ValueError(f"step tensors: {cache.dtype} [{n}, {heads}, {cache.head_dim}] on {cache.device}, "
                         "last axis contiguous")
    return x.data_ptr(), s


def _path(tree, path, n_path):
    if path is None:
        return None
    s = path.stride()
    if path.dtype is not torch.int32 or path.dim() != 2 or path.shape[0] != tree.n_seqs or s[1] != 1 or \
            path.shape[1] < tree.max_tokens or path.device != tree.device:
        raise ValueError("path: int32 [session, max_tokens] on the tree's device")
    return _PATH.pack(path.data_ptr(), _dense(n_path, torch.int32, (tree.n_seqs,), "n_path", tree.device), s[0])


def _on_gpu(cache, x, workspace=None):
    """The kernels follow pointers: none to the host, none to another device, scratch as far as it says."""
    device = cache.device
    _need(workspace is None or workspace.is_contiguous(), "workspace: contiguous")
    if not cache.on_gpu and cache.n_seqs or x is not None and x.device != device or \
            workspace is not None and workspace.device != device:
        raise ValueError(f"cache, tree and workspace: on one CUDA device ({device})")


def _elsewhere(device):
    """The library launches on the current device: whether that is another one."""
    return device.index != torch._C._cuda_getDevice()


def _queue(device, stream=None):
    """The raw handle of a call's stream, of its device: the given one, or the current one."""
    if stream is None:
        return 0 if device.index is None else torch._C._cuda_getCurrentRawStream(device.index)
    _need(getattr(stream, "device", device) == device, f"stream: of the tensors' device ({device})")
    return getattr(stream, "cuda_stream", stream)


def _workspace(cache, n, handle):
    """Scratch of n bytes, kept by the cache for each stream: its calls run in
    order.  A captured call has scratch of its own, which the graph holds."""
    if cache.on_gpu and torch._C._cuda_isCurrentStreamCapturing():
        return torch.empty(n, dtype=torch.uint8, device=cache.device)
    w = cache.scratch.get(handle)
    if w is None or w.numel() < n:
        w = cache.scratch[handle] = torch.empty(n, dtype=torch.uint8, device=cache.device)
    return w


def _on(device, stream, call, *args):
    """A call with its device current, on a given stream (torch's, or a raw handle; None: the device's current one):
    what it allocates belongs to that stream."""
    if stream is None:
        with torch.cuda.device(device):
            return call(*args)
    if not isinstance(stream, torch.cuda.Stream):
        raw = getattr(stream, "cuda_stream", stream)
        stream = torch.cuda.ExternalStream(raw, device=device) if raw else torch.cuda.default_stream(device)
    _queue(device, stream)
    with torch.cuda.stream(stream):
        return call(*args)


def attend(cache: Cache, tree: Tree, q, k_new, v_new, scale=None, out=None, lse=None, workspace=None, stream=None):
    """unison_kv_attend: (out [token, q head, head_dim], lse float32 [token, q
    head]).  scale defaults to head_dim ** -0.5; workspace: a uint8 tensor of
    at least ``attend_workspace`` bytes, else the cache keeps one."""
    if cache.on_gpu and (stream is not None or _elsewhere(cache.device)):
        return _on(cache.device, stream, attend, cache, tree, q, k_new, v_new, scale, out, lse, workspace)
    n, heads = tree.n_tokens, q.shape[1]
    qp, qs = _rows(cache, q, n, heads)
    kp, ks = _rows(cache, k_new, n, cache.n_heads)
    vp, vs = _rows(cache, v_new, n, cache.n_heads)
    if out is None:
        out = torch.empty_like(q, memory_format=torch.contiguous_format)
    op, os = _rows(cache, out, n, heads)
    if lse is None:
        lse = torch.empty(n, heads, dtype=torch.float32, device=cache.device)
        lp = lse.data_ptr()
    else:
        lp = _dense(lse, torch.float32, (n, heads), "lse", cache.device)
    _on_gpu(cache, tree, workspace)
    handle = _queue(cache.device)
    if workspace is None:
        workspace = _workspace(cache, attend_workspace(cache, tree, heads), handle)
    rc = lib().unison_kv_attend(
        cache.address, tree.address,
        _STEP.pack(qp, kp, vp, op, lp, 0, qs[0], qs[1], ks[0], ks[1], vs[0], vs[1], os[0], os[1], heads,
                   cache.scale if scale is None else scale),
        workspace.data_ptr(), workspace.numel(), handle)
    if rc:
        binding._check("unison_kv_attend", rc)
    return out, lse


def attend_workspace(cache: Cache, tree: Tree, n_q_heads: int) -> int:
    """Bytes of scratch that attend takes (a function of the sizes and the device alone)."""
    if cache.on_gpu and _elsewhere(cache.device):
        return _on(cache.device, None, attend_workspace, cache, tree, n_q_heads)
    key = tree.max_tokens, n_q_heads
    n = cache.sizes.get(key)
    if n is None:
        n = cache.sizes[key] = int(lib().unison_kv_attend_workspace(cache.address, tree.address, n_q_heads))
    return n


def observe(cache: Cache, tree: Tree, q, lse, k_new, scale=None, path=None, n_path=None, mass_new=None, stream=None):
    """unison_kv_observe: adds to cache.mass; returns mass_new, float32 [token,
    head], the weight of the new tokens themselves."""
    if cache.on_gpu and (stream is not None or _elsewhere(cache.device)):
        return _on(cache.device, stream, observe, cache, tree, q, lse, k_new, scale, path, n_path, mass_new)
    n, heads = tree.n_tokens, q.shape[1]
    qp, qs = _rows(cache, q, n, heads)
    kp, ks = _rows(cache, k_new, n, cache.n_heads)
    lp = _dense(lse, torch.float32, (n, heads), "lse", cache.device)
    _on_gpu(cache, tree)
    if mass_new is None:
        mass_new = torch.empty(n, cache.n_heads, dtype=torch.float32, device=cache.device)
    rc = lib().unison_kv_observe(
        cache.address, tree.address,
        _STEP.pack(qp, kp, 0, 0, lp, _dense(mass_new, torch.float32, (n, cache.n_heads), "mass_new", cache.device),
                   qs[0], qs[1], ks[0], ks[1], 0, 0, 0, 0, heads, cache.scale if scale is None else scale),
        _path(tree, path, n_path), _queue(cache.device))
    if rc:
        binding._check("unison_kv_observe", rc)
    return mass_new


def commit(cache: Cache, tree: Tree, k_new, v_new, mass_new=None, path=None, n_path=None, stream=None) -> None:
    """unison_kv_commit: the accepted tokens go into the pages, length and
    next_pos grow.  Without path every new token is accepted."""
    if cache.on_gpu and _elsewhere(cache.device):
        return _on(cache.device, stream, commit, cache, tree, k_new, v_new, mass_new, path, n_path)
    n = tree.n_tokens
    kp, ks = _rows(cache, k_new, n, cache.n_heads)
    vp, vs = _rows(cache, v_new, n, cache.n_heads)
    mp = _given(mass_new, torch.float32, (n, cache.n_heads), "mass_new", cache.device)
    _on_gpu(cache, tree)
    rc = lib().unison_kv_commit(
        cache.address, tree.address,
        _STEP.pack(0, kp, vp, 0, 0, mp or 0, 0, 0, ks[0], ks[1], vs[0], vs[1], 0, 0, 0, 0.0),
        _path(tree, path, n_path), _queue(cache.device, stream))
    if rc:
        binding._check("unison_kv_commit", rc)


def evict_workspace(cache: Cache) -> int:
    """Bytes of scratch that evict takes (a function of the sizes alone)."""
    n = cache.sizes.get("evict")
    if n is None:
        n = cache.sizes["evict"] = int(lib().unison_kv_evict_workspace(cache.address))
    return n


def evict(cache: Cache, keep, sink=0, recent=0, into: Cache | None = None, workspace=None, stream=None) -> None:
    """unison_kv_evict: at most keep[b] (int32 tensor) slots of each session
    stay, in place or, with ``into``, in another cache."""
    if cache.on_gpu and (stream is not None or _elsewhere(cache.device)):
        return _on(cache.device, stream, evict, cache, keep, sink, recent, into, workspace)
    kp = _dense(keep, torch.int32, (cache.n_seqs,), "keep", cache.device)
    _on_gpu(cache, into, workspace)
    handle = _queue(cache.device)
    if workspace is None:
        workspace = _workspace(cache, evict_workspace(cache), handle)
    rc = lib().unison_kv_evict(cache.address, None if into is None else into.address, kp, sink, recent,
                               workspace.data_ptr(), workspace.numel(), handle)
    if rc:
        binding._check("unison_kv_evict", rc)


def verify(tree: Tree, token, p, q, u, u_sample, path=None, n_path=None, next_token=None, stream=None):
    """unison_kv_verify: (path [session, max_tokens], n_path [session],
    next_token [session]), all int32.  p, q: [token, vocab] probabilities of
    one type (q None: certain drafts); token int32 [token]; u float32 [token];
    u_sample float32 [session]."""
    if p.is_cuda and (stream is not None or _elsewhere(p.device)):
        return _on(p.device, stream, verify, tree, token, p, q, u, u_sample, path, n_path, next_token)
    n, t, total, device = tree.n_seqs, tree.max_tokens, tree.n_tokens, p.device
    dtype, vocab, ps, qs = p.dtype, p.shape[-1], p.stride(), _NO_STRIDES
    ok = dtype in DTYPE and p.shape == (total, vocab) and ps[1] == 1
    if q is not None:
        qs = q.stride()
        ok = ok and q.dtype is dtype and q.shape == (total, vocab) and qs[1] == 1
    _need(ok, "p, q: [token, vocab] of one type, last axis contiguous")
    _need(tree.device == device and (q is None or q.device == device) and (p.is_cuda or n == 0),
          "p, q and the tree: on one CUDA device")
    if path is None:
        path = torch.empty(n, t, dtype=torch.int32, device=device)
    if n_path is None:
        n_path = torch.empty(n, dtype=torch.int32, device=device)
    if next_token is None:
        next_token = torch.empty(n, dtype=torch.int32, device=device)
    s = path.stride()
    _need(path.dtype is torch.int32 and path.dim() == 2 and path.shape[0] == n and path.shape[1] >= t and s[1] == 1 and
          path.device == device, "path: int32 [session, max_tokens] on the device of p")
    rc = lib().unison_kv_verify(
        tree.address,
        _VERIFY.pack(p.data_ptr(), 0 if q is None else q.data_ptr(), ps[0], qs[0],
                     _dense(token, torch.int32, (total,), "token", device),
                     _dense(u, torch.float32, (total,), "u", device),
                     _dense(u_sample, torch.float32, (n,), "u_sample", device), path.data_ptr(),
                     _dense(n_path, torch.int32, (n,), "n_path", device),
                     _dense(next_token, torch.int32, (n,), "next_token", device), s[0], vocab, DTYPE[dtype]),
        _queue(device))
    if rc:
        binding._check("unison_kv_verify", rc)
    return path, n_path, next_token
