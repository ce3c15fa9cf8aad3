"""Host side of the KV-cache operators (no GPU needed): every declared symbol
is exported, and every call refuses what its header excludes before anything
is queued."""
import ctypes as C
import types

import pytest
import torch

from kv_reference import Made
from test_abi import declared_symbols


@pytest.fixture(scope="module")
def kv():
    from paper_2609_09643_gb300 import native
    native.build()
    from paper_2609_09643_gb300 import kv
    return kv


def test_declared_symbols_are_exported(kv):
    lib = C.CDLL(kv.binding.lib_path())
    decl = [s for s in declared_symbols("unison_kv.h")]
    assert decl == sorted(kv.EXPORTS)
    for name in decl:
        assert hasattr(lib, name), name


def _made(**kw):
    return Made([5, 40], [3, 2], device="cpu", **kw)


class _Args:
    """Arguments of every call, on host tensors: a call that is refused never reads them."""

    def __init__(self, kv):
        m = self.m = _made()
        self.kv, self.L = kv, kv.lib()
        self.cache, self.tree = m.cache(kv), m.tree(kv)
        self.into = _made().cache(kv)
        self.out, self.lse = torch.zeros_like(m.q), torch.zeros(m.q.shape[:2])
        self.mass_new = torch.zeros(m.total, m.hkv)
        strides = [s for x in (m.q, m.k_new, m.v_new, self.out) for s in x.stride()[:2]]
        self.step = kv.KvStep(*(x.data_ptr() for x in (m.q, m.k_new, m.v_new, self.out, self.lse, self.mass_new)),
                              *strides, m.q.shape[1], 0.1)
        self.path_t = torch.zeros(2, 3, dtype=torch.int32)
        self.path = kv.KvPath(self.path_t.data_ptr(), self.path_t.data_ptr(), 3)
        self.work = torch.zeros(64 << 20, dtype=torch.uint8)
        self.bytes = self.work.numel()
        self.keep = torch.zeros(2, dtype=torch.int32).data_ptr()
        self.sink = self.recent = 0
        p = torch.zeros(m.total, 100)
        i = torch.zeros(64, dtype=torch.int32)
        self.hold = (p, i)
        self.v = kv.KvVerify(p.data_ptr(), p.data_ptr(), 100, 100, i.data_ptr(), i.data_ptr(), i.data_ptr(),
                             i.data_ptr(), i.data_ptr(), i.data_ptr(), 3, 100, 2)

    def attend(self):
        return self.L.unison_kv_attend(self.cache.address, self.tree.address, bytes(self.step), self.work.data_ptr(),
                                       self.bytes, None)

    def observe(self):
        return self.L.unison_kv_observe(self.cache.address, self.tree.address, bytes(self.step), bytes(self.path), None)

    def commit(self):
        return self.L.unison_kv_commit(self.cache.address, self.tree.address, bytes(self.step), bytes(self.path), None)

    def evict(self):
        return self.L.unison_kv_evict(self.cache.address, self.into.address, self.keep, self.sink, self.recent,
                                      self.work.data_ptr(), self.bytes, None)

    def verify(self):
        return self.L.unison_kv_verify(self.tree.address, bytes(self.v), None)


ARG, RANGE = -1, -4
CACHE = ("attend", "observe", "commit", "evict")
STEP = ("attend", "observe", "commit")
REFUSED = [
    # calls, what is changed, expected code
    (CACHE, lambda a: setattr(a.cache.struct, "page_size", 0), RANGE),
    (CACHE, lambda a: setattr(a.cache.struct, "n_seqs", -1), RANGE),
    (CACHE, lambda a: setattr(a.cache.struct, "n_heads", 0), RANGE),
    (CACHE, lambda a: setattr(a.cache.struct, "head_dim", 60), RANGE),
    (CACHE, lambda a: setattr(a.cache.struct, "head_dim", 264), RANGE),
    (CACHE, lambda a: setattr(a.cache.struct, "max_pages", 1 << 28), RANGE),
    (CACHE, lambda a: setattr(a.cache.struct, "dtype", 2), ARG),
    (CACHE, lambda a: setattr(a.cache.struct, "length", None), ARG),
    (CACHE, lambda a: setattr(a.cache.struct, "page_table", None), ARG),
    (CACHE, lambda a: setattr(a.cache.struct, "k", None), ARG),
    (CACHE, lambda a: setattr(a.cache.struct, "k", a.cache.struct.k + 8), ARG),
    (CACHE, lambda a: setattr(a.cache.struct, "k_slot", 12), ARG),
    (("attend", "commit", "evict"), lambda a: setattr(a.cache.struct, "v_head", 4), ARG),
    (("observe", "evict"), lambda a: setattr(a.cache.struct, "mass", None), ARG),
    ((*STEP, "verify"), lambda a: setattr(a.tree.struct, "max_tokens", 65), RANGE),
    ((*STEP, "verify"), lambda a: setattr(a.tree.struct, "max_tokens", 0), RANGE),
    ((*STEP, "verify"), lambda a: setattr(a.tree.struct, "n_tokens", -1), RANGE),
    ((*STEP, "verify"), lambda a: setattr(a.tree.struct, "offsets", None), ARG),
    (STEP, lambda a: setattr(a.tree.struct, "n_seqs", 3), ARG),
    (("attend", "observe"), lambda a: setattr(a.step, "n_q_heads", 7), RANGE),
    (("attend", "observe"), lambda a: setattr(a.step, "n_q_heads", 2 * 65), RANGE),
    (("attend", "observe"), lambda a: setattr(a.step, "n_q_heads", 0), RANGE),
    (("attend", "observe"), lambda a: setattr(a.step, "q", None), ARG),
    (("attend", "observe"), lambda a: setattr(a.step, "q_token", 4), ARG),
    (("attend", "commit"), lambda a: setattr(a.step, "v_new", None), ARG),
    (STEP, lambda a: setattr(a.step, "k_new", a.step.k_new + 2), ARG),
    (("attend",), lambda a: setattr(a.step, "out", None), ARG),
    (("observe",), lambda a: setattr(a.step, "lse", None), ARG),
    (("observe", "commit"), lambda a: setattr(a.path, "n_path", None), ARG),
    (("attend", "evict"), lambda a: setattr(a, "bytes", 16), ARG),
    (("evict",), lambda a: setattr(a, "keep", None), ARG),
    (("evict",), lambda a: setattr(a, "sink", -1), RANGE),
    (("evict",), lambda a: setattr(a, "recent", -1), RANGE),
    (("evict",), lambda a: setattr(a.into.struct, "head_dim", 128), ARG),
    (("evict",), lambda a: setattr(a.into.struct, "n_heads", 1), ARG),
    (("evict",), lambda a: setattr(a.into.struct, "v", None), ARG),
    (("verify",), lambda a: setattr(a.v, "vocab", 0), RANGE),
    (("verify",), lambda a: setattr(a.v, "vocab", (1 << 22) + 1), RANGE),
    (("verify",), lambda a: setattr(a.v, "dtype", 3), ARG),
    (("verify",), lambda a: setattr(a.v, "path_stride", 2), ARG),
    (("verify",), lambda a: setattr(a.v, "u", None), ARG),
    (("verify",), lambda a: setattr(a.v, "next_token", None), ARG),
    (("verify",), lambda a: setattr(a.tree.struct, "parent", None), ARG),
]


@pytest.mark.parametrize("i", range(len(REFUSED)))
def test_refusals(kv, i):
    calls, change, code = REFUSED[i]
    for call in calls:
        a = _Args(kv)
        change(a)
        assert getattr(a, call)() == code, call


def test_null_structs_are_refused(kv):
    a, L = _Args(kv), kv.lib()
    assert L.unison_kv_attend(None, a.tree.address, bytes(a.step), a.work.data_ptr(), a.bytes, None) == ARG
    assert L.unison_kv_attend(a.cache.address, None, bytes(a.step), a.work.data_ptr(), a.bytes, None) == ARG
    assert L.unison_kv_attend(a.cache.address, a.tree.address, None, a.work.data_ptr(), a.bytes, None) == ARG
    assert L.unison_kv_observe(a.cache.address, a.tree.address, None, None, None) == ARG
    assert L.unison_kv_commit(a.cache.address, a.tree.address, None, None, None) == ARG
    assert L.unison_kv_evict(None, None, a.keep, 0, 0, a.work.data_ptr(), a.bytes, None) == ARG
    assert L.unison_kv_verify(None, bytes(a.v), None) == ARG
    assert L.unison_kv_verify(a.tree.address, None, None) == ARG
    assert L.unison_kv_attend_workspace(None, None, 8) == 0
    assert L.unison_kv_evict_workspace(None) == 0


def test_binding_refuses_other_types_and_shapes(kv):
    m = _made()
    cache, tree = m.cache(kv), m.tree(kv)
    for bad in (m.q.float(), m.q[:, :, :32], m.q[:2], m.q.transpose(1, 2)):
        with pytest.raises(ValueError):
            kv.attend(cache, tree, bad, m.k_new, m.v_new, stream=0)
    with pytest.raises(ValueError):
        kv.attend(cache, tree, m.q, m.k_new[:, :1], m.v_new, stream=0)
    with pytest.raises(ValueError):
        kv.Cache(m.k, m.v.half(), m.page_table, m.length)
    with pytest.raises(ValueError):
        kv.Cache(m.k, m.v, m.page_table.long(), m.length)
    with pytest.raises(ValueError):
        kv.Cache(m.k, m.v, m.page_table, m.length, mass=m.mass.double())
    with pytest.raises(ValueError):
        kv.Tree(m.offsets, 3)
    with pytest.raises(ValueError):
        kv.Tree(m.offsets, 3, mask=m.mask.int())
    with pytest.raises(ValueError):
        kv.evict(cache, torch.zeros(3, dtype=torch.int32), stream=0)
    p = torch.zeros(m.total, 10)
    i = torch.zeros(m.total, dtype=torch.int32)
    with pytest.raises(ValueError):
        kv.verify(tree, i, p, p.half(), torch.zeros(m.total), torch.zeros(2), stream=0)
    with pytest.raises(ValueError):
        kv.verify(tree, i.long(), p, p, torch.zeros(m.total), torch.zeros(2), stream=0)


def test_empty_batches_do_nothing(kv):
    m = Made([], [], device="cpu")
    cache, tree = m.cache(kv), m.tree(kv)
    kv.attend(cache, tree, m.q, m.k_new, m.v_new, stream=0)
    kv.observe(cache, tree, m.q, torch.zeros(0, 8), m.k_new, stream=0)
    kv.commit(cache, tree, m.k_new, m.v_new, stream=0)
    kv.evict(cache, torch.zeros(0, dtype=torch.int32), stream=0)
    i = torch.zeros(0, dtype=torch.int32)
    kv.verify(tree, i, torch.zeros(0, 10), None, torch.zeros(0), torch.zeros(0), stream=0)


def test_room_of_a_page_table_is_limited(kv):
    cache = _made().cache(kv)
    cache.struct.page_size = 1 << 15
    for pages, fits in (((1 << 16) - 3, True), ((1 << 16) - 2, False)):
        cache.struct.max_pages = pages
        assert (kv.lib().unison_kv_evict_workspace(cache.address) > 0) == fits


@pytest.mark.parametrize("d", [64, 128, 256])
@pytest.mark.parametrize("group,tokens", [(1, 1), (2, 16), (4, 64), (12, 64)])
def test_scratch_is_whole_pieces_of_16_bytes(kv, d, group, tokens):
    """For any number of multiprocessors (without a GPU: one), so that what lies
    behind the first records is aligned where their number is odd, too."""
    m = _made(d=d, group=group)
    tree = kv.Tree(m.offsets, tokens, mask=m.mask)
    assert kv.attend_workspace(m.cache(kv), tree, m.q.shape[1]) % 16 == 0


class _There(torch.Tensor):
    """A host tensor that says it is on the second GPU."""
    device = property(lambda self: torch.device("cuda", 1))
    is_cuda = property(lambda self: True)


def _calls_there(kv):
    """Every call on tensors of the second GPU, outputs and scratch given; the last one asks for the scratch's size."""
    there = lambda x: x.as_subclass(_There)  # noqa: E731
    zeros = lambda *s, dtype=torch.float32: there(torch.zeros(s, dtype=dtype))  # noqa: E731
    ints = lambda *s: zeros(*s, dtype=torch.int32)  # noqa: E731
    m = _made()
    for name, x in vars(m).items():
        if isinstance(x, torch.Tensor):
            setattr(m, name, there(x))
    cache, tree, n, heads = m.cache(kv), m.tree(kv), m.total, m.q.shape[1]
    out, lse, new = there(torch.zeros_like(m.q)), zeros(n, heads), zeros(n, m.hkv)
    work = zeros(1 << 20, dtype=torch.uint8)
    p = zeros(n, 10)
    return [
        lambda **kw: kv.attend(cache, tree, m.q, m.k_new, m.v_new, out=out, lse=lse, workspace=work, **kw),
        lambda **kw: kv.observe(cache, tree, m.q, lse, m.k_new, mass_new=new, **kw),
        lambda **kw: kv.commit(cache, tree, m.k_new, m.v_new, **kw),
        lambda **kw: kv.evict(cache, ints(2), workspace=work, **kw),
        lambda **kw: kv.verify(tree, ints(n), p, p, zeros(n), zeros(2), path=ints(2, 3), n_path=ints(2),
                               next_token=ints(2), **kw),
        lambda: kv.attend_workspace(cache, tree, heads)]


def test_calls_run_on_the_device_of_their_tensors(kv, monkeypatch):
    """The library launches on the current device: with another one current, a
    call makes its tensors' device current, and puts the other one back."""
    current, seen = [0], []

    class On:
        def __init__(self, device):
            self.index = torch.device(device).index

        def __enter__(self):
            self.last, current[0] = current[0], self.index

        def __exit__(self, *_):
            current[0] = self.last

    class Library:
        def __getattr__(self, name):
            return lambda *args: seen.append((name, current[0])) or 0

    monkeypatch.setattr(torch._C, "_cuda_getDevice", lambda: current[0])
    monkeypatch.setattr(torch.cuda, "device", On)
    monkeypatch.setattr(torch._C, "_cuda_getCurrentRawStream", lambda index: 0)
    monkeypatch.setattr(kv, "lib", Library)
    for first in (0, 1):
        current[0] = first
        for call in _calls_there(kv):
            call()
            assert current == [first]
    names = [f"unison_kv_{x}" for x in ("attend", "observe", "commit", "evict", "verify", "attend_workspace")]
    assert seen == [(x, 1) for x in names * 2]

    class Stream:  # of the first GPU
        device, cuda_stream = torch.device("cuda", 0), 7

    monkeypatch.setattr(torch.cuda, "Stream", Stream)
    del seen[:]
    for call in _calls_there(kv)[:-1]:
        with pytest.raises(ValueError, match="stream"):
            call(stream=Stream())
    assert not seen


def test_binding_refuses_calls_without_a_wanted_tensor(kv, monkeypatch):
    there = lambda x: x.as_subclass(_There)  # noqa: E731
    zeros = lambda *s, dtype=torch.float32: there(torch.zeros(s, dtype=dtype))  # noqa: E731
    m = _made()
    for name, x in vars(m).items():
        if isinstance(x, torch.Tensor):
            setattr(m, name, there(x))
    monkeypatch.setattr(torch._C, "_cuda_getDevice", lambda: 1)
    monkeypatch.setattr(torch._C, "_cuda_getCurrentRawStream", lambda index: 0)
    sizes = {"unison_kv_evict_workspace": lambda cache: 16}  # every other function is not to be called
    monkeypatch.setattr(kv, "lib", lambda: types.SimpleNamespace(
        **{x: lambda *_: pytest.fail("called") for x in kv.EXPORTS} | sizes))
    cache, tree, n = m.cache(kv), m.tree(kv), m.total
    path, lse, new = zeros(2, 3, dtype=torch.int32), zeros(n, 8), zeros(n, 2)
    p, i, u, us, two = zeros(n, 10), zeros(n, dtype=torch.int32), zeros(n), zeros(2), zeros(2, dtype=torch.int32)
    outs = dict(path=path, n_path=two, next_token=two)
    for name, call in (("n_path", lambda: kv.observe(cache, tree, m.q, lse, m.k_new, path=path, mass_new=new)),
                       ("n_path", lambda: kv.commit(cache, tree, m.k_new, m.v_new, path=path)),
                       ("lse", lambda: kv.observe(cache, tree, m.q, None, m.k_new, mass_new=new)),
                       ("keep", lambda: kv.evict(cache, None)),
                       ("token", lambda: kv.verify(tree, None, p, p, u, us, **outs)),
                       ("u", lambda: kv.verify(tree, i, p, p, None, us, **outs)),
                       ("u_sample", lambda: kv.verify(tree, i, p, p, u, None, **outs)),
                       ("length", lambda: kv.Cache(m.k, m.v, m.page_table, None))):
        with pytest.raises(ValueError, match=rf"^{name}:"):
            call()


@pytest.mark.parametrize("bad", [lambda n: torch.zeros(1, dtype=torch.uint8).expand(n),
                                 lambda n: torch.zeros(2 * n, dtype=torch.uint8)[::2]])
def test_binding_refuses_scratch_with_gaps(kv, bad):
    """Elements are not bytes in a row there: an expanded tensor's are one byte."""
    m = _made()
    cache, tree, n = m.cache(kv), m.tree(kv), 1 << 20
    keep = torch.zeros(2, dtype=torch.int32)
    for call in (lambda w: kv.attend(cache, tree, m.q, m.k_new, m.v_new, workspace=w),
                 lambda w: kv.evict(cache, keep, workspace=w)):
        with pytest.raises(ValueError, match="contiguous"):
            call(bad(n))
        with pytest.raises(ValueError, match="CUDA"):  # this one is refused for being on the host alone
            call(torch.zeros(n, dtype=torch.uint8))


def test_binding_refuses_the_host_and_other_devices(kv):
    """Kernels follow pointers, so a tensor elsewhere is refused before any launch."""
    m = _made()
    cache, tree = m.cache(kv), m.tree(kv)
    p, i = torch.zeros(m.total, 10), torch.zeros(m.total, dtype=torch.int32)
    lse, keep = torch.zeros(m.total, m.q.shape[1]), torch.zeros(2, dtype=torch.int32)
    for call in (lambda: kv.attend(cache, tree, m.q, m.k_new, m.v_new, stream=0),
                 lambda: kv.observe(cache, tree, m.q, lse, m.k_new, stream=0),
                 lambda: kv.commit(cache, tree, m.k_new, m.v_new, stream=0),
                 lambda: kv.evict(cache, keep, stream=0),
                 lambda: kv.verify(tree, i, p, p, torch.zeros(m.total), torch.zeros(2), stream=0)):
        with pytest.raises(ValueError, match="CUDA"):
            call()
    there = lambda x: torch.empty_like(x, device="meta")  # noqa: E731
    for call in (lambda: kv.Cache(m.k, there(m.v), m.page_table, m.length),
                 lambda: kv.Cache(m.k, m.v, there(m.page_table), m.length),
                 lambda: kv.Cache(m.k, m.v, m.page_table, there(m.length)),
                 lambda: kv.Cache(m.k, m.v, m.page_table, m.length, mass=there(m.mass)),
                 lambda: kv.Tree(m.offsets, 3, mask=there(m.mask)),
                 lambda: kv.attend(cache, tree, there(m.q), m.k_new, m.v_new, stream=0),
                 lambda: kv.evict(cache, there(keep), stream=0)):
        with pytest.raises(ValueError, match="device| on "):
            call()
