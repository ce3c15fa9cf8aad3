"""Host side of rotation, shared prefixes and sampling (no GPU needed): every
call refuses what its header excludes before anything is queued."""
import pytest
import torch

from kv_reference import Made

ARG, RANGE = -1, -4


@pytest.fixture(scope="module")
def kv():
    from paper_2609_09643_gb300 import native
    native.build()
    from paper_2609_09643_gb300 import kv
    return kv


class _Args:
    """Arguments of every call, on host tensors: a call that is refused never reads them."""

    def __init__(self, kv):
        m = self.m = Made([5, 40], [3, 2], device="cpu")
        pm = self.pm = Made([100], [0], device="cpu", seed=1)
        self.L, self.cache, self.tree = kv.lib(), m.cache(kv), m.tree(kv)
        self.pre_cache = pm.cache(kv)
        self.first = torch.tensor([0, 2], dtype=torch.int32)
        self.prefix = kv.Prefix(self.pre_cache, self.first)
        self.out, self.lse = torch.zeros_like(m.q), torch.zeros(m.q.shape[:2])
        strides = [s for x in (m.q, m.k_new, m.v_new, self.out) for s in x.stride()[:2]]
        self.step = kv.KvStep(*(x.data_ptr() for x in (m.q, m.k_new, m.v_new, self.out, self.lse)), None, *strides,
                              m.q.shape[1], 0.1)
        self.work = torch.zeros(64 << 20, dtype=torch.uint8)
        self.bytes = kv.attend_shared_workspace(self.cache, self.prefix, self.tree, 8)
        self.freq, self.weight = torch.zeros(32), torch.zeros(64, dtype=torch.bfloat16)
        r = [x.data_ptr() for x in (m.q, m.k_new, m.q, m.k_new, self.weight, self.weight, self.freq)]
        self.r = kv.KvRotate(*r, None, *strides[:4], *strides[:4], m.total, 8, 64, 0, 0, 1e-6)
        self.x, self.i = torch.zeros(4, 100), torch.zeros(4, dtype=torch.int32)
        self.p = torch.zeros(4, 100)
        self.s = kv.KvSample(self.x.data_ptr(), self.p.data_ptr(), self.x.data_ptr(), self.i.data_ptr(), None, None, None,
                             None, 100, 100, 4, 100, 2, 2, 1.0, 0, 1.0, 0.0)

    def attend_shared(self):
        return self.L.unison_kv_attend_shared(self.cache.address, self.prefix.address, self.tree.address,
                                              bytes(self.step), self.work.data_ptr(), self.bytes, None)

    def rotate(self):
        return self.L.unison_kv_rotate(self.cache.address, self.tree.address, bytes(self.r), None)

    def sample(self):
        return self.L.unison_kv_sample(bytes(self.s), None)


BOTH = ("attend_shared", "rotate")
REFUSED = [
    # calls, what is changed, expected code
    (BOTH, lambda a: setattr(a.cache.struct, "page_size", 0), RANGE),
    (BOTH, lambda a: setattr(a.cache.struct, "head_dim", 60), RANGE),
    (BOTH, lambda a: setattr(a.cache.struct, "dtype", 2), ARG),
    (BOTH, lambda a: setattr(a.tree.struct, "max_tokens", 65), RANGE),
    (BOTH, lambda a: setattr(a.tree.struct, "offsets", None), ARG),
    (BOTH, lambda a: setattr(a.tree.struct, "n_seqs", 3), ARG),
    (("attend_shared",), lambda a: setattr(a.pre_cache.struct, "page_size", 0), RANGE),
    (("attend_shared",), lambda a: setattr(a.pre_cache.struct, "n_heads", 1), ARG),
    (("attend_shared",), lambda a: setattr(a.pre_cache.struct, "head_dim", 128), ARG),
    (("attend_shared",), lambda a: setattr(a.pre_cache.struct, "dtype", 1), ARG),
    (("attend_shared",), lambda a: setattr(a.pre_cache.struct, "length", None), ARG),
    (("attend_shared",), lambda a: setattr(a.pre_cache.struct, "k", None), ARG),
    (("attend_shared",), lambda a: setattr(a.pre_cache.struct, "v_slot", 12), ARG),
    (("attend_shared",), lambda a: setattr(a.prefix.struct, "first", None), ARG),
    (("attend_shared",), lambda a: setattr(a.prefix.struct, "cache", None), ARG),
    (("attend_shared",), lambda a: setattr(a.cache.struct, "v", None), ARG),
    (("attend_shared",), lambda a: setattr(a.step, "n_q_heads", 7), RANGE),
    (("attend_shared",), lambda a: setattr(a.step, "q", None), ARG),
    (("attend_shared",), lambda a: setattr(a.step, "out_head", 4), ARG),
    (("attend_shared",), lambda a: setattr(a.tree.struct, "n_tokens", 1 << 28), RANGE),
    (("attend_shared",), lambda a: setattr(a, "bytes", a.bytes - 16), ARG),
    (("rotate",), lambda a: setattr(a.cache.struct, "next_pos", None), ARG),
    (("rotate",), lambda a: setattr(a.r, "n_tokens", 4), ARG),
    (("rotate",), lambda a: setattr(a.r, "rot_dim", 66), RANGE),
    (("rotate",), lambda a: setattr(a.r, "rot_dim", 31), RANGE),
    (("rotate",), lambda a: setattr(a.r, "rot_dim", -2), RANGE),
    (("rotate",), lambda a: setattr(a.r, "eps", -1.0), RANGE),
    (("rotate",), lambda a: setattr(a.r, "eps", float("nan")), RANGE),
    (("rotate",), lambda a: setattr(a.r, "n_q_heads", -1), RANGE),
    (("rotate",), lambda a: setattr(a.r, "q", None), ARG),
    (("rotate",), lambda a: setattr(a.r, "k_out", a.r.k_out + 2), ARG),
    (("rotate",), lambda a: setattr(a.r, "k_head", 4), ARG),
    (("rotate",), lambda a: setattr(a.r, "inv_freq", None), ARG),
    (("rotate",), lambda a: setattr(a.r, "weight_dtype", 1), ARG),
    (("rotate",), lambda a: setattr(a.r, "q_weight", a.r.q_weight + 2), ARG),
    (("sample",), lambda a: setattr(a.s, "vocab", 0), RANGE),
    (("sample",), lambda a: setattr(a.s, "vocab", (1 << 22) + 1), RANGE),
    (("sample",), lambda a: setattr(a.s, "n_rows", -1), RANGE),
    (("sample",), lambda a: setattr(a.s, "n_rows", (1 << 27) + 1), RANGE),
    (("sample",), lambda a: setattr(a.s, "dtype", 3), ARG),
    (("sample",), lambda a: setattr(a.s, "p_dtype", -1), ARG),
    (("sample",), lambda a: setattr(a.s, "logits", None), ARG),
    (("sample",), lambda a: setattr(a.s, "u", None), ARG),
    (("sample",), lambda a: setattr(a.s, "token", None), ARG),
    (("sample",), lambda a: setattr(a.s, "p", a.s.logits), ARG),
    (("sample",), lambda a: setattr(a.s, "p_row", 99), ARG),
    (("rotate",), lambda a: (setattr(a.r, "position", a.r.inv_freq), setattr(a.r, "n_tokens", 1 << 25)), RANGE),
    (("sample",), lambda a: (setattr(a.s, "token", None), setattr(a.s, "u", None), setattr(a.s, "p", None)), ARG),
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
    assert L.unison_kv_rotate(None, a.tree.address, bytes(a.r), None) == ARG
    assert L.unison_kv_rotate(a.cache.address, None, bytes(a.r), None) == ARG
    assert L.unison_kv_rotate(a.cache.address, a.tree.address, None, None) == ARG
    assert L.unison_kv_sample(None, None) == ARG
    for args in ((None, a.prefix.address, a.tree.address), (a.cache.address, None, a.tree.address),
                 (a.cache.address, a.prefix.address, None)):
        assert L.unison_kv_attend_shared(*args, bytes(a.step), a.work.data_ptr(), a.bytes, None) == ARG
        assert L.unison_kv_attend_shared_workspace(*args, 8) == 0
    assert L.unison_kv_attend_shared(a.cache.address, a.prefix.address, a.tree.address, None, a.work.data_ptr(), a.bytes,
                                     None) == ARG


def test_empty_calls_do_nothing(kv):
    m = Made([], [], device="cpu")
    cache, tree = m.cache(kv), m.tree(kv)
    prefix = kv.Prefix(Made([], [], device="cpu").cache(kv), torch.zeros(1, dtype=torch.int32))
    kv.rotate(cache, tree, m.q, m.k_new, torch.zeros(32))
    kv.rotate(cache, None, m.q, m.k_new, torch.zeros(32), position=torch.zeros(0, dtype=torch.int32))
    kv.attend_shared(cache, prefix, tree, m.q, m.k_new, m.v_new)
    assert kv.sample(torch.zeros(0, 10), torch.zeros(0)).shape == (0,)
    assert kv.probabilities(torch.zeros(0, 10)).shape == (0, 10)


def test_binding_refuses_other_types_shapes_and_places(kv):
    m, pm = Made([5, 40], [3, 2], device="cpu"), Made([9], [0], device="cpu")
    cache, tree = m.cache(kv), m.tree(kv)
    prefix = kv.Prefix(pm.cache(kv), torch.zeros(2, dtype=torch.int32))
    f = torch.zeros(32)
    pos = torch.zeros(5, dtype=torch.int32)
    bad = [
        lambda: kv.Prefix(pm.cache(kv), torch.zeros(2)),
        lambda: kv.Prefix(pm.cache(kv), torch.zeros(3, dtype=torch.int32)),
        lambda: kv.attend_shared(cache, prefix, tree, m.q, m.k_new, m.v_new),  # on the host
        lambda: kv.attend_shared(cache, prefix, tree, m.q.half(), m.k_new, m.v_new),
        lambda: kv.rotate(cache, tree, m.q, m.k_new, f),  # on the host
        lambda: kv.rotate(cache, None, m.q, m.k_new, f),  # no positions
        lambda: kv.rotate(cache, None, m.q, m.k_new, f, position=pos.long()),
        lambda: kv.rotate(cache, None, m.q, m.k_new, f, position=pos[:4]),
        lambda: kv.rotate(cache, None, m.q, m.k_new[:4], f, position=pos),
        lambda: kv.rotate(cache, tree, m.q, m.k_new, f.double()),
        lambda: kv.rotate(cache, tree, m.q, m.k_new, f, q_weight=torch.zeros(64, dtype=torch.float16)),
        lambda: kv.rotate(cache, tree, m.q, m.k_new, f, q_weight=torch.zeros(64), k_weight=torch.zeros(64).bfloat16()),
        lambda: kv.rotate(cache, tree, m.q, m.k_new, f, k_weight=torch.zeros(32)),
        lambda: kv.rotate(cache, tree, m.q, m.k_new, f, q_out=torch.zeros(5, 8, 64)),
        lambda: kv.sample(torch.zeros(2, 10), torch.zeros(2)),  # on the host
        lambda: kv.sample(torch.zeros(10), torch.zeros(1)),
        lambda: kv.sample(torch.zeros(2, 10).double(), torch.zeros(2)),
        lambda: kv.sample(torch.zeros(10, 2).T, torch.zeros(2)),
        lambda: kv.sample(torch.zeros(0, 10), torch.zeros(1)),
        lambda: kv.sample(torch.zeros(0, 10), None),
        lambda: kv.sample(torch.zeros(0, 10), torch.zeros(0), top_k=torch.zeros(0)),
        lambda: kv.sample(torch.zeros(0, 10), torch.zeros(0), temperature=torch.zeros(1)),
        lambda: kv.sample(torch.zeros(0, 10), torch.zeros(0), p=torch.zeros(0, 11)),
        lambda: kv.sample(torch.zeros(0, 10), torch.zeros(0), token=torch.zeros(0)),
        lambda: kv.probabilities(torch.zeros(0, 10), p=torch.zeros(0, 10).double()),
    ]
    for i, call in enumerate(bad):
        with pytest.raises(ValueError):
            call()
            print("not refused:", i)


def test_every_kernel_waits_before_anything_else():
    """A kernel is set up while the one before it on the stream ends.  What that one wrote, and what those before it
    wrote, is promised to be seen only behind a wait of the kernel's own: it comes first in all of them."""
    import os
    import re
    from paper_2609_09643_gb300 import native
    seen = 0
    for name in native.SOURCES:
        if not name.startswith("kv_"):
            continue
        with open(os.path.join(native.CSRC, name)) as f:
            text = re.sub(r"//[^\n]*", "", f.read())
        for at in re.finditer(r"__global__", text):
            body = text[text.index("{", at.start()) + 1:]
            assert body.split(None, 1)[0] == "follow_last_kernel();", (name, body[:80])
            seen += 1
    assert seen >= 12


def test_a_cache_keeps_a_bounded_list_of_sizes(kv):
    m, pm = Made([5, 40], [3, 2], device="cpu"), Made([100], [0], device="cpu")
    cache, prefix = m.cache(kv), kv.Prefix(pm.cache(kv), torch.tensor([0, 2], dtype=torch.int32))
    offsets = torch.zeros(3, dtype=torch.int32)
    for n in range(1, 2000):  # drafts of differing size: every step has another number of tokens
        tree = kv.Tree(offsets, 64, n_tokens=n)
        size = kv.attend_shared_workspace(cache, prefix, tree, 8)
        assert size > 0 and size == kv.attend_shared_workspace(cache, prefix, tree, 8)
    assert len(cache.sizes) <= 256
