"""Orders that the tensor-core kernels of the KV-cache operators rely on, on the
CPU: the events of a kernel's warps and what each of them waits for make a
graph, and a place of a ring may be written again only where every read of it
comes before in that graph, whatever the warps' speeds are.  Ring lengths come
from the sources."""
import os
import random
import re

import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2609_09643_gb300", "csrc")


def constants(name):
    """The `constexpr int` values of a source, those that build on each other included."""
    with open(os.path.join(CSRC, name)) as f:
        text = f.read()
    values = {}
    for line in re.findall(r"^constexpr int (k[^;]*);", text, re.M):
        for part in re.sub(r"<[^>]*>", "", line).split(", "):
            key, _, expr = part.partition(" = ")
            try:
                values[key] = eval(expr, {}, dict(values))
            except (NameError, SyntaxError):
                pass  # of template parameters or sizeof
    return text, values


class Order:
    """Events in an order in which they can happen; each knows all that surely came before it."""

    def __init__(self):
        self.before, self.bit = {}, {}

    def add(self, event, *after):
        seen = 0
        for a in after:
            if a in self.before:
                seen |= self.before[a] | 1 << self.bit[a]
        self.bit[event] = len(self.bit)
        self.before[event] = seen

    def surely(self, first, then):
        return bool(self.before[then] >> self.bit[first] & 1)


def observe_order(chunks, slots, buffers):
    """Observation: chunks[t] products of key tile t go through `buffers` places of tensor memory to two groups of
    warps in turn; a tile's accounts are written before its keys are handed on and read by the group that adds up."""
    o, job_of, last = Order(), [], {0: None, 1: None}
    for t, n in enumerate(chunks):
        o.add(("accounts", t), ("accounts", t - 1), ("slot free", t - slots))
        jobs = range(len(job_of), len(job_of) + n)
        first = t & 1 if n & 1 else 0
        for j in jobs:
            o.add(("product", j), ("product", j - 1), ("accounts", t), ("buffer free", j - buffers))
            group = first ^ (j - jobs[0]) & 1
            o.add(("buffer free", j), ("product", j), last[group])
            last[group] = ("buffer free", j)
            job_of.append(t)
        o.add(("slot free", t), ("product", jobs[-1]))
        other = last[1 - first] if n > 1 else None  # its sum
        o.add(("accounts read", t), last[first], other)
        last[first] = ("accounts read", t)
    return o


def late_accounts(chunks, slots, buffers, ring):
    o = observe_order(chunks, slots, buffers)
    return [t for t in range(len(chunks) - ring) if not o.surely(("accounts read", t), ("accounts", t + ring))]


def observe_sequences():
    r = random.Random(1)
    yield from ([n] * 60 for n in range(1, 5))
    yield from ([r.choice(of) for _ in range(80)] for of in ((1, 2), (1, 3), (1, 1, 1, 4), (1, 2, 3, 4)) for _ in range(10))
    for n in (2, 3, 4):  # sessions of few and of many rows follow each other
        yield [1 if t // 7 & 1 else n for t in range(80)]


@pytest.mark.parametrize("slots", [2, 3, 4, 5, 6])
def test_observed_accounts_are_read_before_their_place_is_taken_again(slots):
    text, k = constants("kv_observe_tc.cu")
    assert "marks.next(P.slots + kMoreMarks)" in text and slots <= k["kMostSlots"]
    for chunks in observe_sequences():
        assert not late_accounts(chunks, slots, k["kBuffers"], slots + k["kMoreMarks"]), chunks


def test_the_order_of_accounts_is_tight():
    """One place fewer is too few: the statement above says something."""
    _, k = constants("kv_observe_tc.cu")
    assert late_accounts([1] * 60, 4, k["kBuffers"], 4 + k["kBuffers"] + 1)
