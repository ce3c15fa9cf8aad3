"""Orders that the tensor-core kernels of the KV-cache operators rely on, on the
CPU: the events of a kernel's warps and what each of them waits for make a
graph, and a place of a ring may be written again only where every read of it
comes before in that graph, whatever the warps' speeds are.  Ring lengths come
from the sources."""
import graphlib
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


def ring_order(n, turns):
    """Attention: the order of n tiles' keys and values in the ring (kv_attend_tc.cu, item_of)."""
    if not turns or n == 1:
        return [x for t in range(n) for x in (("keys", t), ("values", t))]
    return [("keys", 0)] + [x for t in range(1, n) for x in (("keys", t), ("values", t - 1))] + [("values", n - 1)]


def attend_order(segments, slots, sets):
    """Attention: segments of (query tiles, key tiles).  The roles' events in their programs' order, each with what it
    waits for; `sets`: a segment's copies wait for the one that used its set of flags before (0: they do not)."""
    roles = {"copies": [], "products": [], 0: [], 1: []}
    items, base, joins = [], 0, 0

    def event(role, name, *waits):
        roles[role].append((name, waits))

    for s, (tiles, n) in enumerate(segments):
        turns, at = tiles == 1, lambda t: base + t
        # copies
        waits = [("queries free", s - 1)]
        if sets and s >= sets:
            waits += [("done", s - sets, 0), ("done", s - sets, 1)]
        event("copies", ("queries", s), *waits)
        for what, t in ring_order(n, turns):
            i = len(items)
            event("copies", (what, at(t)), *([("free", *items[i - slots])] if i >= slots else []))
            items.append((what, at(t)))
        event("copies", ("flags", s))

        # products
        def scores(t):
            for q in ([t & 1] if turns else [0, 1]):
                event("products", ("scores", q, at(t)), ("keys", at(t)), ("queries", s))
            event("products", ("free", "keys", at(t)))
            if t == n - 1:
                event("products", ("queries free", s))

        def values(t, q):
            event("products", ("sums", q, at(t)), ("values", at(t)), ("weights", q, at(t)),
                  *([("flags", s)] if t == n - 1 else []))
        if turns:
            for t in range(min(n, 2)):
                scores(t)
            for t in range(n):
                values(t, t & 1)
                event("products", ("free", "values", at(t)))
                if t + 2 < n:
                    scores(t + 2)
        else:
            scores(0)
            for t in range(n):
                for q in (0, 1):
                    values(t, q)
                    if q == 1:
                        event("products", ("free", "values", at(t)))
                    if t + 1 < n:
                        event("products", ("scores", q, at(t + 1)), ("keys", at(t + 1)), ("queries", s))
                        if q == 1:
                            event("products", ("free", "keys", at(t + 1)))
                            if t + 2 == n:
                                event("products", ("queries free", s))
        # weights
        for q in (0, 1):
            mine = range(q, n, 2) if turns else range(n)
            for t in mine:
                owed = q == 1 and t == mine[0] and joins > 0
                event(q, ("weights", q, at(t)), ("scores", q, at(t)), *([("half free", joins - 1)] if owed else []))
            join = turns and n > 1
            if len(mine):
                event(q, ("summed", s, q), ("sums", q, at(mine[-1])))
                if join and q == 1:
                    event(q, ("half", joins))
                else:
                    event(q, ("flags read", s, q), *([("half", joins)] if join else []))
                    if join:
                        event(q, ("half free", joins))
            event(q, ("done", s, q))
        joins += turns and n > 1
        base += n

    deps = {}
    for role in roles.values():
        last = None
        for name, waits in role:
            assert name not in deps
            deps[name] = [w for w in (last, *waits) if w is not None]
            last = name
    for name in deps:
        deps[name] = [w for w in deps[name] if w in deps]
    o = Order()
    for name in graphlib.TopologicalSorter(deps).static_order():  # raises where waits go in a circle
        o.add(name, *deps[name])
    return o


def attend_sequences():
    r = random.Random(2)
    yield from ([(tiles, n)] * 14 for tiles in (1, 2) for n in (1, 2, 3, 6))
    # after a tree over a long context, sessions of few rows that have no cache yet
    yield [(2, 3)] + [(1, 1)] * 12
    yield [(1, 4)] + [(1, 1)] * 12
    for _ in range(40):
        yield [(r.choice((1, 2)), r.choice((1, 1, 1, 2, 5))) for _ in range(16)]


def late_flags(segments, slots, waits, ring):
    o = attend_order(segments, slots, waits)
    return [(s, q) for s in range(len(segments) - ring) for q in (0, 1)
            if ("flags read", s, q) in o.bit and not o.surely(("flags read", s, q), ("flags", s + ring))]


def attend_flags():
    """(sets of flags, how many of them a segment's copies wait for) of the source."""
    text, k = constants("kv_attend_tc.cu")
    assert "odd[kOddSets][4]" in text
    return k["kOddSets"], k["kOddSets"] if "copier.wait(smem_u32(&sh.seg_done[seg_no % kOddSets])" in text else 0


@pytest.mark.parametrize("slots", [5, 8])
def test_attention_reads_a_segments_flags_before_they_are_written_again(slots):
    sets, waits = attend_flags()
    for segments in attend_sequences():
        assert not late_flags(segments, slots, waits, sets), segments


def test_the_order_of_flags_needs_the_wait():
    """Tight rings and program order alone do not do: the statement above says something."""
    sets, _ = attend_flags()
    assert late_flags([(2, 3)] + [(1, 1)] * 12, 8, 0, sets)


@pytest.mark.parametrize("slots", [5, 8])
def test_attention_reads_which_keys_exist_before_that_is_written_again(slots):
    text, _ = constants("kv_attend_tc.cu")
    assert "row_ok[8][4]" in text
    for segments in attend_sequences():
        o, total = attend_order(segments, slots, 0), sum(n for _, n in segments)
        for t in range(total - 8):
            for q in (0, 1):
                if ("weights", q, t) in o.bit:
                    assert o.surely(("weights", q, t), ("keys", t + 8)), (segments, t, q)


@pytest.mark.parametrize("slots", [5, 8])
def test_attentions_sums_are_read_before_the_next_ones_overwrite_them(slots):
    for segments in attend_sequences():
        o, base, readers = attend_order(segments, slots, 0), 0, {0: [], 1: []}
        for s, (tiles, n) in enumerate(segments):
            for q in (0, 1):
                mine = range(q, n, 2) if tiles == 1 else range(n)
                if len(mine):
                    for event in readers[q]:
                        assert o.surely(event, ("sums", q, base + mine[0])), (segments, s, q)
            both = tiles == 1 and n > 1  # the first slot's warps join both
            for q in (0, 1):
                if ("flags read", s, q) in o.bit or both:
                    readers[q] = [("flags read", s, 0 if both else q)]
            base += n
