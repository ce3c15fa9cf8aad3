"""The KV-cache operators this framework is timed on.

One serving step over the paged cache of agent sessions: attention of new
tokens (one, a chain or a tree of drafts) over the cache, verification of the
drafts, accumulation of the attention weight that every cached token gets,
commitment of the accepted tokens to the pages, and eviction of the least
attended tokens, in place or into another tier's cache.

With ``own`` false the operators run in their plain form (elementary torch
operations, 32-bit arithmetic); with ``own`` true they are the framework's.
"""
from __future__ import annotations

import math

import torch

own = False

TYPES = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}
FIX = 2.0 ** 40  # probabilities are summed and inverted as whole multiples of 2^-40


def listed():
    gqa = dict(hq=32, hkv=8, d=128, dtype="bf16", layout="hnd")
    return [
        # One agent's next token over a short context: the latency of a call.
        dict(gqa, name="attend-one", kind="attend", seqs=1, len_lo=2100, len_hi=2100, tokens=1, ragged=0, page=16),
        # A decode step of a serving batch: contexts from a first turn to a long session.
        dict(gqa, name="attend-batch", kind="attend", seqs=64, len_lo=512, len_hi=32768, tokens=1, ragged=0, page=64),
        # Two very long agent sessions with a small draft tree, slots outside heads, half precision.
        dict(gqa, name="attend-long", kind="attend", seqs=2, len_lo=131071, len_hi=131071, tokens=8, ragged=0, page=128,
             layout="nhd", dtype="fp16"),
        # A small model: odd head size, group and page, drafts of differing size, sessions that have no cache yet.
        dict(name="attend-odd", kind="attend", seqs=37, len_lo=0, len_hi=5001, tokens=13, ragged=1, page=24, hq=14,
             hkv=2, d=96, dtype="bf16", layout="nhd"),
        # Large draft trees for a batch: 64 nodes x 8 heads read every cached key.
        dict(gqa, name="attend-tree", kind="attend", seqs=32, len_lo=15000, len_hi=16384, tokens=64, ragged=0, page=64,
             hq=64),
        # After a decode step: the weights of up to four accepted tokens of eight drafted.
        dict(gqa, name="observe-step", kind="observe", seqs=64, len_lo=512, len_hi=32768, tokens=8, accepted=4, page=64),
        # Before a large eviction: an observation window of 64 tokens over long contexts.
        dict(gqa, name="observe-window", kind="observe", seqs=16, len_lo=8192, len_hi=32768, tokens=64, accepted=64,
             page=64, hq=64),
        # One session at its budget: commit the accepted tokens, evict as many.
        dict(name="step-one", kind="step", seqs=1, keep=1000, tokens=5, page=16, hkv=2, d=128, dtype="bf16",
             layout="hnd"),
        # A serving batch at its budgets.
        dict(name="step-batch", kind="step", seqs=64, keep=4096, tokens=8, page=64, hkv=8, d=128, dtype="bf16",
             layout="hnd"),
        # Demotion of sessions to another tier with a quarter of their tokens.
        dict(name="demote", kind="demote", seqs=16, len_lo=8192, len_hi=32768, keep=8192, page=64, hkv=8, d=128,
             dtype="bf16", layout="hnd"),
        # One session's chain of four drafts.
        dict(name="verify-one", kind="verify", seqs=1, tokens=5, vocab=32000, tree=0, dtype="fp32"),
        # Draft trees of a serving batch over a large vocabulary.
        dict(name="verify-batch", kind="verify", seqs=128, tokens=32, vocab=128000, tree=1, dtype="fp32"),
    ]


def _log_int(rng, lo, hi):
    x = int(round(2.0 ** rng.uniform(math.log2(lo), math.log2(hi))))
    return x - 1 if x == 3 << 10 else x


def draw(rng):
    kind = rng.choice(["attend", "attend", "observe", "step", "demote", "verify"])
    if kind == "verify":
        seqs, tokens, vocab = _log_int(rng, 1, 128), _log_int(rng, 1, 32), _log_int(rng, 1000, 128000)
        vocab = vocab // 64 * 64 - 64 * (vocab // 64 == 48) if rng.random() < 0.5 else vocab
        return dict(kind=kind, seqs=seqs, tokens=tokens, vocab=vocab, tree=rng.randint(0, 1),
                    dtype=rng.choice(["fp32", "fp32", "bf16", "fp16"]))
    shape = dict(kind=kind, page=rng.choice([8, 16, 24, 32, 64, 100, 128]), dtype=rng.choice(["bf16", "fp16"]),
                 d=rng.choice([64, 96, 128, 128, 128]), layout=rng.choice(["hnd", "nhd"]), hkv=rng.choice([1, 2, 4, 8]))
    if kind == "step":
        return dict(shape, seqs=_log_int(rng, 1, 64), keep=_log_int(rng, 100, 4096), tokens=rng.randint(1, 8))
    len_hi = _log_int(rng, 100, 131072)
    len_lo = rng.choice([0, 1, len_hi // 8, len_hi])
    seqs = max(1, min(_log_int(rng, 1, 64), (64 << 13) // len_hi))
    if kind == "demote":
        return dict(shape, seqs=seqs, len_lo=len_lo, len_hi=len_hi, keep=_log_int(rng, 10, max(11, len_hi)))
    tokens = rng.choice([1, 1, 2, 5, 8, 13, 32, 64])
    hq = shape["hkv"] * rng.choice([1, 3, 4, 7, 8])
    if kind == "observe":
        return dict(shape, seqs=seqs, len_lo=len_lo, len_hi=len_hi, tokens=tokens, accepted=rng.randint(1, tokens),
                    hq=hq)
    return dict(shape, seqs=seqs, len_lo=len_lo, len_hi=len_hi, tokens=tokens, ragged=rng.randint(0, 1), hq=hq)


# ----------------------------------------------------------------- inputs --
def _lengths(case):
    """Cached tokens of each session: spread evenly over the logarithm, odd (they end inside pages and tiles)."""
    n, lo, hi = case["seqs"], case["len_lo"], case["len_hi"]
    base = max(lo, 1)
    lens = [int(round(base * (hi / base) ** (i / max(n - 1, 1)))) if hi > base else hi for i in range(n)]
    if lo == 0 and n > 1:
        lens[0] = 0
    return [x | 1 if x else 0 for x in lens]


def _counts(case):
    """New tokens of each session."""
    n, t = case["seqs"], case["tokens"]
    return [1 + (5 * i + 2) % t for i in range(n)] if case.get("ragged") else [t] * n


def _accepted(case):
    return [1 + (3 * i + case["accepted"] - 1) % case["accepted"] for i in range(case["seqs"])]


def _pool(g, n_pages, case):
    """K or V of all pages, [page, head, slot, dim] as a view of either layout."""
    p, h, s, d = n_pages, case["hkv"], case["page"], case["d"]
    shape = (p, h, s, d) if case["layout"] == "hnd" else (p, s, h, d)
    x = torch.randn(shape, generator=g, device="cuda", dtype=TYPES[case["dtype"]])
    return x if case["layout"] == "hnd" else x.permute(0, 2, 1, 3)


def _paged(g, case, lens, room):
    """A cache whose pages lie in the pool in random order, with pages for `room` further tokens and -1 behind them."""
    ps = case["page"]
    need = torch.tensor([-(-(x + room) // ps) for x in lens])
    table = torch.full((len(lens), max(1, int(need.max()))), -1, dtype=torch.int32)
    order = torch.randperm(int(need.sum()), generator=torch.Generator().manual_seed(int(g.initial_seed())))
    table[torch.arange(table.shape[1])[None] < need[:, None]] = order.to(torch.int32)
    n_pages = max(1, int(need.sum()))
    return dict(k=_pool(g, n_pages, case), v=_pool(g, n_pages, case), page_table=table.cuda(),
                length=torch.tensor(lens, dtype=torch.int32, device="cuda"))


def _weights(g, cache, case):
    """Accumulated weight (heavy tailed) and position of every slot of a cache that has been evicted from before."""
    pages, ps = cache["k"].shape[0], case["page"]
    cache["mass"] = torch.randn((pages, case["hkv"], ps), generator=g, device="cuda").mul_(1.5).exp_()
    slots = cache["page_table"].shape[1] * ps
    pos = torch.arange(slots, device="cuda", dtype=torch.int32).view(1, -1, ps).expand(case["seqs"], -1, -1)
    cache["pos"] = torch.zeros((pages, case["hkv"], ps), dtype=torch.int32, device="cuda")
    real = cache["page_table"] >= 0
    cache["pos"][cache["page_table"][real].long()] = pos[real][:, None]
    cache["next_pos"] = cache["length"].clone()


def _drafts(g, case, counts, tree):
    """New tokens: offsets, parents (node 0 is the last sampled token) and the ancestors of every node as bits."""
    n, t = len(counts), case["tokens"]
    counts = torch.tensor(counts, device="cuda")
    offsets = torch.zeros(n + 1, dtype=torch.int32, device="cuda")
    offsets[1:] = counts.cumsum(0)
    node = torch.arange(t, device="cuda").expand(n, t)
    back = 1 + (torch.rand((n, t), generator=g, device="cuda") * (4 if tree else 1)).long()
    parent = (node - back).clamp(min=0)
    parent[:, 0] = -1
    bit = torch.ones((), dtype=torch.int64, device="cuda") << node
    mask = bit.clone()
    for i in range(1, t):
        mask[:, i] |= mask.gather(1, parent[:, i:i + 1])[:, 0]
    real = node < counts[:, None]
    return dict(offsets=offsets, parent=parent[real].to(torch.int32), mask=mask[real], tokens=t)


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(int(seed))
    kind = case["kind"]
    if kind == "verify":
        return _prepare_verify(case, g)
    dt, d = TYPES[case["dtype"]], case["d"]

    def rand(*shape):
        return torch.randn(shape, generator=g, device="cuda", dtype=dt)

    s = dict(kind=kind)
    if kind in ("attend", "observe"):
        lens = _lengths(case)
        counts = _counts(case)
        s["cache"] = _paged(g, case, lens, case["tokens"])
        s["tree"] = _drafts(g, case, counts, tree=case["tokens"] > 5 and kind == "attend")
        n = sum(counts)
        s.update(q=rand(n, case["hq"], d) * 1.5, k_new=rand(n, case["hkv"], d), v_new=rand(n, case["hkv"], d),
                 scale=d ** -0.5)
    if kind == "observe":
        _weights(g, s["cache"], case)
        # the path that verification accepted, and the statistics that attention returned
        s["n_path"] = torch.tensor(_accepted(case), dtype=torch.int32, device="cuda")
        node = torch.arange(case["tokens"], dtype=torch.int32, device="cuda").expand(case["seqs"], -1)
        s["path"] = torch.where(node < s["n_path"][:, None], node, -1).contiguous()
        s["lse"] = _plain_attend(s)["lse"]
    if kind == "step":
        lens = [case["keep"]] * case["seqs"]
        counts = [case["tokens"]] * case["seqs"]
        s["cache"] = _paged(g, case, lens, case["tokens"])
        _weights(g, s["cache"], case)
        s["tree"] = _drafts(g, case, counts, tree=False)
        n = sum(counts)
        s.update(k_new=rand(n, case["hkv"], d), v_new=rand(n, case["hkv"], d),
                 mass_new=torch.rand((n, case["hkv"]), generator=g, device="cuda"))
        n_path = [1 + i % case["tokens"] for i in range(case["seqs"])]
        s["n_path"] = torch.tensor(n_path, dtype=torch.int32, device="cuda")
        node = torch.rand((case["seqs"], case["tokens"]), generator=g, device="cuda")
        node[:, 0] = -1  # the path starts at the root and ascends
        rank = torch.arange(case["tokens"], device="cuda")
        n_path = s["n_path"][:, None]
        pick = node.argsort(1)
        pick = torch.where(rank < n_path, pick, case["tokens"]).sort(1).values
        s["path"] = torch.where(rank < n_path, pick, -1).to(torch.int32)
        s["keep"] = s["cache"]["length"].clone()
        s.update(sink=4, recent=max(8, case["keep"] // 16))
    if kind == "demote":
        lens = _lengths(case)
        s["cache"] = _paged(g, case, lens, 1)
        _weights(g, s["cache"], case)
        s["into"] = _paged(g, case, [min(x, case["keep"]) for x in lens], 1)
        _weights(g, s["into"], case)
        for name in ("k", "v", "mass", "pos"):
            s["into"][name].zero_()
        s["into"]["length"].zero_()
        s["keep"] = torch.full((case["seqs"],), case["keep"], dtype=torch.int32, device="cuda")
        s.update(sink=4, recent=case["keep"] // 16)
    if own:  # a serving program keeps its cache's and its batch's descriptions
        from paper_2609_09643_gb300 import kv
        s["handle"] = kv.Cache(**s["cache"])
        if "into" in s:
            s["handle_into"] = kv.Cache(**s["into"])
        if "tree" in s:
            s["batch"] = kv.Tree(s["tree"]["offsets"], s["tree"]["tokens"], mask=s["tree"]["mask"],
                                 parent=s["tree"]["parent"])
    return s


def _prepare_verify(case, g):
    n, t, v = case["seqs"], case["tokens"], case["vocab"]
    s = dict(kind="verify", tree=_drafts(g, case, [t] * n, tree=bool(case["tree"])))
    # a peaked target and a draft model near it; drafted tokens are drawn from the parent's draft distribution
    x = torch.randn((n * t, v), generator=g, device="cuda") * 3
    s["p"] = torch.softmax(x, 1)
    x += torch.randn((n * t, v), generator=g, device="cuda") * 0.7
    x = torch.softmax(x, 1)
    offset = torch.arange(n, device="cuda").repeat_interleave(t) * t
    row = offset + s["tree"]["parent"].clamp(min=0)
    u = torch.rand((n * t, 1), generator=g, device="cuda")
    c = x.cumsum(1)
    s["token"] = torch.searchsorted(c[row], u * c[row][:, -1:]).clamp(max=v - 1)[:, 0].to(torch.int32)
    s["q"] = x.to(TYPES[case["dtype"]])
    s["p"] = s["p"].to(TYPES[case["dtype"]])
    s["u"] = torch.rand(n * t, generator=g, device="cuda")
    s["u_sample"] = torch.rand(n, generator=g, device="cuda")
    if own:  # a serving program keeps its batch's description
        from paper_2609_09643_gb300 import kv
        s["batch"] = kv.Tree(s["tree"]["offsets"], t, mask=s["tree"]["mask"], parent=s["tree"]["parent"])
    return s


# ------------------------------------------------------------ plain forms --
def _slots(c, x):
    """Pool array x of a cache as [seq, head, slot, ...]."""
    x = x[c["page_table"].clamp(min=0).long()].transpose(1, 2)
    return x.reshape(x.shape[0], x.shape[1], -1, *x.shape[4:])


def _by_sequence(tree, x):
    """Rows of new tokens as [seq, token, ...], and which of them exist."""
    at = tree["offsets"][:-1, None].long() + torch.arange(tree["tokens"], device=x.device)
    real = at < tree["offsets"][1:, None]
    return x[at.clamp(max=x.shape[0] - 1)], real


def _scores(s, rows, real, mask):
    """Scaled products of rows [seq, row, hq, d] with all cached and all new keys, -inf where one is not seen, as
    [seq, hkv, row, group, key]."""
    c, tree = s["cache"], s["tree"]
    keys = _slots(c, c["k"]).float()
    b, h, n, d = keys.shape
    new, there = _by_sequence(tree, s["k_new"])
    keys = torch.cat([keys, new.transpose(1, 2).float()], 2)
    r, group = rows.shape[1], rows.shape[2] // h
    q = rows.float().view(b, r, h, group, d).permute(0, 2, 1, 3, 4).reshape(b, h, r * group, d)
    x = torch.matmul(q, keys.transpose(2, 3)).mul_(s["scale"]).view(b, h, r, group, -1)
    node = torch.arange(tree["tokens"], device=keys.device)
    seen = ((mask[:, :, None] >> node) & 1).bool() & there[:, None, :] & real[:, :, None]
    cached = (torch.arange(n, device=keys.device) < c["length"][:, None])[:, None, :] & real[:, :, None]
    seen = torch.cat([cached, seen], 2)
    return x.masked_fill_(~seen[:, None, :, None, :], -math.inf)


def _plain_attend(s):
    c, tree = s["cache"], s["tree"]
    q, real = _by_sequence(tree, s["q"])
    x = _scores(s, q, real, _by_sequence(tree, tree["mask"])[0])
    top = x.amax(-1, keepdim=True)
    top = torch.where(top == -math.inf, 0.0, top)
    x = (x - top).exp_()
    total = x.sum(-1, keepdim=True)
    lse = (total.log() + top)[..., 0]
    values = torch.cat([_slots(c, c["v"]).float(), _by_sequence(tree, s["v_new"])[0].transpose(1, 2).float()], 2)
    b, h, r, group, n = x.shape
    out = torch.matmul(x.view(b, h, r * group, n), values).view(b, h, r, group, -1)
    out = out / torch.where(total == 0, 1.0, total)
    out = out.permute(0, 2, 1, 3, 4).reshape(b, r, h * group, -1)
    return dict(out=out[real].to(s["q"].dtype), lse=lse.permute(0, 2, 1, 3).reshape(b, r, h * group)[real].contiguous())


def _plain_observe(s):
    c, tree = s["cache"], s["tree"]
    at = s["path"].clamp(min=0).long()
    real = torch.arange(at.shape[1], device=at.device) < s["n_path"][:, None]
    seq = torch.arange(at.shape[0], device=at.device)[:, None]
    q = _by_sequence(tree, s["q"])[0][seq, at]
    lse = _by_sequence(tree, s["lse"])[0][seq, at]
    mask = _by_sequence(tree, tree["mask"])[0][seq, at]
    x = _scores(s, q, real, mask)
    b, h, r, group, _ = x.shape
    x = (x - lse.view(b, r, h, group).transpose(1, 2)[..., None]).exp_().sum((2, 3))
    n = x.shape[2] - tree["tokens"]
    table = c["page_table"]
    per_page = x[:, :, :n].reshape(b, h, table.shape[1], -1).transpose(1, 2).flatten(0, 1)
    c["mass"].index_add_(0, table.clamp(min=0).flatten().long(), per_page)
    there = _by_sequence(tree, s["k_new"])[1]
    return dict(mass=c["mass"], mass_new=x[:, :, n:].transpose(1, 2)[there].contiguous())


def _plain_commit(s):
    c, ps = s["cache"], s["cache"]["k"].shape[2]
    rank = torch.arange(s["path"].shape[1], device="cuda")
    seq, i = (rank < s["n_path"][:, None]).nonzero(as_tuple=True)
    node = s["tree"]["offsets"][seq].long() + s["path"][seq, i]
    slot = c["length"][seq].long() + i
    page, off = c["page_table"][seq, slot // ps].long(), slot % ps
    c["k"][page, :, off] = s["k_new"][node]
    c["v"][page, :, off] = s["v_new"][node]
    c["mass"][page, :, off] = s["mass_new"][node]
    c["pos"][page, :, off] = (c["next_pos"][seq] + i.to(torch.int32))[:, None]
    c["length"] += s["n_path"]
    c["next_pos"] += s["n_path"]


def _kept(c, keep, sink, recent):
    """Which slots stay, [seq, head, slot], and how many of each session."""
    mass, pos = _slots(c, c["mass"]), _slots(c, c["pos"])
    slot = torch.arange(mass.shape[2], device=mass.device)
    there = slot < c["length"][:, None, None]
    safe = (pos < sink) | (pos >= c["next_pos"][:, None, None] - recent)
    rank = torch.where(there, torch.where(safe, math.inf, mass), -math.inf)
    order = rank.sort(dim=-1, descending=True, stable=True).indices
    n = torch.minimum(c["length"], keep)
    best = (slot < n[:, None, None]).expand_as(order)
    return torch.zeros_like(best).scatter(2, order, best), n


def _plain_evict(s):
    c, ps = s["cache"], s["cache"]["k"].shape[2]
    kept, n = _kept(c, s["keep"], s["sink"], s["recent"])
    slot = torch.arange(kept.shape[2], device=kept.device)
    inside = slot < n[:, None, None]
    to_seq, to_head, to = (~kept & inside).nonzero(as_tuple=True)
    of_seq, of_head, of = (kept & ~inside).nonzero(as_tuple=True)
    to_page = c["page_table"][to_seq, to // ps].long()
    of_page = c["page_table"][of_seq, of // ps].long()
    for x in (c["k"], c["v"], c["mass"], c["pos"]):
        x[to_page, to_head, to % ps] = x[of_page, of_head, of % ps]
    c["length"].copy_(n)
    return {name: c[name] for name in ("k", "v", "mass", "pos", "length", "next_pos")}


def _plain_demote(s):
    c, into, ps = s["cache"], s["into"], s["cache"]["k"].shape[2]
    kept, n = _kept(c, s["keep"], s["sink"], s["recent"])
    seq, head, of = kept.nonzero(as_tuple=True)
    to = (kept.cumsum(2) - 1)[seq, head, of]
    page, to_page = c["page_table"][seq, of // ps].long(), into["page_table"][seq, to // ps].long()
    for name in ("k", "v", "mass", "pos"):
        into[name][to_page, head, to % ps] = c[name][page, head, of % ps]
    into["length"].copy_(n)
    into["next_pos"].copy_(c["next_pos"])
    return {name: into[name] for name in ("k", "v", "mass", "pos", "length", "next_pos")}


def _weight(x):
    return torch.where(x > 0, x, 0.0).clamp(max=1.0)


def _plain_verify(s):
    tree = s["tree"]
    t, offset = tree["tokens"], tree["offsets"][:-1].long()
    n, v = offset.shape[0], s["p"].shape[1]
    cur = torch.zeros_like(offset)
    z = torch.ones(n, device="cuda")
    d = _weight(s["p"][offset].float())
    path = torch.full((n, t), -1, dtype=torch.int64, device="cuda")
    path[:, 0] = 0
    n_path = torch.ones(n, dtype=torch.int64, device="cuda")
    seq = torch.arange(n, device="cuda")
    for i in range(1, t):  # a node's parent comes before it: one pass finds the whole path
        node = offset + i
        tried = tree["parent"][node] == cur
        token = s["token"][node].long()
        q = _weight(s["q"][offset + cur].float())
        accepted = tried & ((s["u"][node] * q[seq, token]) * z < d[seq, token])
        rejected = (tried & ~accepted)[:, None]
        d = torch.where(rejected, (d - z[:, None] * q).clamp(min=0.0), d)
        left = (d * FIX).to(torch.int64).sum(1).float() / FIX
        z = torch.where(rejected[:, 0], left, torch.where(accepted, 1.0, z))
        cur = torch.where(accepted, i, cur)
        d = torch.where(accepted[:, None], _weight(s["p"][node].float()), d)
        path[seq, torch.where(accepted, n_path, 0)] = torch.where(accepted, i, 0)
        n_path += accepted
    w = (d * FIX).to(torch.int64)
    w = torch.where(w.sum(1, keepdim=True) > 0, w, (_weight(s["p"][offset + cur].float()) * FIX).to(torch.int64))
    c = w.cumsum(1)
    total, u = c[:, -1], (s["u_sample"] * 2.0 ** 24).to(torch.int64)
    goal = u * (total >> 24) + ((u * (total & ((1 << 24) - 1))) >> 24)  # floor(u total), in 64 bits
    token = torch.where(total > 0, (c <= goal[:, None]).sum(1), -1)
    return dict(path=path.to(torch.int32), n_path=n_path.to(torch.int32), token=token.to(torch.int32))


def run(state):
    s = state
    if not own:
        if s["kind"] == "step":
            _plain_commit(s)
            return _plain_evict(s)
        return {"attend": _plain_attend, "observe": _plain_observe, "demote": _plain_demote,
                "verify": _plain_verify}[s["kind"]](s)
    from paper_2609_09643_gb300 import kv
    if s["kind"] == "attend":
        out, lse = kv.attend(s["handle"], s["batch"], s["q"], s["k_new"], s["v_new"], s["scale"])
        return dict(out=out, lse=lse)
    if s["kind"] == "observe":
        mass_new = kv.observe(s["handle"], s["batch"], s["q"], s["lse"], s["k_new"], s["scale"], path=s["path"],
                              n_path=s["n_path"])
        return dict(mass=s["cache"]["mass"], mass_new=mass_new)
    if s["kind"] == "step":
        kv.commit(s["handle"], s["batch"], s["k_new"], s["v_new"], mass_new=s["mass_new"], path=s["path"],
                  n_path=s["n_path"])
        kv.evict(s["handle"], s["keep"], sink=s["sink"], recent=s["recent"])
        return {name: s["cache"][name] for name in ("k", "v", "mass", "pos", "length", "next_pos")}
    if s["kind"] == "demote":
        kv.evict(s["handle"], s["keep"], sink=s["sink"], recent=s["recent"], into=s["handle_into"])
        return {name: s["into"][name] for name in ("k", "v", "mass", "pos", "length", "next_pos")}
    path, n_path, token = kv.verify(s["batch"], s["token"], s["p"], s["q"], s["u"], s["u_sample"])
    return dict(path=path, n_path=n_path, token=token)


# ------------------------------------------------------------------- work --
def work(case):
    kind = case["kind"]
    if kind == "verify":
        # the last row of each session's target probabilities, and the draft's: nearly every walk ends in a rejection
        size = 4 if case["dtype"] == "fp32" else 2
        rows = 2 if case["tokens"] > 1 else 1
        return dict(bytes=case["seqs"] * (rows * case["vocab"] * size + 20 * case["tokens"]),
                    flops=case["seqs"] * case["vocab"] * 4)
    h, d, e, n = case["hkv"], case["d"], 2, case["seqs"]
    if kind == "step":
        moved = sum(1 + i % case["tokens"] for i in range(n))  # committed, and as many evicted
        scan = sum(case["keep"] + 1 + i % case["tokens"] for i in range(n)) * h * 8
        return dict(bytes=scan + moved * h * (4 * (2 * d * e) + 4 * 8), flops=scan / 8)
    if kind == "demote":
        lens = _lengths(case)
        rows = sum(min(x, case["keep"]) for x in lens) * h
        return dict(bytes=sum(lens) * h * 8 + rows * 2 * (2 * d * e + 8), flops=sum(lens) * h)
    lens, counts = _lengths(case), _counts(case)
    hq = case["hq"]
    if kind == "attend":
        flops = sum(4 * t * hq * (x + t) * d for x, t in zip(lens, counts))
        new = sum(counts) * (2 * hq * d * e + 2 * h * d * e + 4 * hq + 8)
        return dict(bytes=sum(lens) * h * 2 * d * e + new, flops=flops)
    rows = _accepted(case)
    flops = sum(2 * r * hq * (x + t) * d for x, t, r in zip(lens, counts, rows))
    new = sum(rows) * (hq * d * e + 4 * hq) + sum(counts) * (h * d * e + 4 * h)
    return dict(bytes=sum(lens) * h * (d * e + 8) + new, flops=flops)


# ------------------------------------------------------- 64-bit arithmetic --
def exact(case, seed):
    """The operators' definitions, one session (and head) at a time, in 64 bits."""
    if case["kind"] == "verify":
        return None  # whole numbers, by an arithmetic that is exact in itself
    global own
    was, own = own, False
    try:
        s = prepare(case, seed)
    finally:
        own = was
    c = s["cache"]
    lens, ps = c["length"].tolist(), c["k"].shape[2]

    def place(cache, b, count):
        at = torch.arange(count, device="cuda")
        return cache["page_table"][b].long()[at // ps], at % ps

    if case["kind"] in ("attend", "observe"):
        off, bits = s["tree"]["offsets"].tolist(), s["tree"]["mask"].tolist()
        hq, h = case["hq"], case["hkv"]
        g = hq // h
        out = torch.zeros(s["q"].shape, dtype=torch.float64, device="cuda")
        lse = torch.zeros(s["q"].shape[:2], dtype=torch.float64, device="cuda")
        mass = c["mass"].double() if "mass" in c else None
        mass_new = torch.zeros(s["k_new"].shape[:2], dtype=torch.float64, device="cuda")
        for b, n in enumerate(lens):
            page, slot = place(c, b, n)
            nodes = range(off[b], off[b + 1])
            take = list(nodes) if case["kind"] == "attend" else [off[b] + i for i in s["path"][b].tolist() if i >= 0]
            sees = torch.tensor([[bits[i] >> j & 1 for j in range(len(nodes))] for i in take], device="cuda").bool()
            sees = torch.cat([torch.ones((len(take), n), dtype=torch.bool, device="cuda"), sees], 1)
            for head in range(h):
                k = torch.cat([c["k"][page, head, slot], s["k_new"][off[b]:off[b + 1], head]]).double()
                q = s["q"][take, head * g:(head + 1) * g].double()
                x = torch.einsum("tgd,nd->tgn", q, k) * s["scale"]
                x = torch.where(sees[:, None], x, -math.inf)
                if case["kind"] == "attend":
                    v = torch.cat([c["v"][page, head, slot], s["v_new"][off[b]:off[b + 1], head]]).double()
                    total = torch.logsumexp(x, 2)
                    lse[off[b]:off[b + 1], head * g:(head + 1) * g] = total
                    out[off[b]:off[b + 1], head * g:(head + 1) * g] = torch.exp(x - total[..., None]) @ v
                else:
                    w = torch.exp(x - s["lse"][take, head * g:(head + 1) * g, None].double()).sum((0, 1))
                    mass[page, head, slot] += w[:n]
                    mass_new[off[b]:off[b + 1], head] = w[n:]
        return dict(out=out, lse=lse) if case["kind"] == "attend" else dict(mass=mass, mass_new=mass_new)

    to = s["into"] if case["kind"] == "demote" else c
    if case["kind"] == "step":
        off, paths, first = s["tree"]["offsets"].tolist(), s["path"].tolist(), c["next_pos"].tolist()
        for b, path in enumerate(paths):
            for i, node in enumerate(x for x in path if x >= 0):
                page, slot = int(c["page_table"][b, lens[b] // ps]), lens[b] % ps
                for name, new in (("k", "k_new"), ("v", "v_new"), ("mass", "mass_new")):
                    c[name][page, :, slot] = s[new][off[b] + node]
                c["pos"][page, :, slot] = first[b] + i
                lens[b] += 1
                c["next_pos"][b] += 1
    for b, n in enumerate(lens):
        page, slot = place(c, b, n)
        most = min(n, int(s["keep"][b]))
        for head in range(case["hkv"]):
            pos = c["pos"][page, head, slot]
            safe = (pos < s["sink"]) | (pos >= int(c["next_pos"][b]) - s["recent"])
            value = torch.where(safe, math.inf, c["mass"][page, head, slot].double())
            kept = value.sort(dim=0, descending=True, stable=True).indices[:most].sort().values
            if case["kind"] == "demote":
                of, at = kept, torch.arange(most, device="cuda")
            else:
                free = torch.ones(most, dtype=torch.bool, device="cuda")
                free[kept[kept < most]] = False
                of, at = kept[kept >= most], free.nonzero()[:, 0]
            to_page = to["page_table"][b].long()[at // ps]
            for name in ("k", "v", "mass"):
                to[name][to_page, head, at % ps] = c[name][page[of], head, slot[of]]
    return {name: to[name].double() for name in ("k", "v", "mass")} | dict(pos=None, length=None, next_pos=None)
