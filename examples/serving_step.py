"""Agent sessions served from a KV cache in two tiers.

Every step runs the KV operators on the fast tier's cache, without waiting for
the GPU in between: attention over the drafted trees, verification of the
drafts, the weight that the accepted tokens give to the cached ones, their keys
and values into the pages, eviction down to each session's budget.  In a tool
gap the live ranking names the sessions that should leave the fast tier; their
most attended tokens are copied to the other tier's cache (their pages here are
the program's to give away then).

The model is left out: queries, keys, values and probabilities are random, of
the shapes that a model of one layer would give.

    python examples/serving_step.py [--sessions 8] [--steps 16]
"""
import argparse
import os
import sys

import numpy as np
import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

import synth  # noqa: E402
from paper_2609_09643_gb300 import binding as B, kv  # noqa: E402

HEADS, GROUP, DIM, PAGE, VOCAB = 8, 4, 128, 64, 32000


def tier(sessions, slots):
    """An empty cache with pages for `slots` tokens of every session."""
    per = -(-slots // PAGE)
    shape = (sessions * per, HEADS, PAGE)
    new = lambda *s, dtype: torch.zeros(s, dtype=dtype, device="cuda")  # noqa: E731
    ints = lambda: new(sessions, dtype=torch.int32)  # noqa: E731
    table = torch.randperm(sessions * per).to(torch.int32).view(sessions, per).cuda()
    return kv.Cache(new(*shape, DIM, dtype=torch.bfloat16), new(*shape, DIM, dtype=torch.bfloat16), table, ints(),
                    mass=new(*shape, dtype=torch.float32), pos=new(*shape, dtype=torch.int32), next_pos=ints(),
                    status=ints())


def prompt(cache, tokens):
    """The sessions' first tokens, 64 at a time: a chain of which all are accepted."""
    for first in range(0, tokens, kv.MAX_TOKENS):
        n = min(kv.MAX_TOKENS, tokens - first)
        total = cache.n_seqs * n
        chain = kv.Tree(torch.arange(0, total + 1, n, dtype=torch.int32, device="cuda"), n, n_tokens=total)
        k, v = (torch.randn(total, HEADS, DIM, device="cuda").to(torch.bfloat16) for _ in range(2))
        kv.commit(cache, chain, k, v)


def drafts(sessions, width, depth):
    """Trees of `depth` levels, `width` drafts from each accepted-so-far node's first child."""
    parent, mask = [-1], [1]
    for _ in range(depth):
        at = len(parent) - width if len(parent) > 1 else 0
        for _ in range(width):
            mask.append(mask[at] | 1 << len(parent))
            parent.append(at)
    n = len(parent)
    rep = lambda x, dtype: torch.tensor(x * sessions, dtype=dtype, device="cuda")  # noqa: E731
    offsets = torch.arange(0, sessions * n + 1, n, dtype=torch.int32, device="cuda")
    return kv.Tree(offsets, n, mask=rep(mask, torch.int64), parent=rep(parent, torch.int32)), parent


def main(sessions=8, steps=16, prompt_tokens=600, budget=512, width=3, depth=3, seed=0, quiet=False):
    torch.manual_seed(seed)
    fast, far = tier(sessions, prompt_tokens + 64 + steps * (depth + 1)), tier(sessions, budget)
    tree, parent = drafts(sessions, width, depth)
    n = tree.n_tokens
    prompt(fast, prompt_tokens)
    keep = torch.full((sessions,), budget, dtype=torch.int32, device="cuda")
    rows = torch.tensor(parent, device="cuda").clamp(min=0).repeat(sessions) + \
        torch.arange(sessions, device="cuda").repeat_interleave(len(parent)) * len(parent)
    told = torch.zeros(sessions, dtype=torch.int64, device="cuda")
    for _ in range(steps):
        q = torch.randn(n, HEADS * GROUP, DIM, device="cuda").to(torch.bfloat16)
        k, v = (torch.randn(n, HEADS, DIM, device="cuda").to(torch.bfloat16) for _ in range(2))
        logits = torch.randn(n, VOCAB, device="cuda") * 4
        p = torch.softmax(logits, 1)
        draft = torch.softmax(logits + torch.randn_like(logits) * 0.3, 1)
        token = torch.multinomial(draft[rows], 1)[:, 0].to(torch.int32)
        u, u_sample = torch.rand(n, device="cuda"), torch.rand(sessions, device="cuda")

        out, lse = kv.attend(fast, tree, q, k, v)
        path, n_path, next_token = kv.verify(tree, token, p, draft, u, u_sample)
        mass_new = kv.observe(fast, tree, q, lse, k, path=path, n_path=n_path)
        kv.commit(fast, tree, k, v, mass_new=mass_new, path=path, n_path=n_path)
        kv.evict(fast, keep, sink=4, recent=32)
        told += n_path

    # a tool gap: the ranking names the sessions to leave the fast tier
    live = synth.make_records(seed, sessions)
    live.kv_tok[:] = fast.length.cpu().numpy().astype(live.kv_tok.dtype)
    live.tier[:] = 1
    live.flags[:] = 0
    params = dict(sigma_q=np.full(51, 2048, np.uint16), k=max(1, sessions // 4))
    ranked = B.rank_outputs(sessions, params["k"], 0)
    B.rank(B.records_to_device(live), params, ranked)
    victims = B.rank_result(ranked)["victims"].astype(np.int64)
    leave = torch.zeros(sessions, dtype=torch.int32, device="cuda")
    leave[torch.from_numpy(victims).cuda()] = budget // 4
    kv.evict(fast, leave, sink=4, recent=32, into=far)
    if not quiet:
        print(f"{sessions} sessions, {steps} steps: {told.float().mean() / steps:.2f} tokens accepted a step, "
              f"{fast.length.tolist()} slots kept; sessions {sorted(victims.tolist())} left with "
              f"{far.length.tolist()} slots")
    return dict(fast=fast, far=far, out=out, told=told, victims=victims, next_token=next_token)


if __name__ == "__main__":
    a = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    a.add_argument("--sessions", type=int, default=8)
    a.add_argument("--steps", type=int, default=16)
    a = a.parse_args()
    main(a.sessions, a.steps)
