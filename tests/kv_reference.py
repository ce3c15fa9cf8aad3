"""Plain 64-bit statements of the KV-cache operators, session by session and
head by head (numpy; shares no code with the library), and the makers of their
inputs."""
import math

import numpy as np
import torch

TYPES = {"bf16": torch.bfloat16, "fp16": torch.float16}
UNIT = {"bf16": 2.0 ** -8, "fp16": 2.0 ** -11}  # half an ulp, relative


def f64(x):
    return x.detach().cpu().to(torch.float64).numpy()


class Made:
    """A paged cache with its step's tensors.  Unused slots and pages hold
    `junk`, which nothing may read."""

    def __init__(self, lens, counts, hkv=2, group=4, d=64, page=16, dtype="bf16", layout="hnd", seed=0, room=64,
                 junk=float("nan"), tree=True, device="cuda", marks=True):
        r = np.random.default_rng(seed)
        g = torch.Generator().manual_seed(seed)
        dt = TYPES[dtype]
        self.dtype, self.lens, self.counts, self.group, self.page = dtype, list(lens), list(counts), group, page
        n = len(lens)
        need = [-(-(x + room) // page) for x in lens]
        pages = sum(need) + 3
        order = r.permutation(pages)[:sum(need)]
        table = np.full((n, max(need + [1])), -1, np.int32)
        at = 0
        for b, k in enumerate(need):
            table[b, :k] = order[at:at + k]
            at += k
        self.table = table

        def pool(fill):
            shape = (pages, hkv, page, d) if layout == "hnd" else (pages, page, hkv, d)
            x = torch.full(shape, junk, dtype=dt)
            x = x if layout == "hnd" else x.permute(0, 2, 1, 3)
            for b, m in enumerate(lens):
                for s in range(0, m, page):
                    k = min(page, m - s)
                    x[table[b, s // page], :, :k] = fill(hkv, k, d).to(dt)
            return x.to(device) if layout == "hnd" else x.permute(0, 2, 1, 3).to(device).permute(0, 2, 1, 3)

        normal = lambda *s: torch.randn(*s, generator=g)  # noqa: E731
        self.k, self.v = pool(normal), pool(normal)
        self.page_table = torch.from_numpy(table).to(device)
        self.length = torch.tensor(lens, dtype=torch.int32, device=device)
        self.status = torch.zeros(n, dtype=torch.int32, device=device)
        if marks:
            self.mass = torch.exp(normal(pages, hkv, page)).to(device)
            self.pos = torch.from_numpy(r.integers(0, 1 << 20, (pages, hkv, page)).astype(np.int32)).to(device)
            self.next_pos = torch.tensor([x + 7 for x in lens], dtype=torch.int32, device=device)
        off = np.concatenate(([0], np.cumsum(counts))).astype(np.int32)
        total = int(off[-1])
        self.off, self.total = off, total
        self.offsets = torch.from_numpy(off).to(device)
        self.q = (normal(total, hkv * group, d) * 1.5).to(dt).to(device)
        self.k_new, self.v_new = (normal(total, hkv, d).to(dt).to(device) for _ in range(2))
        parent, mask = np.full(total, -1, np.int32), np.zeros(total, np.uint64)
        for b, t in enumerate(counts):
            for i in range(t):
                p = -1 if i == 0 else int(r.integers(max(0, i - 3), i)) if tree else i - 1
                parent[off[b] + i] = p
                mask[off[b] + i] = (mask[off[b] + p] if p >= 0 else np.uint64(0)) | np.uint64(1 << i)
        self.parent_np, self.mask_np = parent, mask
        self.parent = torch.from_numpy(parent).to(device)
        self.mask = torch.from_numpy(mask.view(np.int64)).to(device)
        self.hkv, self.d, self.scale = hkv, d, d ** -0.5

    def cache(self, kv, **kw):
        a = dict(status=self.status)
        if hasattr(self, "mass"):
            a.update(mass=self.mass, pos=self.pos, next_pos=self.next_pos)
        a.update(kw)
        return kv.Cache(self.k, self.v, self.page_table, self.length, **a)

    def tree(self, kv, **kw):
        return kv.Tree(self.offsets, max([*self.counts, 1]), n_tokens=self.total,
                       **dict(dict(mask=self.mask, parent=self.parent), **kw))

    def slots(self, x, b, n=None):
        """Array x of session b's first n slots: [slot, head, ...] (absent pages: 0)."""
        n = self.lens[b] if n is None else n
        s = np.arange(n)
        return x[self.table[b, s // self.page], :, s % self.page]


def attend(m, mask=None, scale=None):
    """(out, lse, bound of |out|'s error, bound of |lse|'s) in 64 bits."""
    mask = m.mask_np if mask is None else mask
    scale = m.scale if scale is None else scale
    k, v, q, kn, vn = (f64(x) for x in (m.k, m.v, m.q, m.k_new, m.v_new))
    out, lse = np.zeros(q.shape), np.full(q.shape[:2], -np.inf)
    tol, tol_lse = np.zeros(q.shape), np.zeros(q.shape[:2])
    eps, G = UNIT[m.dtype], m.group
    for b, n in enumerate(m.lens):
        for i in range(m.counts[b]):
            row = m.off[b] + i
            seen = [j for j in range(m.counts[b]) if int(mask[row]) >> j & 1]
            new = [m.off[b] + j for j in seen]
            for h in range(m.hkv):
                keys = np.concatenate([m.slots(k, b)[:, h], kn[new, h]])
                vals = np.concatenate([m.slots(v, b)[:, h], vn[new, h]])
                if not len(keys):
                    continue
                for g in range(h * G, h * G + G):
                    with np.errstate(all="ignore"):
                        s = keys @ q[row, g] * scale
                        size = np.max(np.abs(keys) @ np.abs(q[row, g])) * abs(scale)
                        top = s.max()
                        e = np.exp(s - top)
                        w = e / e.sum()
                        out[row, g] = w @ vals
                        lse[row, g] = top + math.log(e.sum())
                        # a product: its rounding along the sum; the base-2 exponent's rounding
                        ds = (m.d / 8 + 4) * 2.0 ** -23 * (size + 1) + 2.0 ** -21
                        # a weight is rounded to the type (in fp16 below 2^-14 to steps of 2^-24),
                        # and so is the result
                        spread = w @ np.abs(vals)
                        tol[row, g] = spread * (2.1 * eps + 2 * ds) + 1e-30
                        if m.dtype == "fp16":
                            tol[row, g] += 2.0 ** -24 * np.abs(vals).sum(0) / e.sum() + 2.0 ** -24
                        tol_lse[row, g] = ds + 2.0 ** -22 * abs(lse[row, g])
    return out, lse, tol, tol_lse


def observe(m, lse, paths=None, mask=None):
    """What is added to every cached slot, per session [slot, head], and
    mass_new, with the bounds of their errors."""
    mask = m.mask_np if mask is None else mask
    k, q, kn, lse = f64(m.k), f64(m.q), f64(m.k_new), f64(lse)
    G, added, bound = m.group, [], []
    new, new_bound = np.zeros((m.total, m.hkv)), np.zeros((m.total, m.hkv))
    for b, n in enumerate(m.lens):
        a, t = np.zeros((n, m.hkv)), np.zeros((n, m.hkv))
        for i in (range(m.counts[b]) if paths is None else paths[b]):
            row = m.off[b] + i
            for h in range(m.hkv):
                keys = np.concatenate([m.slots(k, b)[:, h], kn[m.off[b]:m.off[b + 1], h]])
                see = np.array([True] * n + [bool(int(mask[row]) >> j & 1) for j in range(m.counts[b])])
                for g in range(h * G, h * G + G):
                    if lse[row, g] == -np.inf:
                        continue
                    s = keys @ q[row, g] * m.scale
                    w = np.where(see, np.exp(np.where(see, s, 0) - lse[row, g]), 0)
                    size = np.abs(keys) @ np.abs(q[row, g]) * m.scale
                    dw = w * ((m.d / 8 + 4) * 2.0 ** -23 * (size + 1) + 2.0 ** -21 + 2.0 ** -22 * abs(lse[row, g]))
                    a[:, h] += w[:n]
                    t[:, h] += dw[:n]
                    new[m.off[b]:m.off[b + 1], h] += w[n:]
                    new_bound[m.off[b]:m.off[b + 1], h] += dw[n:]
        rows = m.counts[b] * G
        added.append(a)
        bound.append(t + rows * 2.0 ** -23 * a)
        new_bound[m.off[b]:m.off[b + 1]] += rows * 2.0 ** -23 * new[m.off[b]:m.off[b + 1]]
    return added, bound, new, new_bound


def kept(mass, pos, n_slots, keep, sink, recent, next_pos):
    """Slots of one session and head that stay, ascending."""
    def order(s):
        safe = pos[s] < sink or pos[s] >= next_pos - recent
        x = float(mass[s])
        x = -math.inf if math.isnan(x) else x
        return (0, s) if safe else (1, 1 if math.isnan(mass[s]) else 0, -x, s)
    return sorted(sorted(range(n_slots), key=order)[:max(0, min(n_slots, keep))])


def weight(x):
    return np.float32(min(max(float(x), 0.0), 1.0)) if x > 0 else np.float32(0)


def verify(counts, parent, token, p, q, u, u_sample, steps):
    """The walk of every session, one vocabulary entry at a time where it matters."""
    f = np.float32
    off = np.concatenate(([0], np.cumsum(counts)))
    paths, tokens = [], []
    w = lambda row: np.where(row > 0, np.minimum(row, f(1)), f(0)).astype(f)  # noqa: E731
    fix = lambda d: [int(x) for x in np.floor(d.astype(np.float64) * 2.0 ** 40)]  # noqa: E731
    V = p.shape[1]
    for b, t in enumerate(counts):
        if t == 0:
            paths.append([])
            tokens.append(-1)
            continue
        cur, path, z, d = 0, [0], f(1), w(p[off[b]])
        for i in range(1, t):
            x = int(token[off[b] + i])
            if parent[off[b] + i] != cur or not 0 <= x < V:
                continue
            y = w(q[off[b] + cur]) if q is not None else None
            if f(f(u[off[b] + i] * (y[x] if y is not None else f(1))) * z) < d[x]:
                cur, z = i, f(1)
                path.append(i)
                d = w(p[off[b] + i])
            else:
                if y is not None:
                    d = np.maximum(d - (z * y).astype(f), f(0)).astype(f)
                else:
                    d = d.copy()
                    d[x] = 0
                z = f(f(sum(fix(d))) * f(2.0 ** -40))
        c = fix(d)
        if sum(c) == 0:
            c = fix(w(p[off[b] + cur]))
        goal, run, chosen = int(u_sample[b] * 2 ** 24) * sum(c) >> 24, 0, -1
        for x, k in enumerate(c):
            run += k
            if run > goal:
                chosen = x
                break
        paths.append(path)
        tokens.append(chosen)
    out = np.full((len(counts), steps), -1, np.int64)
    for b, path in enumerate(paths):
        out[b, :len(path)] = path
    return out, np.array([len(x) for x in paths]), np.array(tokens)
