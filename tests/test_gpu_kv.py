"""The KV-cache operators on the GPU against plain 64-bit statements
(kv_reference.py), at the sizes, masks and layouts where they can go wrong.
Tolerances are bounds of the roundings that the operators document."""
import math

import numpy as np
import pytest
import torch

import kv_reference as ref
from kv_reference import Made, f64

pytestmark = pytest.mark.gpu
INF, NAN = float("inf"), float("nan")


@pytest.fixture(scope="module")
def kv():
    from paper_2609_09643_gb300 import native
    native.build()
    from paper_2609_09643_gb300 import kv
    return kv


def check_attend(kv, m, mask=None, cache=None, scale=None, **kw):
    cache = m.cache(kv) if cache is None else cache
    tree = m.tree(kv)
    out, lse = kv.attend(cache, tree, m.q, m.k_new, m.v_new, scale, **kw)
    torch.cuda.synchronize()
    assert not m.status.any()
    want, want_lse, tol, tol_lse = ref.attend(m, mask=mask, scale=scale)
    got, got_lse = f64(out), f64(lse)
    assert np.array_equal(np.isnan(got), np.isnan(want))
    assert np.array_equal(got_lse == -np.inf, want_lse == -np.inf)
    ok = np.isfinite(want)
    assert np.array_equal(got[~ok & ~np.isnan(want)], want[~ok & ~np.isnan(want)])
    worst = np.max(np.abs(got[ok] - want[ok]) / (tol[ok] + 1e-30), initial=0)
    assert worst <= 1, worst
    ok = np.isfinite(want_lse)
    assert np.max(np.abs(got_lse[ok] - want_lse[ok]) / tol_lse[ok], initial=0) <= 1
    return out, lse


# ----------------------------------------------------------------- attend --
@pytest.mark.parametrize("d", [8, 64, 72, 96, 128, 136, 256])
@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
def test_attend_head_sizes(kv, d, dtype):
    check_attend(kv, Made([0, 1, 63, 200], [1, 3, 2, 5], d=d, dtype=dtype, layout="nhd", seed=d))


@pytest.mark.parametrize("group,counts", [(1, [1, 1, 1]), (1, [64, 17, 2]), (3, [5, 1, 6]), (4, [4, 4, 4]),
                                          (5, [7, 0, 64]), (8, [64, 33, 1]), (16, [64, 1, 3]), (64, [1, 64, 2])])
@pytest.mark.parametrize("d", [64, 128])
def test_attend_rows(kv, group, counts, d):
    """Rows per KV head from 1 to 4096: every row tile, full and ragged."""
    check_attend(kv, Made([70, 300, 129], counts, group=group, hkv=2, d=d, seed=group))


@pytest.mark.parametrize("group,counts", [(12, [64, 43, 1]), (9, [64, 57, 22]), (16, [33, 48, 40])])
@pytest.mark.parametrize("d", [64, 128])
def test_attend_three_row_groups(kv, group, counts, d):
    """513 to 768 rows per KV head: three CTAs share a run's keys, and the
    sessions' segments are split."""
    check_attend(kv, Made([2000, 300, 129], counts, group=group, hkv=2, d=d, seed=group))


@pytest.mark.parametrize("group", [1, 16])
@pytest.mark.parametrize("page", [1, 7, 16, 24, 64, 100, 256])
def test_attend_pages_and_lengths(kv, page, group):
    lens = [0, 1, 2, 15, 16, 17, 63, 64, 65, 127, 128, 129, 255, 257, 1000]
    check_attend(kv, Made(lens, [1 + i % 9 for i in range(len(lens))], page=page, hkv=1, group=group, seed=page,
                          layout="hnd" if page % 2 else "nhd"))


@pytest.mark.parametrize("counts", [1, 40])
def test_attend_long_context_split_over_all_ctas(kv, counts):
    check_attend(kv, Made([40011], [counts], hkv=1, group=4, d=128, page=64, seed=5))


def test_attend_many_sessions(kv):
    """More sessions than a CTA has threads, some without new tokens."""
    n = 300
    check_attend(kv, Made([(37 * i) % 150 for i in range(n)], [i % 4 for i in range(n)], hkv=1, group=2, seed=9))


@pytest.mark.parametrize("group", [4, 16])
def test_attend_masks_that_leave_rows_empty(kv, group):
    m = Made([0, 0, 30], [5, 20, 3], group=group, seed=3)
    mask = m.mask_np.copy()
    mask[[1, 4, 7, 25]] = 0          # nothing at all
    mask[2] = np.uint64(1 << 40)     # a node that does not exist
    mask[26] = ~np.uint64(0)         # all nodes, and more bits than there are
    m.mask = torch.from_numpy(mask.view(np.int64)).cuda()
    m.status.zero_()
    out, lse = check_attend(kv, m, mask=mask)
    assert float(out[1].abs().max()) == 0 and bool((lse[1] == -INF).all())


def test_attend_without_mask_is_a_chain(kv):
    m = Made([50, 0], [6, 64], seed=4, tree=False)
    a, al = check_attend(kv, m)
    b, bl = kv.attend(m.cache(kv), m.tree(kv, mask=None), m.q, m.k_new, m.v_new)
    assert torch.equal(a, b) and torch.equal(al, bl)


@pytest.mark.parametrize("group", [4, 16])
@pytest.mark.parametrize("bad", [INF, -INF, NAN])
def test_attend_hidden_nodes_do_not_reach_a_row(kv, bad, group):
    """A node's key and value may be anything where a mask hides it; where one
    is seen, infinities and NaN come through as in the formula."""
    m = Made([40, 0], [6, 20], group=group, seed=8)
    m.v_new[3, 0, 5] = bad
    m.v_new[9, 1] = bad
    m.k_new[12, 1] = NAN
    check_attend(kv, m)


@pytest.mark.parametrize("d", [64, 128])
def test_attend_odd_values_of_many_short_segments(kv, d):
    """Large trees over a context, each followed by sessions without one, many to
    a CTA: whose new values hold infinities and NaN stays with the session."""
    lens, counts = [130, 0, 0, 0, 0, 0] * 150, [64, 9, 12, 16, 1, 10] * 150
    m = Made(lens, counts, hkv=1, group=4, d=d, page=32, seed=d, room=0)
    for i, bad in zip(range(5, m.total, 29), [INF, NAN, -INF, INF] * m.total):
        m.v_new[i, 0, i % d] = bad
    check_attend(kv, m)


def test_attend_visible_infinities(kv):
    m = Made([100, 100], [2, 2], seed=8)
    m.v[int(m.table[0, 1]), 1, 3, 7] = INF
    m.v[int(m.table[0, 2]), 0, 3, 7] = NAN
    check_attend(kv, m)
    m.q[0, 0, 0] = NAN
    check_attend(kv, m)


def test_attend_large_and_equal_scores(kv):
    """Scores far outside exp's range, and all the same."""
    m = Made([500, 77], [3, 40], group=4, d=128, seed=2)
    m.q *= 60
    check_attend(kv, m)
    m.k.zero_()
    m.k_new.zero_()
    check_attend(kv, m)


@pytest.mark.parametrize("group,tokens", [(1, 1), (8, 3), (1, 40), (4, 40)])
def test_attend_many_small_weights_in_half_precision(kv, group, tokens):
    """Each of 4,000 weights is 2^-25.2 of the largest, less than fp16's steps near 0; all of them are what the
    output consists of.  A weight counts down to 2^-31 at least: it may be off by 2^-32 (half a step), and the
    output by half a step of its own, 2^-25.  (The log-sum: 62 additions to about 1 in 32 bits, its own rounding.)"""
    n, sessions = 4000, 320  # so many that a CTA has whole sessions
    m = Made([0] * sessions, [tokens] * sessions, hkv=1, group=group, page=64, dtype="fp16", room=n + 64, seed=1)
    m.length.fill_(n)
    m.k.zero_()
    m.v.fill_(1)
    first = torch.from_numpy(m.table[:, 0]).long().cuda()
    m.k[first, 0, 0, 0], m.v[first, 0, 0] = 17.5, 0
    m.q.zero_()
    m.q[..., 0] = 1
    m.k_new.zero_()
    m.k_new[..., 0], m.v_new[:] = -100, 0
    out, lse = kv.attend(m.cache(kv), m.tree(kv), m.q, m.k_new, m.v_new, scale=1.0)
    small = (n - 1) * math.exp(-17.5)
    want = small / (1 + small)
    assert np.max(np.abs(f64(out) - want)) <= n * 2.0 ** -32 + 2.0 ** -25 + 2.0 ** -18 * want
    assert np.max(np.abs(f64(lse) - 17.5 - math.log1p(small))) <= 2.0 ** -17


@pytest.mark.parametrize("group,tokens", [(1, 1), (1, 40), (4, 40)])
@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
def test_attend_scores_beyond_24_bits(kv, group, tokens, dtype):
    """Scores from 2^16 to 2^26, ascending through the tiles and down again: the
    largest key has all the weight, whose value is the output as it is."""
    n = 900
    m = Made([n], [tokens], hkv=1, group=group, dtype=dtype, seed=4)
    s = torch.arange(n)
    at = torch.from_numpy(m.table[0]).long()[s // m.page].cuda(), 0, (s % m.page).cuda()
    size = 2.0 ** (torch.where(s < 700, s, 1399 - s).float() / 70)  # 1 .. 2^10, in steps of 1%
    m.k[at] = 0
    m.k[(*at, 0)] = size.to(m.k.dtype).cuda()
    keys = m.k[(*at, 0)].float()
    m.q.zero_()
    m.k_new.zero_()
    for q in (2.0 ** 13, 2.0 ** 14, 2.0 ** 15):
        m.q[..., 0] = q
        out, lse = kv.attend(m.cache(kv), m.tree(kv), m.q, m.k_new, m.v_new, scale=2.0)
        best = (keys == keys.max()).nonzero()[:, 0]
        want = m.v[at][best].double().mean(0)
        assert float((out.double() - want).abs().max()) <= float(want.abs().max()) * ref.UNIT[dtype] * 2
        assert float((lse / (2 * q * keys.max()) - 1).abs().max()) <= 2.0 ** -21


@pytest.mark.parametrize("scale", [0.0, -0.3, 2.5])
def test_attend_scale(kv, scale):
    check_attend(kv, Made([100, 3], [2, 30], group=4, seed=6), scale=scale)


def test_attend_strided_rows_stream_and_workspace(kv):
    m = Made([90, 700], [4, 6], group=4, hkv=2, d=64, seed=12)
    both = torch.full((m.total, 24, 80), NAN, dtype=torch.bfloat16, device="cuda")
    both[:, :8, :64], both[:, 8:10, :64], both[:, 10:12, :64] = m.q, m.k_new, m.v_new
    m.q, m.k_new, m.v_new = both[:, :8, :64], both[:, 8:10, :64], both[:, 10:12, :64]
    out = both[:, 12:20, :64]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    work = torch.full((kv.attend_workspace(m.cache(kv), m.tree(kv), 8),), 255, dtype=torch.uint8, device="cuda")
    side.wait_stream(torch.cuda.current_stream())
    check_attend(kv, m, out=out, workspace=work, stream=side)
    assert bool(both[:, 20:].isnan().all()) and bool(both[:, :, 64:].isnan().all())


def test_scratch_and_results_belong_to_the_given_stream(kv):
    m = Made([300, 41], [4, 2], group=4, hkv=2, d=64, seed=14)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    check_attend(kv, m, stream=side.cuda_stream)  # a raw handle
    cache, tree = m.cache(kv), m.tree(kv)
    with torch.cuda.stream(side):
        want = kv.attend(cache, tree, m.q, m.k_new, m.v_new)[0]
    for handle in (side, side.cuda_stream):
        got = kv.attend(cache, tree, m.q, m.k_new, m.v_new, stream=handle)[0]
        side.synchronize()
        assert torch.equal(got, want) and list(cache.scratch) == [side.cuda_stream]
    got = kv.attend(cache, tree, m.q, m.k_new, m.v_new, stream=0)[0]  # the default stream
    torch.cuda.synchronize()
    assert torch.equal(got, want) and list(cache.scratch) == [side.cuda_stream, 0]


def test_one_cache_on_two_streams_at_once(kv):
    """Each stream has scratch of its own: calls that overlap do not disturb each other."""
    m = Made([9000, 17, 900, 3000], [8, 1, 30, 5], group=4, d=128, page=64, seed=24)
    cache, tree = m.cache(kv), m.tree(kv)
    want = kv.attend(cache, tree, m.q, m.k_new, m.v_new)
    other = m.q.flip(0).contiguous()
    want_other = kv.attend(cache, tree, other, m.k_new, m.v_new)
    torch.cuda.synchronize()
    sides, got = [torch.cuda.Stream() for _ in range(2)], [[], []]
    for _ in range(10):
        for i, q in enumerate((m.q, other)):
            got[i].append(kv.attend(cache, tree, q, m.k_new, m.v_new, stream=sides[i]))
    torch.cuda.synchronize()
    for results, (out, lse) in zip(got, (want, want_other)):
        assert all(torch.equal(o, out) and torch.equal(x, lse) for o, x in results)
    work = [cache.scratch[s.cuda_stream] for s in sides]
    assert work[0].data_ptr() != work[1].data_ptr()


def test_attend_absent_pages_and_bad_values_are_reported(kv):
    m = Made([100, 50, 20], [2, 20, 3], group=4, page=16, seed=13)
    full = [m.slots(f64(x), 0) for x in (m.k, m.v)]
    m.page_table[0, 2] = -1                    # slots 32 .. 47 absent
    m.page_table[1, 0] = m.k.shape[0] + 100    # outside the pool
    m.length[2] = 1 << 30
    out, lse = kv.attend(m.cache(kv), m.tree(kv), m.q, m.k_new, m.v_new)
    assert m.status.tolist() == [-4, -4, -4]
    keep = [s for s in range(100) if not 32 <= s < 48]
    k, v = (np.concatenate([x[keep][:, 0], f64(n)[:1, 0]]) for x, n in zip(full, (m.k_new, m.v_new)))
    s = k @ f64(m.q)[0, 0] * m.scale
    w = np.exp(s - s.max())
    assert np.allclose(f64(out)[0, 0], w @ v / w.sum(), atol=0.02)
    assert math.isclose(float(lse[0, 0]), s.max() + math.log(w.sum()), abs_tol=1e-4)


def _without_page(m, b, page):
    """Session b loses a page: its slots count as absent, for the kernels by the
    table, for the reference by leaving them out."""
    ref_m = Made.__new__(Made)
    ref_m.__dict__.update(m.__dict__)
    m.page_table[b, page] = -1
    ref_m.table = m.table.copy()
    ref_m.table[b, page:-1] = m.table[b, page + 1:]
    ref_m.lens = list(m.lens)
    ref_m.lens[b] -= m.page
    return ref_m


@pytest.mark.parametrize("page", [8, 16, 32, 64, 128, 256, 24])
@pytest.mark.parametrize("group,d,layout", [(16, 128, "hnd"), (2, 64, "nhd")])
def test_absent_pages_in_the_middle(kv, page, group, d, layout):
    """A page that is missing inside tiles that are full otherwise, for attention
    of many and of few rows and for the observed weight."""
    m = Made([1500, 700], [9, 5], hkv=3, group=group, d=d, page=page, layout=layout, seed=page)
    start = m.mass.clone()
    r = _without_page(m, 0, 2)
    out, lse = kv.attend(m.cache(kv), m.tree(kv), m.q, m.k_new, m.v_new)
    want, want_lse, tol, tol_lse = ref.attend(r)
    assert np.max(np.abs(f64(out) - want) / (tol + 1e-30)) <= 1
    assert np.max(np.abs(f64(lse) - want_lse) / tol_lse) <= 1
    kv.observe(m.cache(kv), m.tree(kv), m.q, lse, m.k_new)
    added, bound, _, _ = ref.observe(r, lse)
    for b in range(2):
        s = np.arange(r.lens[b])
        at = (r.table[b, s // page], slice(None), s % page)
        got = (f64(m.mass) - f64(start))[at]
        assert np.all(np.abs(got - added[b]) <= bound[b] + 2.0 ** -22 * np.abs(f64(m.mass)[at]))
    assert m.status.tolist() == [-4, 0]


def test_attend_same_bits_again_and_in_a_graph(kv):
    m = Made([3000, 17, 900], [8, 1, 30], group=4, d=128, seed=14)
    cache, tree = m.cache(kv), m.tree(kv)
    a, al = kv.attend(cache, tree, m.q, m.k_new, m.v_new)
    out, lse = torch.zeros_like(a), torch.zeros_like(al)
    work = torch.empty(kv.attend_workspace(cache, tree, m.q.shape[1]), dtype=torch.uint8, device="cuda")
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        kv.attend(cache, tree, m.q, m.k_new, m.v_new, out=out, lse=lse, workspace=work)
    for _ in range(3):
        out.zero_()
        g.replay()
        assert torch.equal(a, out) and torch.equal(al, lse)


def test_attend_offsets_beyond_32_bits(kv):
    """A pool of more than 2^32 elements: the last pages are read where they are."""
    pages, page, d = 9000, 64, 128
    k = torch.zeros((pages, 64, page, d), dtype=torch.bfloat16, device="cuda")  # 4.7e9 elements
    m = Made([200], [2], hkv=2, group=4, d=d, page=page, seed=15)
    m.table[0, :4] = [pages - 1, 3, pages - 2, pages - 3]
    small, m.page_table = (m.k, m.v), torch.from_numpy(m.table).cuda()
    v = k.view(pages, 32, 2, page, d)
    for i, (name, off) in enumerate((("k", 30), ("v", 31))):
        pool = v[:, off]
        made = torch.randn((4, 2, page, d), device="cuda").to(torch.bfloat16)
        pool[torch.tensor([pages - 1, 3, pages - 2, pages - 3], device="cuda")] = made
        setattr(m, name, pool)
    del small
    cache = kv.Cache(m.k, m.v, m.page_table, m.length)
    out, lse = kv.attend(cache, m.tree(kv), m.q, m.k_new, m.v_new)
    used = [pages - 1, 3, pages - 2, pages - 3]
    m.k, m.v = (x[torch.tensor(used, device="cuda")] for x in (m.k, m.v))
    m.table[0, :4] = [0, 1, 2, 3]
    want, want_lse, tol, tol_lse = ref.attend(m)
    assert np.max(np.abs(f64(out) - want) / tol) <= 1 and np.max(np.abs(f64(lse) - want_lse) / tol_lse) <= 1


# ---------------------------------------------------------------- observe --
def check_observe(kv, m, paths=None, lse=None):
    cache, tree = m.cache(kv), m.tree(kv)
    if lse is None:
        lse = torch.from_numpy(ref.attend(m)[1]).float().cuda()
    path = n_path = None
    if paths is not None:
        path = torch.full((len(paths), tree.max_tokens), -1, dtype=torch.int32)
        for b, p in enumerate(paths):
            path[b, :len(p)] = torch.tensor(p, dtype=torch.int32)
        path, n_path = path.cuda(), torch.tensor([len(p) for p in paths], dtype=torch.int32, device="cuda")
    before = f64(m.mass)
    new = kv.observe(cache, tree, m.q, lse, m.k_new, path=path, n_path=n_path)
    torch.cuda.synchronize()
    assert not m.status.any()
    added, bound, want_new, bound_new = ref.observe(m, lse, paths)
    expect, tol = before.copy(), np.zeros(before.shape)
    for b, n in enumerate(m.lens):
        s = np.arange(n)
        at = (m.table[b, s // m.page], slice(None), s % m.page)
        expect[at] += added[b]
        tol[at] = bound[b] + 2.0 ** -23 * np.abs(expect[at])
    after = f64(m.mass)
    assert np.array_equal(after[tol == 0], before[tol == 0])  # slots that are not in use
    assert np.max(np.abs(after - expect)[tol > 0] / tol[tol > 0], initial=0) <= 1
    assert np.array_equal(f64(new) == 0, want_new == 0)
    assert np.max(np.abs(f64(new) - want_new) / (bound_new + 1e-30), initial=0) <= 1
    return new


@pytest.mark.parametrize("d", [8, 64, 96, 128, 256])
@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
def test_observe_head_sizes(kv, d, dtype):
    check_observe(kv, Made([0, 1, 63, 300], [1, 3, 2, 5], d=d, dtype=dtype, layout="nhd", seed=d))


@pytest.mark.parametrize("group,counts", [(1, [1, 1, 1]), (4, [64, 17, 2]), (8, [64, 33, 0]), (16, [64, 1, 3])])
@pytest.mark.parametrize("d", [64, 128, 256])
def test_observe_rows(kv, group, counts, d):
    """Query rows per KV head from 1 to 1024."""
    check_observe(kv, Made([70, 300, 129], counts, group=group, hkv=2, d=d, seed=group))


@pytest.mark.parametrize("page", [1, 7, 64, 100])
@pytest.mark.parametrize("group", [2, 16])
def test_observe_paths_pages_and_lengths(kv, page, group):
    lens = [0, 1, 64, 65, 127, 128, 129, 500]
    m = Made(lens, [9] * len(lens), page=page, group=group, hkv=1, seed=page)
    paths = [[0], [], [0, 1], [0, 2, 8], [3], list(range(9)), [0, 8], [0, 1, 5, 7]]
    check_observe(kv, m, paths)


def test_observe_many_sessions(kv):
    n = 300
    check_observe(kv, Made([(37 * i) % 150 for i in range(n)], [i % 4 for i in range(n)], hkv=1, group=2, seed=9))


def test_observe_long_context(kv):
    check_observe(kv, Made([30011], [7], hkv=1, group=4, d=128, page=64, seed=5))


@pytest.mark.parametrize("group", [4, 16])
def test_observe_rows_that_saw_nothing(kv, group):
    m = Made([0, 100], [20, 20], group=group, seed=3)
    lse = torch.from_numpy(ref.attend(m)[1]).float().cuda()
    lse[2], lse[25, 1] = -INF, -INF
    m.q[2] = NAN  # a row without weight gives none, whatever it holds
    check_observe(kv, m, lse=lse)


def test_observe_same_bits_again(kv):
    m = Made([3000, 17, 900], [8, 1, 30], group=4, d=128, seed=14)
    lse = torch.from_numpy(ref.attend(m)[1]).float().cuda()
    start = m.mass.clone()
    a = check_observe(kv, m, lse=lse)
    first = m.mass.clone()
    m.mass.copy_(start)
    b = kv.observe(m.cache(kv), m.tree(kv), m.q, lse, m.k_new)
    assert torch.equal(a, b) and torch.equal(first, m.mass)


@pytest.mark.parametrize("group,d", [(4, 64), (2, 256)])
def test_observe_reports_paths_with_other_nodes(kv, group, d):
    """Nodes that a session has not give no weight; they and clamped lengths are reported."""
    m = Made([150, 20, 5, 6, 7], [4] * 5, group=group, d=d, seed=2)
    path, n_path = _bad_paths()
    good = [[0, 2], [0, 2], [0, 1, 3], [0, 1, 2, 3], []]
    lse = torch.from_numpy(ref.attend(m)[1]).float().cuda()
    before = f64(m.mass)
    new = kv.observe(m.cache(kv), m.tree(kv), m.q, lse, m.k_new, path=path, n_path=n_path)
    assert m.status.tolist() == [-4, -4, 0, -4, -4]
    added, bound, want_new, bound_new = ref.observe(m, lse, good)
    for b, n in enumerate(m.lens):
        s = np.arange(n)
        at = (m.table[b, s // m.page], slice(None), s % m.page)
        got = f64(m.mass)[at]
        assert np.all(np.abs(got - before[at] - added[b]) <= bound[b] + 2.0 ** -23 * np.abs(got))
    assert np.all(np.abs(f64(new) - want_new) <= bound_new)


# ----------------------------------------------------------------- commit --
@pytest.mark.parametrize("page,layout", [(1, "hnd"), (7, "nhd"), (16, "hnd"), (64, "nhd")])
@pytest.mark.parametrize("d", [8, 96, 128])
def test_commit(kv, page, layout, d):
    lens = [0, 1, 15, 16, 40]
    m = Made(lens, [1, 4, 0, 9, 64], page=page, layout=layout, d=d, seed=1)
    paths = [[0], [0, 2], [], [], [0, 3, 9, 10, 63]]
    path = torch.full((5, 64), -1, dtype=torch.int32)
    for b, p in enumerate(paths):
        path[b, :len(p)] = torch.tensor(p, dtype=torch.int32)
    n_path = torch.tensor([len(p) for p in paths], dtype=torch.int32, device="cuda")
    new = torch.rand((m.total, m.hkv), device="cuda")
    want = {x: getattr(m, x).clone() for x in ("k", "v", "mass", "pos")}
    for b, p in enumerate(paths):
        for i, node in enumerate(p):
            s = lens[b] + i
            at = (int(m.table[b, s // page]), slice(None), s % page)
            row = m.off[b] + node
            want["k"][at], want["v"][at], want["mass"][at] = m.k_new[row], m.v_new[row], new[row]
            want["pos"][at] = lens[b] + 7 + i
    kv.commit(m.cache(kv), m.tree(kv), m.k_new, m.v_new, mass_new=new, path=path.cuda(), n_path=n_path)
    for x in want:
        a, b = getattr(m, x), want[x]
        assert torch.equal(a.nan_to_num(-9.0), b.nan_to_num(-9.0)) if a.is_floating_point() else torch.equal(a, b), x
    grown = [n + len(p) for n, p in zip(lens, paths)]
    assert m.length.tolist() == grown and m.next_pos.tolist() == [x + 7 for x in grown]
    assert m.status.tolist() == [0] * 5


def test_commit_without_path_marks_or_room(kv):
    m = Made([10, 30], [5, 6], page=8, room=6, seed=2, marks=False)
    m.page_table[1, 4] = -1  # slots 32 ..: session 1 has no room for six more
    before = m.k.clone()
    kv.commit(m.cache(kv), m.tree(kv), m.k_new, m.v_new)
    assert m.length.tolist() == [15, 30] and m.status.tolist() == [0, -9]
    for i in range(5):
        s = 10 + i
        assert torch.equal(m.k[int(m.table[0, s // 8]), :, s % 8], m.k_new[i])
    for page in m.table[1]:
        if page >= 0:
            assert torch.equal(m.k[int(page)].nan_to_num(-9.0), before[int(page)].nan_to_num(-9.0))


def _bad_paths():
    """(paths, lengths of paths) of five sessions of four tokens, the good one in the middle: a node behind the last
    one, a node below 0, a good path, more nodes than tokens, fewer than none."""
    path = torch.tensor([[0, 2, 4, -1], [0, -1, 2, -1], [0, 1, 3, -1], [0, 1, 2, 3], [0, 1, 2, 3]], dtype=torch.int32)
    return path.cuda(), torch.tensor([3, 3, 3, 7, -2], dtype=torch.int32, device="cuda")


@pytest.mark.parametrize("page", [1, 8])
def test_commit_refuses_paths_with_other_nodes(kv, page):
    """No slot counts that holds nothing: a session whose path names a node that
    it has not stays as it is; path lengths are clamped.  Both are reported."""
    lens = [10, 20, 5, 6, 7]
    m = Made(lens, [4] * 5, page=page, seed=2)
    path, n_path = _bad_paths()
    before = {x: getattr(m, x).clone() for x in ("k", "v", "mass", "pos")}
    kv.commit(m.cache(kv), m.tree(kv), m.k_new, m.v_new, path=path, n_path=n_path)
    assert m.length.tolist() == [10, 20, 8, 10, 7]
    assert m.next_pos.tolist() == [17, 27, 15, 17, 14]
    assert m.status.tolist() == [-4, -4, 0, -4, -4]
    for b, nodes in ((2, [0, 1, 3]), (3, [0, 1, 2, 3])):
        for i, node in enumerate(nodes):
            s = lens[b] + i
            at = (int(m.table[b, s // page]), slice(None), s % page)
            for x, new in (("k", m.k_new), ("v", m.v_new)):
                assert torch.equal(getattr(m, x)[at], new[m.off[b] + node])
            for x in before:
                before[x][at] = getattr(m, x)[at]
    for x, old in before.items():  # nothing else was written
        assert torch.equal(getattr(m, x).nan_to_num(-9.0), old.nan_to_num(-9.0)) if old.is_floating_point() else \
            torch.equal(getattr(m, x), old), x


# ------------------------------------------------------------------ evict --
def check_evict(kv, m, keep, sink, recent, into=None, marks=True):
    """Both forms against a sort of every session's and head's slots."""
    lens, table, page = m.length.tolist(), m.table, m.page
    mass, pos, k, v = f64(m.mass), m.pos.cpu().numpy(), m.k.clone(), m.v.clone()
    next_pos = m.next_pos.tolist()
    to = m if into is None else into
    want = {x: getattr(to, x).clone() for x in ("k", "v", "mass", "pos")}
    source = {"k": k, "v": v, "mass": m.mass.clone(), "pos": m.pos.clone()}
    n_kept = []
    for b, n in enumerate(lens):
        n_kept.append(max(0, min(n, keep[b])))
        at = lambda s, t: (int(t[b, s // page]), h, s % page)  # noqa: E731
        for h in range(m.hkv):
            w = np.array([mass[at(s, table)] for s in range(n)])
            p = np.array([pos[at(s, table)] for s in range(n)]) if marks else np.arange(n)
            stay = ref.kept(w, p, n, keep[b], sink, recent, next_pos[b] if marks else n)
            if into is None:
                free = [s for s in range(n_kept[b]) if s not in set(stay)]
                moves = list(zip([s for s in stay if s >= n_kept[b]], free))
            else:
                moves = list(zip(stay, range(len(stay))))
            for a, z in moves:
                for x in want:
                    t = to.table
                    want[x][int(t[b, z // to.page]), h, z % to.page] = source[x][at(a, table)]
    extra = {} if marks else dict(pos=None, next_pos=None)
    kv.evict(m.cache(kv, **extra), torch.tensor(keep, dtype=torch.int32, device="cuda"), sink=sink, recent=recent,
             into=None if into is None else into.cache(kv, **extra))
    torch.cuda.synchronize()
    for x in want:
        if x == "pos" and not marks:
            continue
        a, b = getattr(to, x), want[x]
        assert torch.equal(a.nan_to_num(-9.0), b.nan_to_num(-9.0)) if a.is_floating_point() else torch.equal(a, b), x
    assert to.length.tolist() == n_kept


def _plain_marks(m, ties=False, seed=0):
    r = np.random.default_rng(seed)
    for b, n in enumerate(m.lens):
        s = np.arange(n)
        at = (torch.from_numpy(m.table[b, s // m.page]).long().cuda(), slice(None),
              torch.from_numpy(s % m.page).long().cuda())
        m.pos[at] = torch.from_numpy(np.stack([r.permutation(n) for _ in range(m.hkv)], 1).astype(np.int32)).cuda()
        if ties:
            m.mass[at] = torch.from_numpy(r.integers(0, 3, (n, m.hkv)).astype(np.float32)).cuda()
    m.next_pos.copy_(m.length)


@pytest.mark.parametrize("page", [1, 7, 16, 64])
@pytest.mark.parametrize("ties", [False, True])
def test_evict_in_place(kv, page, ties):
    m = Made([0, 1, 5, 64, 65, 200, 300, 1030, 2100], [1] * 9, page=page, seed=page, room=1)
    _plain_marks(m, ties)
    check_evict(kv, m, [0, 0, 9, 64, 64, 100, 7, 1029, 1], 2, 5)


@pytest.mark.parametrize("ties", [False, True])
def test_evict_into_another_cache(kv, ties):
    lens = [0, 1, 5, 64, 65, 200, 300, 1030, 2100]
    keep = [0, 0, 9, 64, 64, 100, 7, 1029, -3]
    m = Made(lens, [1] * 9, page=16, seed=3, room=1, d=96, layout="nhd")
    _plain_marks(m, ties)
    into = Made([0] * 9, [1] * 9, page=24, room=1030, seed=4, d=96)
    into.lens = lens
    check_evict(kv, m, keep, 3, 11, into)
    assert into.next_pos.tolist() == m.next_pos.tolist() and m.length.tolist() == lens


def test_evict_special_weights(kv):
    """NaN goes first, then -inf; -0 is 0; equal weights keep the lower slot."""
    m = Made([40, 40], [1, 1], page=16, hkv=1, seed=5, room=1)
    _plain_marks(m)
    vals = torch.tensor([NAN, -INF, INF, -0.0, 0.0, 1e-45, -1.0, 3.0, NAN, 0.0] * 4)
    for b in range(2):
        s = torch.arange(40)
        m.mass[torch.from_numpy(m.table[b])[s // 16].long().cuda(), 0, (s % 16).cuda()] = vals.cuda()
    check_evict(kv, m, [13, 33], 0, 0)


def test_evict_protected_slots_fill_the_budget(kv):
    m = Made([100, 100], [1, 1], page=16, seed=6, room=1)
    _plain_marks(m)
    check_evict(kv, m, [10, 12], 8, 50)


def test_evict_without_positions(kv):
    m = Made([100, 2049], [1, 1], page=16, seed=7, room=1)
    check_evict(kv, m, [30, 2000], 4, 9, marks=False)


@pytest.mark.parametrize("page", [7, 16])  # slots one by one, and by four
@pytest.mark.parametrize("without", ["pos", "next_pos"])
@pytest.mark.parametrize("place", ["in", "into"])
def test_evict_with_half_of_the_positions(kv, page, without, place):
    """Positions count only where next_pos tells the next one: without either a
    slot's index is its position, whatever pos holds; pos moves along all the same."""
    lens, keep, sink, recent = [100, 60, 9], [40, 30, 9], 2, 5
    m = Made(lens, [1] * 3, page=page, seed=page, room=1)
    m.pos += 5000  # far above the lengths, as after many evictions
    to = m if place == "in" else Made([0] * 3, [1] * 3, page=16, room=40, seed=1)
    mass, pos, k = f64(m.mass), m.pos.clone(), m.k.clone()
    drop = {without: None}
    kv.evict(m.cache(kv, **drop), torch.tensor(keep, dtype=torch.int32, device="cuda"), sink=sink, recent=recent,
             into=None if place == "in" else to.cache(kv, **drop))
    assert to.length.tolist() == keep
    for b, n in enumerate(lens):
        for h in range(m.hkv):
            at = lambda s: (int(m.table[b, s // page]), h, s % page)  # noqa: B023, E731
            stay = ref.kept([mass[at(s)] for s in range(n)], range(n), n, keep[b], sink, recent, n)
            if place == "in":
                free = [s for s in range(keep[b]) if s not in stay]
                want = {s: s for s in stay if s < keep[b]} | dict(zip(free, [s for s in stay if s >= keep[b]]))
            else:
                want = dict(enumerate(stay))
            for z, a in want.items():
                there = (int(to.table[b, z // to.page]), h, z % to.page)
                assert torch.equal(to.k[there], k[at(a)])
                assert without == "pos" or int(to.pos[there]) == int(pos[at(a)])


def test_evict_into_a_cache_without_room(kv):
    m = Made([100, 60], [1, 1], page=16, seed=8, room=1)
    _plain_marks(m)
    into = Made([0, 0], [1, 1], page=16, room=32, seed=9)
    into.lens = [100, 60]
    kv.evict(m.cache(kv), torch.tensor([50, 20], dtype=torch.int32, device="cuda"), into=into.cache(kv))
    assert into.length.tolist() == [32, 20] and into.status.tolist() == [-9, 0]


@pytest.mark.parametrize("n,keep", [(40000, 39990), (40000, 13000), (131000, 100), (131000, 130999), (200000, 99999)])
@pytest.mark.parametrize("place", ["in", "into"])
def test_evict_long_sessions(kv, n, keep, place):
    """Selection against torch's sort, at lengths that no plain loop covers."""
    m = Made([0], [1], hkv=2, d=8, page=64, room=n, seed=n)
    m.length.fill_(n)
    m.lens = [n]
    m.k.copy_(torch.randn(m.k.shape).to(torch.bfloat16))
    m.v.copy_(-m.k)
    m.mass.copy_(torch.randint(0, 5000, m.mass.shape).float())
    m.next_pos.fill_(n)
    s = torch.arange(n)
    pages, off = torch.from_numpy(m.table[0])[s // 64].long().cuda(), (s % 64).cuda()
    m.pos[pages, :, off] = torch.arange(n, dtype=torch.int32, device="cuda")[:, None]
    w = m.mass[pages, :, off].clone()
    w[:5], w[n - 17:] = INF, INF
    stay = w.T.sort(dim=1, descending=True, stable=True).indices[:, :keep].sort(1).values
    old = m.k.clone()
    to = m if place == "in" else Made([0], [1], hkv=2, d=8, page=64, room=keep, seed=1)
    kv.evict(m.cache(kv), torch.tensor([keep], dtype=torch.int32, device="cuda"), sink=5, recent=17,
             into=None if place == "in" else to.cache(kv))
    assert int(to.length) == keep
    t = torch.arange(keep)
    to_page, to_off = torch.from_numpy(to.table[0])[t // 64].long().cuda(), (t % 64).cuda()
    for h in range(2):
        got = to.pos[to_page, h, to_off].long()  # = the slot that came here
        if place == "in":
            inside = stay[h] < keep
            want = torch.arange(keep, device="cuda")
            hole = torch.ones(keep, dtype=torch.bool, device="cuda")
            hole[stay[h][inside]] = False
            want[hole] = stay[h][~inside]
        else:
            want = stay[h]
        assert torch.equal(got, want)
        assert torch.equal(to.k[to_page, h, to_off], old[pages[want], h, off[want]])
        assert torch.equal(to.v[to_page, h, to_off], -old[pages[want], h, off[want]])


# ----------------------------------------------------------------- verify --
def _verify_inputs(counts, vocab, seed, sharp=3.0, near=0.7, dtype=torch.float32, tree=True):
    m = Made([0] * len(counts), counts, seed=seed, tree=tree, hkv=1, group=1, d=8)
    g = torch.Generator().manual_seed(seed)
    x = torch.randn((m.total, vocab), generator=g) * sharp
    p = torch.softmax(x, 1)
    q = torch.softmax(x + near * torch.randn((m.total, vocab), generator=g), 1)
    token = torch.zeros(m.total, dtype=torch.int32)
    for b, t in enumerate(counts):
        for i in range(1, t):
            row = int(m.off[b] + m.parent_np[m.off[b] + i])
            token[m.off[b] + i] = int(torch.multinomial(q[row], 1, generator=g))
    u, us = torch.rand(m.total, generator=g), torch.rand(len(counts), generator=g)
    return m, token, p.to(dtype), q.to(dtype), u, us


def check_verify(kv, m, token, p, q, u, us, want_q=True):
    tree = m.tree(kv)
    dev = lambda x: None if x is None else x.cuda()  # noqa: E731
    path, n_path, nxt = kv.verify(tree, dev(token), dev(p), dev(q), dev(u), dev(us))
    f = lambda x: None if x is None else x.float().numpy()  # noqa: E731
    want = ref.verify(m.counts, m.parent_np, token.numpy(), f(p), f(q), u.numpy(), us.numpy(), tree.max_tokens)
    assert np.array_equal(path.cpu().numpy(), want[0])
    assert np.array_equal(n_path.cpu().numpy(), want[1])
    assert np.array_equal(nxt.cpu().numpy(), want[2])
    return want


@pytest.mark.parametrize("vocab", [1, 2, 31, 33, 1000, 4097, 50001])
@pytest.mark.parametrize("tree", [False, True])
def test_verify_vocabularies(kv, vocab, tree):
    check_verify(kv, *_verify_inputs([1, 5, 9, 3], vocab, vocab, tree=tree))


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16, torch.float16])
@pytest.mark.parametrize("near", [0.0, 0.3, 3.0])
def test_verify_types_and_distances(kv, dtype, near):
    check_verify(kv, *_verify_inputs([64, 0, 1, 20, 33], 2000, 7, near=near, dtype=dtype))


def test_verify_certain_drafts(kv):
    m, token, p, _, u, us = _verify_inputs([20, 40, 8], 300, 11, sharp=2.0)
    check_verify(kv, m, token, p, None, u, us)


def test_verify_many_sessions_agree_with_the_target(kv):
    """One child per session, drawn from q: the emitted token follows p."""
    n, vocab = 20000, 7
    counts = [2] * n
    m = Made([0] * n, counts, seed=1, hkv=1, group=1, d=8, page=64, room=0)
    g = torch.Generator().manual_seed(5)
    p = torch.softmax(torch.randn(vocab, generator=g), 0)
    q = torch.softmax(torch.randn(vocab, generator=g), 0)
    token = torch.multinomial(q, 2 * n, replacement=True, generator=g).to(torch.int32)
    rows = lambda x: x[None].expand(2 * n, -1).contiguous().cuda()  # noqa: E731
    path, n_path, nxt = kv.verify(m.tree(kv), token.cuda(), rows(p), rows(q), torch.rand(2 * n, generator=g).cuda(),
                                  torch.rand(n, generator=g).cuda())
    first = torch.where(n_path.cpu() == 2, token[1::2], nxt.cpu())
    freq = torch.bincount(first.long(), minlength=vocab) / n
    assert float((freq - p).abs().max()) < 5 * math.sqrt(0.25 / n)


@pytest.mark.parametrize("siblings", [2, 3, 5])
def test_verify_siblings_agree_with_the_target(kv, siblings):
    """Several children of the root, drawn from q independently: the emitted token follows p all the same."""
    n, vocab, t = 20000, 7, siblings + 1
    m = Made([0] * n, [t] * n, seed=1, hkv=1, group=1, d=8, page=64, room=0)
    m.parent = torch.tensor([-1] + [0] * siblings, dtype=torch.int32).repeat(n).cuda()
    g = torch.Generator().manual_seed(siblings)
    p = torch.softmax(torch.randn(vocab, generator=g) * 1.5, 0)
    q = torch.softmax(torch.randn(vocab, generator=g) * 1.5, 0)
    token = torch.multinomial(q, n * t, replacement=True, generator=g).to(torch.int32)
    rows = lambda x: x[None].expand(n * t, -1).contiguous().cuda()  # noqa: E731
    path, n_path, nxt = kv.verify(m.tree(kv), token.cuda(), rows(p), rows(q), torch.rand(n * t, generator=g).cuda(),
                                  torch.rand(n, generator=g).cuda())
    path, n_path = path.cpu().long(), n_path.cpu()
    taken = token.view(n, t).gather(1, path[:, 1:2].clamp(min=0))[:, 0]
    first = torch.where(n_path == 2, taken, nxt.cpu())
    assert bool((n_path <= 2).all()) and bool((n_path == 1).any())
    freq = torch.bincount(first.long(), minlength=vocab) / n
    assert float((freq - p).abs().max()) < 5 * math.sqrt(0.25 / n)


def test_verify_rows_without_weight_and_bad_nodes(kv):
    m, token, p, q, u, us = _verify_inputs([6, 6, 6, 6, 6], 100, 13)
    p[m.off[0]] = 0
    p[m.off[1]], q[m.off[1]] = q[m.off[1]].clone(), q[m.off[1]].clone()  # residual of nothing
    u[m.off[1]:m.off[2]] = 1 - 2.0 ** -24
    p[m.off[2], 3], p[m.off[2], 4], q[m.off[2], 5] = NAN, INF, NAN
    token[m.off[3] + 1], token[m.off[3] + 2] = -1, 100  # passed over
    m.parent_np[m.off[4] + 1], m.parent_np[m.off[4] + 2] = 77, -5
    m.parent = torch.from_numpy(m.parent_np).cuda()
    p[m.off[0] + 1:m.off[1]] = 0
    want = check_verify(kv, m, token, p, q, u, us)
    assert want[2][0] == -1


def test_verify_rows_with_a_stride(kv):
    m, token, p, q, u, us = _verify_inputs([5, 9], 997, 17)
    wide = torch.full((m.total, 1021), NAN, device="cuda")
    wide[:, :997] = p.cuda()
    a = kv.verify(m.tree(kv), token.cuda(), wide[:, :997], q.cuda(), u.cuda(), us.cuda())
    b = kv.verify(m.tree(kv), token.cuda(), p.cuda(), q.cuda(), u.cuda(), us.cuda())
    assert all(torch.equal(x, y) for x, y in zip(a, b))


# ------------------------------------------------------------------- step --
def test_a_whole_step_without_synchronisation_and_in_a_graph(kv):
    """attend, verify, observe, commit, evict in one graph: replaying it runs
    the step on the state that the last one left."""
    def make():
        m = Made([200, 33, 0], [8, 8, 8], group=4, d=64, seed=21, room=64)
        _plain_marks(m)
        return m, *_verify_inputs([8, 8, 8], 500, 21)[1:]

    def step(m, token, p, q, u, us, hold):
        cache, tree = m.cache(kv), m.tree(kv)
        out, lse = kv.attend(cache, tree, m.q, m.k_new, m.v_new)
        path, n_path, nxt = kv.verify(tree, token, p, q, u, us)
        new = kv.observe(cache, tree, m.q, lse, m.k_new, path=path, n_path=n_path)
        kv.commit(cache, tree, m.k_new, m.v_new, mass_new=new, path=path, n_path=n_path)
        kv.evict(cache, hold, sink=2, recent=8)
        return out, nxt

    states = []
    for graph in (False, True):
        m, *rest = make()
        rest = [x.cuda() for x in rest]
        hold = torch.tensor([200, 40, 5], dtype=torch.int32, device="cuda")
        if graph:
            backup = {x: getattr(m, x).clone() for x in ("k", "v", "mass", "pos", "length", "next_pos")}
            step(m, *rest, hold)
            for x, y in backup.items():
                getattr(m, x).copy_(y)
            g = torch.cuda.CUDAGraph()
            with torch.cuda.graph(g):
                step(m, *rest, hold)
            for _ in range(4):
                g.replay()
        else:
            for _ in range(4):
                step(m, *rest, hold)
        torch.cuda.synchronize()
        states.append([getattr(m, x).nan_to_num(-9.0) if x in ("k", "v", "mass") else getattr(m, x)
                       for x in ("k", "v", "mass", "pos", "length", "next_pos", "status")])
    assert all(torch.equal(a, b) for a, b in zip(*states))
    assert states[0][4].tolist() == [200, 40, 5] and states[0][6].tolist() == [0, 0, 0]


def test_the_serving_example(kv):
    """examples/serving_step.py: budgets hold, positions are distinct, demoted
    sessions arrive with their most attended tokens."""
    import importlib.util
    import os
    path = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "serving_step.py")
    spec = importlib.util.spec_from_file_location("serving_step", path)
    example = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(example)
    r = example.main(sessions=5, steps=6, prompt_tokens=300, budget=256, quiet=True)
    fast, far = r["fast"], r["far"]
    assert fast.length.tolist() == [256] * 5
    assert [n > 0 for n in far.length.tolist()] == [b in r["victims"] for b in range(5)]
    assert fast.status.tolist() == [0] * 5 and far.status.tolist() == [0] * 5
    assert fast.next_pos.tolist() == (300 + r["told"]).tolist()
    assert bool(torch.isfinite(r["out"].float()).all())
    slot = torch.arange(256, device="cuda")
    for b in range(5):
        page = fast.page_table[b].long()[slot // 64]
        pos = fast.pos[page, :, slot % 64]
        for h in range(pos.shape[1]):
            assert pos[:, h].unique().numel() == 256
            assert set(range(4)) <= set(pos[:, h].tolist())  # the sink stayed
