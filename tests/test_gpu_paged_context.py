"""GPU parity of the attention over shared and over long contexts in the paged cache against its float64 oracle.

Tolerances count roundings, as in test_gpu_paged: a score is off by at most err, a probability by 2 err of itself, a float sum of n terms by
(n + 64) 2^-24 of the sum of magnitudes (twice, for the sums of parts and their joining); probabilities enter the bf16 products with all
their bits.  The result rounds once, by 2^-8 (bf16) or 2^-24 (float) of itself.  Bounds and selected pages have to be equal."""
import copy

import numpy as np
import pytest
import torch

from oracle import paged_context_oracle as pc
from oracle import paged_oracle as po
from paper_2505_24544_amd import binding as bx
from test_gpu_paged import DEV, HEADS, desc_for, dev, host, ints, make, on_gpu, pack, queries, stored, tdt, workspace

pytestmark = pytest.mark.gpu


def check(got, want, dtype, longest):
    (o, lse), (ref, rlse, spread, err) = got, want
    n = longest + 64
    e = err.transpose(0, 2, 1)[..., None]
    half = 2.0 ** -8 if dtype == "bf16" else 2.0 ** -24
    tol = half * np.abs(ref) + spread * (1 + half) * (2 * e + n * 2.0 ** -23) + 1e-37
    got, glse = host(o), host(lse)
    assert np.isfinite(got).all()
    assert (np.abs(got - ref) <= tol).all(), (np.abs(got - ref) / tol).max()
    seen = np.isfinite(rlse)
    assert np.array_equal(np.isneginf(glse), ~seen)
    far = np.abs(glse - np.where(seen, rlse, 0))[seen]
    assert (far <= (2 * err + n * 2.0 ** -23 + 2.0 ** -22 * np.abs(np.where(seen, rlse, 0)))[seen]).all(), far.max()


def outputs(B, M, H, d, dtype):
    return (torch.full((B, M, H, d), float("nan"), dtype=tdt(dtype), device=DEV),
            torch.full((B, H, M), float("nan"), dtype=torch.float32, device=DEV))


def shared(c, q, group_first, n_shared, dtype, *, slots=None, n_true=None, tree=None, scale=0.0, bound=1 << 20):
    B, M, H, d = q.shape
    t, handle = on_gpu(c, dtype)
    desc = desc_for(B, M, H, c["k"].shape[2], d, dtype, bound, softmax_scale=scale)
    o, lse = outputs(B, M, H, d, dtype)
    bits, words = (None, 0) if tree is None else pack(tree)
    bx.beagle_xattn_paged_attend_shared(desc, handle, dev(q, dtype), ints(slots), ints(group_first), ints(n_shared), len(n_shared),
                                        ints(n_true), bits, words, o, lse, workspace(desc, handle, bx.BEAGLE_WS_PAGED_SHARED))
    torch.cuda.synchronize()
    return o, lse


def check_shared(c, q, group_first, n_shared, dtype, **kw):
    print("shared", dtype, q.shape, c["k"].shape, group_first, n_shared, {k: v for k, v in kw.items() if k != "tree"}, flush=True)
    got = shared(c, q, group_first, n_shared, dtype, **kw)
    want = pc.attend_shared(c, q, group_first, n_shared, slots=kw.get("slots"), n_true=kw.get("n_true"), tree=kw.get("tree"),
                            scale=kw.get("scale") or None, bound=kw.get("bound"))
    check(got, want, dtype, max(c["lens"]))
    return got


def with_room(c, pages, dtype):
    c = dict(c, refs=c["refs"] + [0] * pages)
    for x in ("k", "v"):
        c[x] = np.concatenate((c[x], np.full((pages, *c[x].shape[1:]), np.nan)))
    return c


def branches(rng, prefixes, sizes, own, page, G, d, dtype):
    """Groups of branches of one sequence each: (cache, group_first, common rows)."""
    B = sum(sizes)
    longest = max(prefixes) + max(own)
    W = po.pages_of(longest, page) + 1
    lens, first, b = [0] * B, [0], 0
    for n, size in zip(prefixes, sizes):
        lens[b] = n
        b += size
        first.append(b)
    c = make(rng, lens, page, W, sum(po.pages_of(n, page) for n in prefixes) + sum(po.pages_of(x, page) + 1 for x in own) + 2, G, d, dtype)
    for g, n in enumerate(prefixes):
        c = po.fork(c, list(range(first[g] + 1, first[g + 1])), [first[g]] * (sizes[g] - 1))
    for s in range(B):
        if own[s]:
            x = [stored(1.28 * rng.standard_normal((1, own[s], G, d)), dtype) for _ in range(2)]
            c, short = po.append(c, *x, slots=[s])
            assert short == 0
    return c, first, list(prefixes)


# ------------------------------------------------------------------ common rows
@pytest.mark.parametrize("dtype,H,G,d", HEADS)
@pytest.mark.parametrize("M,page,prefixes,sizes,own", [
    (1, 16, [700], [4], [1, 33, 0, 64]),
    (3, 4, [129, 2, 64], [1, 3, 2], [5, 0, 1, 32, 31, 7]),
    (7, 64, [65, 300], [5, 2], [65, 1, 5, 128, 2, 0, 90])])
def test_branches(dtype, H, G, d, M, page, prefixes, sizes, own):
    rng = np.random.default_rng(hash((H, G, d, M)) % 1000)
    c, first, n = branches(rng, prefixes, sizes, own, page, G, d, dtype)
    check_shared(c, queries(rng, sum(sizes), M, H, d, dtype), first, n, dtype)


@pytest.mark.parametrize("dtype,H,G,d", [("bf16", 8, 2, 128), ("f32", 4, 2, 64)])
@pytest.mark.parametrize("n_shared", [[0, 0], [1, 1], [31, 32], [33, 100], [96, 0], [1000, 1 << 30], [-5, 2]])
def test_common_rows_of_any_number(dtype, H, G, d, n_shared):
    """More than the first entry holds, more than the others do, none; the sequences need not begin alike."""
    rng = np.random.default_rng(n_shared[0] & 1023)
    lens = [130, 100, 0, 33, 200, 64, 1]
    c = make(rng, lens, 16, 16, 60, G, d, dtype)
    check_shared(c, queries(rng, 7, 2, H, d, dtype), [0, 4, 7], n_shared, dtype)


@pytest.mark.parametrize("dtype,H,G,d", [("bf16", 4, 4, 128), ("f32", 6, 2, 20)])
@pytest.mark.parametrize("group_first", [[0, 6], [2, 4], [0, 0, 3, 3, 6], [1, 5, 2, 4], [4, 0, 9], [-1, 3, 100], [0, 1, 2, 3, 4, 5, 6], [6, 6]])
def test_groups_of_any_kind(dtype, H, G, d, group_first):
    rng = np.random.default_rng(len(group_first))
    lens = [90, 40, 77, 64, 100, 20]
    c = make(rng, lens, 8, 20, 70, G, d, dtype)
    n = [37, 64, 90, 5, 12, 50][: len(group_first) - 1]
    check_shared(c, queries(rng, 6, 1, H, d, dtype), group_first, n, dtype, slots=[3, 0, -1, 5, 5, 9])


@pytest.mark.parametrize("dtype,H,G,d", [("bf16", 8, 2, 128), ("bf16", 4, 4, 128), ("f32", 4, 2, 64), ("f32", 3, 3, 128)])
@pytest.mark.parametrize("M,T", [(2, 1), (10, 50), (4, 70)])
def test_trees_behind_common_rows(dtype, H, G, d, M, T):
    rng = np.random.default_rng(M + T)
    c, first, n = branches(rng, [130, 45], [3, 2], [T + 20, T, T + 1, T + 64, T + 33], 16, G, d, dtype)
    tree = rng.random((5, M, T)) < 0.4
    tree[1, 0] = False
    n_true = [x - T for x in c["lens"]]
    check_shared(c, queries(rng, 5, M, H, d, dtype), first, n, dtype, n_true=n_true, tree=tree)
    # true rows that end inside, before and at the end of the common ones
    check_shared(c, queries(rng, 5, M, H, d, dtype), first, n, dtype, n_true=[130, 100, 0, 45, -3], tree=tree)
    check_shared(c, queries(rng, 5, M, H, d, dtype), first, n, dtype, n_true=n_true, tree=None)


@pytest.mark.parametrize("bound", [1, 40, 64, 150])
def test_no_row_from_the_longest_length_on_is_seen(bound):
    rng = np.random.default_rng(bound)
    c, first, n = branches(rng, [100], [3], [60, 1, 33], 16, 2, 128, "bf16")
    check_shared(c, queries(rng, 3, 2, 8, 128, "bf16"), first, n, "bf16", bound=bound)


@pytest.mark.parametrize("dtype,H,G,d", [("bf16", 8, 2, 128), ("f32", 4, 2, 64)])
@pytest.mark.parametrize("scale", [1e-30, 3.0, 40.0])
def test_peaked_and_flat_scores(dtype, H, G, d, scale):
    rng = np.random.default_rng(int(scale))
    c, first, n = branches(rng, [200], [3], [40, 70, 9], 16, G, d, dtype)
    check_shared(c, queries(rng, 3, 2, H, d, dtype), first, n, dtype, scale=scale)


@pytest.mark.parametrize("dtype,H,G,d", [("bf16", 32, 8, 128), ("f32", 8, 4, 64)])
def test_many_queries_over_common_rows(dtype, H, G, d):
    """Several blocks of query rows, several cuts of the rows, ends inside of both."""
    rng = np.random.default_rng(3)
    sizes = [13, 1, 6]
    c, first, n = branches(rng, [1700, 900, 333], sizes, [int(x) for x in rng.integers(0, 90, 20)], 32, G, d, dtype)
    check_shared(c, queries(rng, 20, 3, H, d, dtype), first, n, dtype)


def test_more_groups_and_entries_than_the_plan_has_threads():
    rng = np.random.default_rng(5)
    B = 2300
    lens = [int(x) for x in rng.integers(0, 12, B)]
    c = make(rng, lens, 4, 3, sum(po.pages_of(n, 4) for n in lens) + 1, 1, 16, "f32")
    first = sorted(int(x) for x in rng.integers(0, B, 1100))
    n = [int(x) for x in rng.integers(0, 10, len(first) - 1)]
    check_shared(c, queries(rng, B, 1, 1, 16, "f32"), first, n, "f32")


def poison(c, rows, what=(np.nan, np.inf, -np.inf)):
    """K and V of these (page, row) hold what is no number.  (Steps of rows that only some queries see add them up row by row then, in
    another order: such results are held against the oracle, not against the bits that they have without.)"""
    for i, (p, r) in enumerate(rows):
        c["k"][p, r], c["v"][p, r] = what[i % len(what)], what[(i + 1) % len(what)]


@pytest.mark.parametrize("dtype,H,G,d", [("bf16", 4, 2, 128), ("f32", 4, 2, 64)])
def test_what_nobody_sees_does_not_matter(dtype, H, G, d):
    rng = np.random.default_rng(9)
    c = make(rng, [200, 150, 170, 90], 16, 14, 60, G, d, dtype)
    # entry 1 .. 3 take rows 0 .. 69 from slot 0: their own ones there are not seen, nor slot 0's drafted ones
    clean = copy.deepcopy(c)
    for s in (1, 2, 3):
        poison(c, po.rows_of(c, s, 70))
    q, n_true = queries(rng, 4, 2, H, d, dtype), [190, 150, 75, 60]
    tree = np.zeros((4, 2, 95), bool)
    tree[2, :, 3] = tree[3, 0, 29] = True
    poison(c, po.rows_of(c, 0, 200)[190:])
    check_shared(c, q, [0, 4], [70], dtype, n_true=n_true, tree=tree)
    # an entry with fewer true rows than the group has common ones does not see the rest of them, whatever it holds
    poison(c, po.rows_of(c, 0, 70)[60:])
    got = shared(c, q, [0, 4], [70], dtype, n_true=n_true, tree=tree)
    want = pc.attend_shared(clean, q, [0, 4], [70], n_true=n_true, tree=tree)
    check([x[3:] for x in got], [x[3:] for x in want], dtype, 200)


@pytest.mark.parametrize("dtype,H,G,d", [("bf16", 4, 2, 128), ("f32", 4, 2, 64)])
def test_page_numbers_outside_the_pool(dtype, H, G, d):
    rng = np.random.default_rng(10)
    c, first, n = branches(rng, [200], [3], [40, 70, 9], 16, G, d, dtype)
    c["table"][0][2], c["table"][0][5], c["table"][1][13], c["table"][2][0] = -1, len(c["refs"]), 1 << 30, -(1 << 31)
    check_shared(c, queries(rng, 3, 2, H, d, dtype), first, n, dtype)


# Groups of many query rows: 4 heads a kv head, one query, so 9 entries have 36 query rows, 50 have 200.
@pytest.mark.parametrize("entries", [8, 9, 16, 17, 32, 33, 50])
@pytest.mark.parametrize("rows,page", [(1, 16), (31, 4), (64, 64), (65, 128), (200, 4), (333, 16), (1000, 32)])
def test_groups_of_many_query_rows(entries, rows, page):
    rng = np.random.default_rng(entries + rows)
    c, first, n = branches(rng, [rows], [entries], [int(x) for x in rng.integers(0, 40, entries)], page, 2, 128, "bf16")
    check_shared(c, queries(rng, entries, 1, 8, 128, "bf16"), first, n, "bf16")


@pytest.mark.parametrize("sizes,M", [([40, 3, 0, 25, 1], 2), ([9, 1, 2], 5), ([70, 70], 1), ([30, 12], 6), ([2, 1], 40)])
def test_common_rows_that_end_inside_a_tile_for_some(sizes, M):
    """Few true rows, none, short and empty sequences among the many of a group."""
    rng = np.random.default_rng(sum(sizes))
    B = sum(sizes)
    longest = [500, 70, 64, 130, 33][: len(sizes)]
    c, first, n = branches(rng, [x for x, k in zip(longest, sizes) if k], [k for k in sizes if k], [int(x) for x in rng.integers(0, 40, B)], 8, 2, 128, "bf16")
    first, n = [0] + list(np.cumsum(sizes)), longest
    slots, n_true = list(range(B)), [int(x) for x in rng.integers(-5, 540, B)]
    for b in range(1, B, 5):
        slots[b] = int(rng.integers(-1, B + 2))
    tree = rng.random((B, M, 40)) < 0.4
    q = queries(rng, B, M, 8, 128, "bf16")
    check_shared(c, q, first, n, "bf16", slots=slots, n_true=n_true, tree=tree)
    check_shared(c, q, first, n, "bf16", slots=slots)
    check_shared(c, q, first, n, "bf16", slots=slots, bound=65)


@pytest.mark.parametrize("entries", [12, 40])
@pytest.mark.parametrize("scale", [1e-30, 3.0, 40.0])
def test_peaked_and_flat_scores_of_many_query_rows(entries, scale):
    rng = np.random.default_rng(int(scale))
    c, first, n = branches(rng, [700], [entries], [int(x) for x in rng.integers(0, 20, entries)], 16, 2, 128, "bf16")
    check_shared(c, queries(rng, entries, 1, 8, 128, "bf16"), first, n, "bf16", scale=scale)


@pytest.mark.parametrize("entries", [12, 40])
def test_growing_scores_of_many_query_rows(entries):
    """Every row's score is above all before it, by less and by more than the reference may lag behind."""
    rng = np.random.default_rng(entries)
    c, first, n = branches(rng, [600], [entries], [3] * entries, 16, 2, 128, "bf16")
    q = queries(rng, entries, 1, 8, 128, "bf16")
    q[:] = np.sign(q)
    q[1:] = q[:1]
    k = stored(np.arange(600)[:, None, None] / 150.0 * q[0, 0, ::4][None], "bf16")
    for (p, r), row in zip(po.rows_of(c, 0, 600), k):
        c["k"][p, r] = row
    for scale in (0.02, 0.2, 2.0):
        check_shared(c, q, first, n, "bf16", scale=scale)


@pytest.mark.parametrize("entries", [8, 12, 40])
def test_the_largest_values_of_many_query_rows(entries):
    """The row with the largest values is a hundred times as probable as those before it: times that they leave a float's range."""
    rng = np.random.default_rng(entries)
    c, first, n = branches(rng, [300], [entries], [5] * entries, 16, 2, 128, "bf16")
    q = np.sign(queries(rng, 1, 1, 8, 128, "bf16"))
    q[:, :, 1:4], q[:, :, 5:] = q[:, :, :1], q[:, :, 4:5]
    for b in range(entries):
        for p, r in po.rows_of(c, b, 305):
            c["k"][p, r] = 0.0
    p, r = po.rows_of(c, 0, 300)[200]
    c["k"][p, r], c["v"][p, r] = stored(q[0, 0, ::4] * (4.8 / 128), "bf16"), stored(np.full((2, 128), 3e38), "bf16")
    check_shared(c, np.repeat(q, entries, 0), first, n, "bf16", scale=1.0)


@pytest.mark.parametrize("entries", [12, 40])
def test_what_some_of_many_query_rows_do_not_see(entries):
    rng = np.random.default_rng(entries)
    c, first, n = branches(rng, [300], [entries], [5] * entries, 16, 2, 128, "bf16")
    clean = copy.deepcopy(c)
    q, n_true = queries(rng, entries, 1, 8, 128, "bf16"), [290] + [int(x) for x in rng.integers(0, 250, entries - 1)]
    poison(c, po.rows_of(c, 0, 300)[290:])
    check_shared(c, q, first, n, "bf16", n_true=n_true)
    poison(c, po.rows_of(c, 0, 300)[250:])
    got = shared(c, q, first, n, "bf16", n_true=n_true)
    want = pc.attend_shared(clean, q, first, n, n_true=n_true)
    check([x[1:] for x in got], [x[1:] for x in want], "bf16", 305)
    assert torch.isnan(got[0][0]).all()
    # one infinite value that some see: theirs has no bound there, and nobody else's
    c = copy.deepcopy(clean)
    p, r = po.rows_of(c, 0, 300)[100]
    c["v"][p, r, 1, 7] = -np.inf
    got = shared(c, q, first, n, "bf16", n_true=n_true)
    sees = torch.tensor([x > 100 for x in n_true], device=DEV)
    assert torch.equal(~torch.isfinite(got[0][:, 0, 4:, 7]), sees[:, None].expand(entries, 4))
    got[0][:, 0, 4:, 7] = 0
    want[0][:, 0, 4:, 7] = 0
    check(got, want, "bf16", 305)


@pytest.mark.parametrize("entries", [12, 40])
def test_page_numbers_outside_the_pool_of_many_query_rows(entries):
    rng = np.random.default_rng(entries)
    c, first, n = branches(rng, [300], [entries], [5] * entries, 16, 2, 128, "bf16")
    c["table"][0][2], c["table"][0][5], c["table"][0][18], c["table"][3][17] = -1, len(c["refs"]), 1 << 30, -(1 << 31)
    check_shared(c, queries(rng, entries, 1, 8, 128, "bf16"), first, n, "bf16")


@pytest.mark.parametrize("M,groups", [(36, 700), (130, 300)])
def test_units_of_more_pages_than_are_held_at_a_time(M, groups):
    """More groups than workgroups: each takes its 9000 rows of pages of 4 at once.  All groups see the same: one is checked, the others are equal."""
    rng = np.random.default_rng(M)
    c = make(rng, [9100], 4, 2275, 2280, 1, 128, "bf16")
    q = queries(rng, 1, M, 1, 128, "bf16")
    n_true = [9050]
    one = pc.attend_shared(c, q, [0, 1], [9000], n_true=n_true)
    o, lse = shared(c, np.repeat(q, groups, 0), list(range(groups + 1)), [9000] * groups, "bf16", slots=[0] * groups, n_true=n_true * groups)
    check((o[:1], lse[:1]), one, "bf16", 9100)
    assert torch.equal(o, o[:1].expand_as(o)) and torch.equal(lse, lse[:1].expand_as(lse))


@pytest.mark.parametrize("B,groups,M", [(63, 62, 1), (64, 63, 1), (64, 64, 1), (65, 3, 1), (64, 2, 512), (64, 2, 513), (7, 2, 6000)])
def test_either_plan(B, groups, M):
    """On both sides of what one wave plans for."""
    rng = np.random.default_rng(B + M)
    c = make(rng, [int(x) for x in rng.integers(0, 70, B)], 8, 10, 700, 1, 128, "bf16")
    first = [0] + sorted(int(x) for x in rng.integers(0, B, groups - 1)) + [B]
    check_shared(c, queries(rng, B, M, 1, 128, "bf16"), first, [int(x) for x in rng.integers(0, 90, groups)], "bf16")


# ------------------------------------------------------------------ bounds
def bounds(c, before, slots, dtype, first=None, bound=1 << 20):
    t, handle = on_gpu(c, dtype)
    G, d = c["k"].shape[2:]
    out = dev(before, dtype)
    bx.beagle_xattn_paged_bounds(desc_for(len(slots), 1, G, G, d, dtype, bound), handle, ints(slots), ints(first), out)
    torch.cuda.synchronize()
    return out


@pytest.mark.parametrize("dtype,G,d", [("bf16", 2, 128), ("bf16", 9, 128), ("f32", 3, 20), ("f32", 2, 64), ("f32", 1, 4), ("f32", 5, 100)])
@pytest.mark.parametrize("page", [4, 8, 64, 256])
def test_bounds(dtype, G, d, page):
    rng = np.random.default_rng(page + G)
    lens = [0, 1, page - 1, page, page + 1, 5 * page + 3, 3 * page]
    c = make(rng, lens, page, 8, 20, G, d, dtype)
    c["table"][6][1] = -1
    c["table"][5][0] = 20
    k = c["k"][c["table"][5][2]]
    k[1, 0, 0], k[2, 0, 1], k[0, 0, 2], k[:, 0, 3] = np.nan, np.inf, -np.inf, np.nan
    before = stored(rng.standard_normal((20, G, 2, d)), dtype)
    slots, first = [5, 0, 1, 2, 3, -1, 6, 4, 5, 7], [page + 1, 0, 0, 0, 0, 0, -3, page, 4 * page, 0]
    for f in (first, None):
        got = host(bounds(c, before, slots, dtype, f))
        assert np.array_equal(got, pc.bounds(c, before, slots=slots, first=f))
    got = host(bounds(c, before, slots, dtype, None, 2 * page + 1))
    assert np.array_equal(got, pc.bounds(c, before, slots=slots, bound=2 * page + 1))


# ------------------------------------------------------------------ selection
def select(c, q, b, window, sinks, n_select, dtype, *, slots=None, n_true=None, bound=1 << 20):
    B, M, H, d = q.shape
    G = c["k"].shape[2]
    t, handle = on_gpu(c, dtype)
    desc = desc_for(B, M, H, G, d, dtype, bound)
    pages = torch.full((B, G, n_select), 77, dtype=torch.int32, device=DEV)
    bx.beagle_xattn_paged_select(desc, handle, dev(q, dtype), ints(slots), ints(n_true), dev(b, dtype), window, sinks, n_select, pages,
                                 workspace(desc, handle, bx.BEAGLE_WS_PAGED_SELECT))
    torch.cuda.synchronize()
    return pages


def check_select(c, q, b, window, sinks, n_select, dtype, **kw):
    print("select", dtype, q.shape, c["k"].shape, window, sinks, n_select, kw, flush=True)
    got = select(c, q, b, window, sinks, n_select, dtype, **kw).cpu().numpy()
    want = pc.select(c, q, b, window, sinks, n_select, **kw)
    assert np.array_equal(got, want), np.argwhere(got != want)[:5]


def bounds_of(c):
    with np.errstate(all="ignore"):
        return np.nan_to_num(np.stack((c["k"].min(1), c["k"].max(1)), 2), nan=0.5)


@pytest.mark.parametrize("dtype,H,G,d", HEADS)
@pytest.mark.parametrize("M,window,sinks,n_select", [(1, 0, 0, 5), (3, 40, 9, 1), (7, 100, 1, 16), (2, 3, 4, 64), (2, 5000, 0, 3), (2, 0, 5000, 3)])
def test_selected_pages(dtype, H, G, d, M, window, sinks, n_select):
    rng = np.random.default_rng(M + n_select)
    lens = [900, 0, 3, 40, 333, 512]
    c = make(rng, lens, 8, 120, sum(po.pages_of(n, 8) for n in lens) + 2, G, d, dtype)
    q = queries(rng, 6, M, H, d, dtype)
    check_select(c, q, bounds_of(c), window, sinks, n_select, dtype)
    check_select(c, q, bounds_of(c), window, sinks, n_select, dtype, slots=[4, 0, 9, 0, -1, 2], n_true=[300, 850, 3, 0, 5, -1], bound=600)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_equal_and_odd_scores(dtype):
    rng = np.random.default_rng(2)
    c = make(rng, [4000, 2777], 4, 1000, 1700, 2, 128, dtype)
    q = queries(rng, 2, 2, 4, 128, dtype)
    b = np.repeat(np.round(rng.standard_normal((17, 2, 2, 128))), 100, 0)           # a hundred pages of each
    for n in (1, 99, 100, 101, 257, 600):
        check_select(c, q, b, 0, 0, n, dtype)
    check_select(c, q, np.zeros_like(b), 4, 4, 300, dtype)
    b = rng.standard_normal(b.shape)
    b[::3, 0, 0, :5], b[::5, 1, 1, 7], b[1::4, :, 0, 9], b[2::9, 1] = np.inf, -np.inf, np.nan, np.nan
    b = stored(b, dtype)
    q[0, 0, 0, :3], q[1, 1, 2, 5], q[0, 1, 1, 9], q[1, 0, :, ::2] = 0.0, np.inf, np.nan, 0.0
    c["table"][0][11], c["table"][1][600] = -1, 1 << 20
    for n in (3, 333, 900):
        check_select(c, q, b, 16, 0, n, dtype)


@pytest.mark.parametrize("dtype,H,G,d", [("bf16", 8, 2, 128), ("f32", 4, 2, 100)])
@pytest.mark.parametrize("q_scale,b_scale", [(1e-15, 1e-12), (1e-30, 1e-5), (1e12, 1e15), (1e-10, 1e30), (1e18, 1e18), (1e-38, 1e36)])
def test_scores_of_any_size(dtype, H, G, d, q_scale, b_scale):
    """Squares and products that leave a float's range on either side; channels of very different size."""
    rng = np.random.default_rng(7)
    c = make(rng, [3000, 1200], 8, 380, 530, G, d, dtype)
    q, b = queries(rng, 2, 2, H, d, dtype) * q_scale, bounds_of(c) * b_scale
    q, b = stored(q, dtype), stored(b, dtype)
    check_select(c, q, b, 16, 4, 60, dtype)
    b[::2, :, :, ::9] *= 2.0 ** -20
    q[:, :, 1] *= 2.0 ** -30
    check_select(c, stored(q, dtype), stored(b, dtype), 16, 4, 60, dtype)


@pytest.mark.parametrize("B,G,rows", [(9, 8, 530), (3, 2, 5000), (1, 1, 66000)])
def test_either_way_of_selection(B, G, rows):
    """A launch for all heads, or two, with fewer and more pages than a workgroup holds, whole and in part."""
    rng = np.random.default_rng(B)
    c = make(rng, [rows - 37 * b for b in range(B)], 8, rows // 8 + 2, B * rows // 8 + 8, G, 128, "bf16")
    b = stored(np.abs(rng.standard_normal((len(c["refs"]), G, 2, 128))) * [[-1.0], [1.0]], "bf16")
    for M, n in ((1, 3), (5, 33)):
        check_select(c, queries(rng, B, M, 4 * G, 128, "bf16"), b, 64, 4, n, "bf16")


def test_many_query_rows_and_pages():
    rng = np.random.default_rng(6)
    c = make(rng, [2600, 131], 4, 700, 720, 1, 128, "bf16")
    check_select(c, queries(rng, 2, 9, 5, 128, "bf16"), bounds_of(c), 64, 4, 37, "bf16")       # 45 rows: several tiles of queries


# ------------------------------------------------------------------ attention over listed pages
def blocks(c, q, lists, window, sinks, dtype, *, slots=None, n_true=None, tree=None, scale=0.0, bound=1 << 20):
    B, M, H, d = q.shape
    t, handle = on_gpu(c, dtype)
    desc = desc_for(B, M, H, c["k"].shape[2], d, dtype, bound, softmax_scale=scale)
    o, lse = outputs(B, M, H, d, dtype)
    bits, words = (None, 0) if tree is None else pack(tree)
    lists = torch.tensor(np.asarray(lists), dtype=torch.int32, device=DEV)
    bx.beagle_xattn_paged_attend_blocks(desc, handle, dev(q, dtype), ints(slots), ints(n_true), bits, words, window, sinks, lists,
                                        lists.shape[2], o, lse, workspace(desc, handle, bx.BEAGLE_WS_PAGED_BLOCKS))
    torch.cuda.synchronize()
    return o, lse


def check_blocks(c, q, lists, window, sinks, dtype, **kw):
    print("blocks", dtype, q.shape, c["k"].shape, np.shape(lists), window, sinks, {k: v for k, v in kw.items() if k != "tree"}, flush=True)
    got = blocks(c, q, lists, window, sinks, dtype, **kw)
    want = pc.attend_blocks(c, q, lists, window, sinks, slots=kw.get("slots"), n_true=kw.get("n_true"), tree=kw.get("tree"),
                            scale=kw.get("scale") or None, bound=kw.get("bound"))
    check(got, want, dtype, max(c["lens"]))
    return got


def some_pages(rng, c, B, G, n, window, sinks, slots=None, n_true=None, bound=1 << 20):
    out = np.full((B, G, n), -1)
    for b in range(B):
        held = min(po.length(c, b if slots is None else slots[b]), bound)
        nt = held if n_true is None else min(max(n_true[b], 0), held)
        lo, hi = pc.span(nt, window, sinks, c["k"].shape[1])
        for g in range(G):
            mine = sorted(int(x) for x in rng.permutation(np.arange(lo, hi))[:n])
            out[b, g, : len(mine)] = mine
    return out


@pytest.mark.parametrize("dtype,H,G,d", HEADS)
@pytest.mark.parametrize("M,page,window,sinks,n", [(1, 16, 0, 0, 5), (3, 4, 40, 9, 20), (7, 64, 100, 1, 3), (2, 8, 0, 3, 200), (2, 128, 300, 0, 2)])
def test_listed_pages(dtype, H, G, d, M, page, window, sinks, n):
    rng = np.random.default_rng(hash((H, G, d, M)) % 1000)
    lens = [900, 0, 3, page, 333, 2 * page + 1]
    c = make(rng, lens, page, po.pages_of(900, page), sum(po.pages_of(x, page) for x in lens) + 3, G, d, dtype)
    q = queries(rng, 6, M, H, d, dtype)
    check_blocks(c, q, some_pages(rng, c, 6, G, n, window, sinks), window, sinks, dtype)
    kw = dict(slots=[4, 0, 9, 0, -1, 2], bound=600)
    check_blocks(c, q, some_pages(rng, c, 6, G, n, window, sinks, **kw), window, sinks, dtype, **kw)


@pytest.mark.parametrize("dtype,H,G,d", [("bf16", 8, 2, 128), ("bf16", 4, 4, 128), ("f32", 4, 2, 64), ("f32", 3, 3, 128)])
@pytest.mark.parametrize("M,T,window", [(2, 1, 0), (10, 50, 33), (4, 70, 16)])
def test_trees_behind_listed_pages(dtype, H, G, d, M, T, window):
    rng = np.random.default_rng(M + T)
    c = make(rng, [400, 301, 150, T, 16], 16, 30, 90, G, d, dtype)
    tree = rng.random((5, M, T)) < 0.4
    tree[1, 0] = False
    n_true = [400 - T, 301, 150 - T, 0, -3]
    lists = some_pages(rng, c, 5, G, 6, window, 4, n_true=n_true)
    check_blocks(c, queries(rng, 5, M, H, d, dtype), lists, window, 4, dtype, n_true=n_true, tree=tree)
    check_blocks(c, queries(rng, 5, M, H, d, dtype), lists, window, 4, dtype, n_true=n_true, tree=None)


@pytest.mark.parametrize("dtype,H,G,d", [("bf16", 4, 2, 128), ("f32", 4, 2, 64)])
def test_lists_of_any_content(dtype, H, G, d):
    rng = np.random.default_rng(4)
    c = make(rng, [300, 290], 8, 40, 90, G, d, dtype)
    c["table"][1][9], c["table"][0][20] = -1, 1 << 29
    lists = np.array([[[5, 5, 7, 3, 9, -1, 20, 1 << 30], [-1] * 8],
                      [[0, 1, 2, 3, 4, 5, 9, 36], [-(1 << 31), (1 << 31) - 1, 8, 9, 10, 33, 34, 35]]])
    check_blocks(c, queries(rng, 2, 2, H, d, dtype), lists, 20, 9, dtype)
    for _ in range(4):
        check_blocks(c, queries(rng, 2, 2, H, d, dtype), rng.integers(-5, 45, (2, G, 12)), 20, 9, dtype)


@pytest.mark.parametrize("dtype,H,G,d,B", [("bf16", 4, 4, 128, 1), ("bf16", 8, 2, 128, 7), ("f32", 4, 1, 64, 2)])
def test_more_pages_than_are_held_at_a_time(dtype, H, G, d, B):
    rng = np.random.default_rng(8)
    n = 9000 if B == 1 else 5200
    lens = [n - 700 * i for i in range(B)]
    c = make(rng, lens, 4, n // 4, sum(lens) // 4 + 20, G, d, dtype)
    q = queries(rng, B, 1, H, d, dtype)
    check_blocks(c, q, some_pages(rng, c, B, G, 1100, 500, 5), 500, 5, dtype)


@pytest.mark.parametrize("dtype,H,G,d", [("bf16", 4, 2, 128), ("f32", 4, 2, 64)])
def test_pages_that_are_not_listed_do_not_matter(dtype, H, G, d):
    rng = np.random.default_rng(12)
    c = make(rng, [300], 8, 40, 50, G, d, dtype)
    lists = [[[3, 7, 8], [7, 20, 30]]]
    q = queries(rng, 1, 2, H, d, dtype)
    a = check_blocks(c, q, lists, 12, 9, dtype)
    # the heads' rows of pages that they do not see
    for g, mine in enumerate(lists[0]):
        for i in range(2, 36):
            if i not in mine:
                c["k"][c["table"][0][i], :, g] = np.nan
                c["v"][c["table"][0][i], :, g] = np.inf if i % 2 else np.nan
    b = blocks(c, q, lists, 12, 9, dtype)
    assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])


# ------------------------------------------------------------------ together, as a program uses them
@pytest.mark.parametrize("dtype,H,G,d", [("bf16", 8, 2, 128), ("f32", 4, 2, 64)])
def test_a_run_of_them(dtype, H, G, d):
    """Prompts enter the cache, their bounds are taken, sequences branch and go on, bounds follow; pages are selected and
    attended, the branches attend to their common rows; the pool moves and everything still agrees."""
    rng = np.random.default_rng(20)
    B, page, M = 6, 8, 2
    c = make(rng, [0] * B, page, 40, 170, G, d, dtype)
    t, handle = on_gpu(c, dtype)
    bnd = torch.full((170, G, 2, d), 7.0, dtype=tdt(dtype), device=DEV)
    bnd_host = np.full((170, G, 2, d), 7.0)

    def append(c, n, slots, pos):
        x = [stored(1.28 * rng.standard_normal((len(slots), n, G, d)), dtype) for _ in range(2)]
        desc = desc_for(len(slots), n, H, G, d, dtype)
        bx.beagle_xattn_paged_append(desc, handle, ints(slots), ints(pos), None, dev(x[0], dtype), dev(x[1], dtype), None,
                                     workspace(desc, handle, bx.BEAGLE_WS_PAGED_APPEND))
        bx.beagle_xattn_paged_bounds(desc_for(len(slots), 1, H, G, d, dtype), handle, ints(slots), ints(pos), bnd)
        c = po.append(c, *x, slots=slots, pos=pos)[0]
        return c, pc.bounds(c, bnd_host, slots=slots, first=pos)

    c, bnd_host = append(c, 201, [0, 3], [0, 0])
    desc = desc_for(4, 1, H, G, d, dtype)
    bx.beagle_xattn_paged_fork(desc, handle, ints([1, 2, 4, 5]), ints([0, 0, 3, 3]), ints([201, 190, 201, 77]),
                               workspace(desc, handle, bx.BEAGLE_WS_PAGED_FORK))
    c = po.fork(c, [1, 2, 4, 5], [0, 0, 3, 3], [201, 190, 201, 77])
    for step in range(3):
        c, bnd_host = append(c, 7, list(range(B)), [n - step for n in c["lens"]])
    torch.cuda.synchronize()
    assert np.array_equal(host(bnd), bnd_host)

    def look(c, handle, bnd, bnd_host):
        q = queries(rng, B, M, H, d, dtype)
        desc, qd = desc_for(B, M, H, G, d, dtype), dev(q, dtype)
        pages = torch.zeros(B, G, 5, dtype=torch.int32, device=DEV)
        bx.beagle_xattn_paged_select(desc, handle, qd, None, None, bnd, 20, 3, 5, pages, workspace(desc, handle, bx.BEAGLE_WS_PAGED_SELECT))
        got = outputs(B, M, H, d, dtype)
        bx.beagle_xattn_paged_attend_blocks(desc, handle, qd, None, None, None, 0, 20, 3, pages, 5, *got, workspace(desc, handle, bx.BEAGLE_WS_PAGED_BLOCKS))
        want_pages = pc.select(c, q, bnd_host, 20, 3, 5)
        assert np.array_equal(pages.cpu().numpy(), want_pages)
        check(got, pc.attend_blocks(c, q, want_pages, 20, 3), dtype, max(c["lens"]))
        for n in ([190, 77], [201, 201]):
            got = outputs(B, M, H, d, dtype)
            bx.beagle_xattn_paged_attend_shared(desc, handle, qd, None, ints([0, 3, 6]), ints(n), 2, None, None, 0, *got,
                                                workspace(desc, handle, bx.BEAGLE_WS_PAGED_SHARED))
            check(got, pc.attend_shared(c, q, [0, 3, 6], n), dtype, max(c["lens"]))
            if n == [190, 77]:               # the common rows are what each has: plain attention
                check(got, po.attend(c, q), dtype, max(c["lens"]))

    look(c, handle, bnd, bnd_host)
    into = dict(c, k=np.full((120, page, G, d), np.nan), v=np.full((120, page, G, d), np.nan), table=[[-1] * 40 for _ in range(B)],
                lens=[0] * B, refs=[0] * 120)
    t2, handle2 = on_gpu(into, dtype)
    bx.beagle_xattn_paged_compact(desc_for(B, 1, H, G, d, dtype), handle, handle2, None, workspace(desc_for(B, 1, H, G, d, dtype), handle, bx.BEAGLE_WS_PAGED_COMPACT))
    c2, short = po.compact(c, into)
    assert short == 0
    bnd2 = torch.zeros(120, G, 2, d, dtype=tdt(dtype), device=DEV)
    bx.beagle_xattn_paged_bounds(desc_for(B, 1, H, G, d, dtype), handle2, None, None, bnd2)
    bnd2_host = pc.bounds(c2, np.zeros((120, G, 2, d)), slots=range(B))
    torch.cuda.synchronize()
    assert np.array_equal(host(bnd2), bnd2_host)
    look(c2, handle2, bnd2, bnd2_host)


def _calls(rng, dtype="bf16", H=8, G=2, d=128):
    """The four calls on one cache as functions of (queries, outputs, workspaces), and what they need."""
    c, first, n = branches(rng, [300], [4], [40, 70, 9, 130], 16, G, d, dtype)
    t, handle = on_gpu(c, dtype)
    desc = desc_for(4, 2, H, G, d, dtype)
    bnd = dev(bounds_of(c), dtype)
    fixed = dict(t=t, handle=handle, desc=desc, bnd=bnd, first=ints(first), n=ints(n))

    def state():
        return dict(q=torch.zeros(4, 2, H, d, dtype=tdt(dtype), device=DEV), bnd=torch.zeros_like(bnd), pages=torch.zeros(4, G, 6, dtype=torch.int32, device=DEV),
                    one=outputs(4, 2, H, d, dtype), two=outputs(4, 2, H, d, dtype),
                    ws=[workspace(desc, handle, w) for w in (bx.BEAGLE_WS_PAGED_SHARED, bx.BEAGLE_WS_PAGED_SELECT, bx.BEAGLE_WS_PAGED_BLOCKS)])

    def run(s, stream=None):
        bx.beagle_xattn_paged_attend_shared(desc, handle, s["q"], None, fixed["first"], fixed["n"], 1, None, None, 0, *s["one"], s["ws"][0], stream)
        bx.beagle_xattn_paged_bounds(desc, handle, None, None, s["bnd"], stream)
        bx.beagle_xattn_paged_select(desc, handle, s["q"], None, None, bnd, 20, 3, 6, s["pages"], s["ws"][1], stream)
        bx.beagle_xattn_paged_attend_blocks(desc, handle, s["q"], None, None, None, 0, 20, 3, s["pages"], 6, *s["two"], s["ws"][2], stream)

    def results(s):
        return [x.clone() for x in (*s["one"], s["bnd"], s["pages"], *s["two"])]

    def fill(s, seed):
        s["q"].copy_(dev(queries(np.random.default_rng(seed), 4, 2, H, d, dtype), dtype))
    return fixed, state, run, results, fill


def test_a_captured_run_replays():
    fixed, state, run, results, fill = _calls(np.random.default_rng(30))
    s, eager = state(), state()
    run(s)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        run(s)
    for seed in range(5):
        fill(s, seed), fill(eager, seed)
        s["bnd"].fill_(3.0), eager["bnd"].fill_(3.0)
        for x in (*s["one"], *s["two"]):
            x.fill_(float("nan"))
        graph.replay()
        run(eager)
        torch.cuda.synchronize()
        for a, b in zip(results(s), results(eager)):
            assert torch.equal(a, b)


def test_two_graphs_with_one_workspace_take_turns():
    fixed, state, run, results, fill = _calls(np.random.default_rng(32))
    both, eager = [state(), state()], state()
    both[1]["ws"] = both[0]["ws"]
    graphs = []
    run(both[0])
    torch.cuda.synchronize()
    for s in both:
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[-1]):
            run(s)
    for seed in range(4):
        for i, (s, graph) in enumerate(zip(both, graphs)):
            fill(s, 2 * seed + i)
            graph.replay()
        for i, s in enumerate(both):
            fill(eager, 2 * seed + i)
            run(eager)
            torch.cuda.synchronize()
            for a, b in zip(results(s), results(eager)):
                assert torch.equal(a, b)


def test_two_streams_and_the_same_bits_every_time():
    fixed, state, run, results, fill = _calls(np.random.default_rng(31))
    want = []
    for seed in range(2):
        s = state()
        fill(s, seed)
        run(s)
        torch.cuda.synchronize()
        want.append(results(s))
    both = [state() for _ in range(2)]
    for seed, s in enumerate(both):
        fill(s, seed)
    streams = [torch.cuda.Stream() for _ in range(2)]
    torch.cuda.synchronize()
    for _ in range(10):
        for s, stream in zip(both, streams):
            run(s, stream)
    torch.cuda.synchronize()
    for s, w in zip(both, want):
        for a, b in zip(results(s), w):
            assert torch.equal(a, b)


def test_rows_and_pages_behind_four_gigabytes():
    """The highest pages of a pool whose K alone has more than 2^32 bytes, and the bounds of as many."""
    rng = np.random.default_rng(40)
    G, d, page, P = 8, 128, 64, 34000
    c = make(rng, [200, 150, 130], page, 4, 12, G, d, "bf16")
    high = {p: P - 1 - 3 * p for p in range(12)}
    k, v = (torch.empty(P, page, G, d, dtype=torch.bfloat16, device=DEV) for _ in range(2))
    bnd = torch.empty(P, G, 2, d, dtype=torch.bfloat16, device=DEV)
    for p, at in high.items():
        k[at], v[at] = dev(c["k"][p], "bf16"), dev(c["v"][p], "bf16")
    table = [[high[p] if p >= 0 else -1 for p in row] for row in c["table"]]
    assert k.numel() * 2 > 1 << 32
    table, lens, refs = ints(table), ints(c["lens"]), torch.zeros(P, dtype=torch.int32, device=DEV)
    handle = bx.make_paged_cache(k, v, table, lens, refs)
    q = queries(rng, 3, 1, 16, d, "bf16")
    desc, qd = desc_for(3, 1, 16, G, d, "bf16"), dev(q, "bf16")
    got = outputs(3, 1, 16, d, "bf16")
    bx.beagle_xattn_paged_attend_shared(desc, handle, qd, None, ints([0, 3]), ints([100]), 1, None, None, 0, *got,
                                        workspace(desc, handle, bx.BEAGLE_WS_PAGED_SHARED))
    torch.cuda.synchronize()
    check(got, pc.attend_shared(c, q, [0, 3], [100]), "bf16", 200)
    bx.beagle_xattn_paged_bounds(desc, handle, None, None, bnd)
    torch.cuda.synchronize()
    want = pc.bounds(c, np.zeros((12, G, 2, d)), slots=range(3))
    for s, n in enumerate(c["lens"]):
        for i in range(n // page):
            p = c["table"][s][i]
            assert np.array_equal(host(bnd[high[p]]), want[p])
    pages = torch.zeros(3, G, 1, dtype=torch.int32, device=DEV)
    bx.beagle_xattn_paged_select(desc, handle, qd, None, None, bnd, 0, 0, 1, pages, workspace(desc, handle, bx.BEAGLE_WS_PAGED_SELECT))
    got = outputs(3, 1, 16, d, "bf16")
    bx.beagle_xattn_paged_attend_blocks(desc, handle, qd, None, None, None, 0, 0, 0, pages, 1, *got, workspace(desc, handle, bx.BEAGLE_WS_PAGED_BLOCKS))
    torch.cuda.synchronize()
    picked = pc.select(c, q, want, 0, 0, 1)
    assert np.array_equal(pages.cpu().numpy(), picked)
    check(got, pc.attend_blocks(c, q, picked, 0, 0), "bf16", 200)
