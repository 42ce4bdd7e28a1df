"""What pins the oracle of shared and long contexts (CPU): it reduces to the plain paged attention where the definitions say so,
scores bound what they claim to bound, and selections agree with a ranking written otherwise."""
import copy

import numpy as np
import pytest

from oracle import paged_context_oracle as pc
from oracle import paged_oracle as po


def make(rng, lens, page, W, G, d):
    need = sum(po.pages_of(n, page) for n in lens)
    k, v = rng.standard_normal((2, need + 2, page, G, d))
    c = dict(k=k, v=v, table=[[-1] * W for _ in lens], lens=list(lens), refs=[0] * (need + 2))
    order = [int(p) for p in rng.permutation(need + 2)]
    for s, n in enumerate(lens):
        for i in range(po.pages_of(n, page)):
            c["table"][s][i] = order.pop()
            c["refs"][c["table"][s][i]] = 1
    return c


def branches(rng, c, src, rows, slots, new):
    """Slots that go on from `rows` rows of slot src, each with rows of its own."""
    c = po.fork(c, slots, [src] * len(slots), [rows] * len(slots))
    G, d = c["k"].shape[2:]
    for s, n in zip(slots, new):
        x = rng.standard_normal((2, 1, n, G, d))
        c, short = po.append(c, x[0], x[1], slots=[s])
        assert short == 0
    return c


def alike(a, b, at=1e-12):
    for x, y in zip(a[:2], b[:2]):
        assert np.array_equal(np.isneginf(x), np.isneginf(y))
        assert np.allclose(np.where(np.isneginf(x), 0, x), np.where(np.isneginf(y), 0, y), rtol=at, atol=at)


def test_common_rows_are_plain_attention_on_branches():
    rng = np.random.default_rng(0)
    c = make(rng, [37, 0, 0, 0, 21, 0], 4, 20, 2, 8)
    for x in ("k", "v"):
        c[x] = np.concatenate((c[x], rng.standard_normal((30, *c[x].shape[1:]))))
    c["refs"] += [0] * 30
    c = branches(rng, c, 0, 30, [1, 2, 3], [5, 1, 9])
    c = branches(rng, c, 4, 21, [5], [3])
    q = rng.standard_normal((6, 2, 4, 8))
    slots = [0, 2, 1, 3, 5, 4]
    want = po.attend(c, q, slots=slots)
    for n in ([30, 21], [12, 0], [29, 7], [1, 21]):
        alike(pc.attend_shared(c, q, [0, 4, 6], n, slots=slots), want)
    tree = rng.random((6, 2, 6)) < 0.5
    n_true = [c["lens"][s] - 3 for s in slots]
    alike(pc.attend_shared(c, q, [0, 4, 6], [30, 18], slots=slots, n_true=n_true, tree=tree), po.attend(c, q, slots=slots, n_true=n_true, tree=tree))


def test_common_rows_are_those_of_the_first_entry():
    rng = np.random.default_rng(1)
    c = make(rng, [10, 14, 0], 4, 8, 1, 4)
    q = rng.standard_normal((3, 1, 1, 4))
    o = pc.attend_shared(c, q, [0, 3], [6])[0]
    # the second entry: rows 0 .. 5 of slot 0, 6 .. 13 of its own; the third is empty
    rows = po.rows_of(c, 0, 6) + po.rows_of(c, 1, 14)[6:]
    s = np.array([c["k"][p, r, 0] @ q[1, 0, 0] for p, r in rows]) / 2.0
    w = np.exp(s) / np.exp(s).sum()
    assert np.allclose(o[1, 0, 0], sum(x * c["v"][p, r, 0] for x, (p, r) in zip(w, rows)))
    assert (o[2] == 0).all()
    # what the first entry does not hold is not seen
    o = pc.attend_shared(c, q, [0, 3], [12])[0]
    rows = po.rows_of(c, 0, 10) + po.rows_of(c, 1, 14)[12:]
    s = np.array([c["k"][p, r, 0] @ q[1, 0, 0] for p, r in rows]) / 2.0
    w = np.exp(s) / np.exp(s).sum()
    assert np.allclose(o[1, 0, 0], sum(x * c["v"][p, r, 0] for x, (p, r) in zip(w, rows)))


def test_groups():
    assert pc.groups_of([0, 2, 5], 5) == [(0, 2), (2, 5)]
    assert pc.groups_of([1, 4, 2, 9], 5) == [(1, 4), (4, 4), (4, 5)]
    assert pc.groups_of([-3, 3, 3], 5) == [(0, 3), (3, 3)]


def test_bounds_are_bounds_and_leave_other_pages_alone():
    rng = np.random.default_rng(2)
    c = make(rng, [10, 7], 4, 4, 2, 4)
    before = rng.standard_normal((len(c["refs"]), 2, 2, 4))
    out = pc.bounds(c, before, slots=[0, 1])
    whole = [c["table"][0][0], c["table"][0][1], c["table"][1][0]]
    for p in range(len(c["refs"])):
        if p in whole:
            assert np.array_equal(out[p, :, 0], c["k"][p].min(0)) and np.array_equal(out[p, :, 1], c["k"][p].max(0))
        else:
            assert np.array_equal(out[p], before[p])
    out = pc.bounds(c, before, slots=[0], first=[4])
    assert np.array_equal(out[whole[0]], before[whole[0]]) and not np.array_equal(out[whole[1]], before[whole[1]])
    assert not np.array_equal(pc.bounds(c, before, slots=[0], first=[3])[whole[0]], before[whole[0]])


def test_no_key_of_a_page_exceeds_its_score():
    rng = np.random.default_rng(3)
    for _ in range(50):
        k, q = rng.standard_normal((8, 16)), rng.standard_normal((3, 16))
        assert pc.score(q, k.min(0), k.max(0)) >= (k @ q.T).max() - 1e-6
        one = k[:1]
        assert abs(pc.score(q, one[0], one[0]) - (one @ q.T).max()) < 1e-6        # one key: its own product


def test_selection_against_a_ranking_written_otherwise():
    rng = np.random.default_rng(4)
    c = make(rng, [50, 33, 3], 4, 13, 2, 8)
    q = rng.standard_normal((3, 2, 4, 8))
    b = pc.bounds(c, np.zeros((len(c["refs"]), 2, 2, 8)), slots=range(3))
    for window, sinks, n in ((0, 0, 3), (9, 5, 4), (7, 0, 100), (100, 0, 2), (0, 100, 2)):
        out = pc.select(c, q, b, window, sinks, n)
        for e in range(3):
            lo, hi = pc.span(c["lens"][e], window, sinks, 4)
            for g in range(2):
                at = c["table"][e][lo:hi]
                both = np.stack([b[at, g, 0], b[at, g, 1]])                        # [2, pages, d]
                s = (q[e, :, 2 * g: 2 * g + 2].reshape(-1, 1, 1, 8) * both).max(1).sum(-1).max(0) if at else np.zeros(0)
                want = sorted(np.argsort(-s.astype(np.float32), kind="stable")[:n] + lo)
                assert out[e, g].tolist() == want + [-1] * (n - len(want))


def test_equal_scores_take_the_first_pages():
    rng = np.random.default_rng(5)
    c = make(rng, [40], 4, 10, 1, 4)
    c["k"][:] = 1.0
    b = pc.bounds(c, np.zeros((len(c["refs"]), 1, 2, 4)), slots=[0])
    assert pc.select(c, rng.standard_normal((1, 1, 1, 4)), b, 4, 3, 3)[0, 0].tolist() == [1, 2, 3]


@pytest.mark.parametrize("window,sinks", [(0, 0), (8, 4), (9, 5), (3, 0), (100, 3), (0, 50)])
def test_pages_between_plain_attention_and_a_window(window, sinks):
    rng = np.random.default_rng(6)
    c = make(rng, [50, 33, 3, 0], 4, 13, 2, 8)
    q = rng.standard_normal((4, 2, 4, 8))
    n_true = [45, 33, 1, 0]
    tree = rng.random((4, 2, 5)) < 0.5
    lists = [[list(range(*pc.span(n_true[e], window, sinks, 4))) + [-1] * 2] * 2 for e in range(4)]
    alike(pc.attend_blocks(c, q, lists, window, sinks, n_true=n_true, tree=tree), po.attend(c, q, n_true=n_true, tree=tree))
    # nothing listed: a window from a page's first row on, whole pages of first rows
    empty = [[[-1] * 4] * 2] * 4
    got = pc.attend_blocks(c, q, empty, window, sinks, n_true=n_true, tree=tree)
    for e in range(4):
        lo, hi = pc.span(n_true[e], window, sinks, 4)
        one = dict(c, table=[c["table"][e]], lens=[c["lens"][e]])
        w = n_true[e] - 4 * hi
        if w <= 0:                           # the true rows end with a page: none of them is in the window
            continue
        want = po.attend(one, q[e:e + 1], n_true=[n_true[e]], tree=tree[e:e + 1], window=w, sinks=4 * lo)
        alike([x[e:e + 1] for x in got], want)


def test_numbers_that_list_nothing():
    rng = np.random.default_rng(7)
    c = make(rng, [40], 4, 10, 1, 4)
    q = rng.standard_normal((1, 1, 1, 4))
    clean = pc.attend_blocks(c, q, [[[3, 5, -1, -1, -1, -1]]], 4, 4)
    for odd in ([3, 3, 5, 0, -7, -1], [3, 2, 1, 5, 99, 9], [0, 3, 5, 5, 1 << 20, 4]):
        alike(pc.attend_blocks(c, q, [[odd]], 4, 4), clean)


def test_the_cache_is_not_changed():
    rng = np.random.default_rng(8)
    c = make(rng, [20, 9], 4, 6, 1, 4)
    was = copy.deepcopy(c)
    q = rng.standard_normal((2, 1, 1, 4))
    pc.attend_shared(c, q, [0, 2], [5])
    b = pc.bounds(c, np.zeros((len(c["refs"]), 1, 2, 4)), slots=[0, 1])
    pc.attend_blocks(c, q, pc.select(c, q, b, 4, 1, 2), 4, 1)
    assert c["lens"] == was["lens"] and c["table"] == was["table"] and np.array_equal(c["k"], was["k"])
