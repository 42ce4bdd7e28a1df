"""Calls of the paged cache past what one workgroup holds at once: more counts than the planning workgroup looks at in a trip (16384), more
pages than it keeps in LDS (4096), more entries than it has threads (1024), compactions of two launches (more than 4096 pages), and
attention of more entries than a wave has lanes.  Everything that is moved has to be equal to the oracle's."""
import numpy as np
import pytest
import torch

from oracle import paged_oracle as po
from test_gpu_paged import attend, check_attend, host, make, new_rows, pytestmark, queries, run_append, run_compact, stored  # noqa: F401


def hold(rng, c, free):
    """Every page that no slot names is held by somebody else, but for those of `free`."""
    named = {p for row, n in zip(c["table"], c["lens"]) for p in row[: po.pages_of(n, c["k"].shape[1])]}
    free = set(free) - named
    for p in range(len(c["refs"])):
        if p not in named:
            c["refs"][p] = int(p not in free)
    return len(free)


@pytest.mark.parametrize("spare", [40, 0, -30])          # free pages left over, none, too few
def test_free_pages_are_spread_over_the_counts(spare):
    rng = np.random.default_rng(101)
    N, P = 40, 50000                                      # three trips of 16384 counts, and a ragged one
    c = make(rng, [int(n) for n in rng.integers(0, 30, N)], 4, 60, P, 1, 4, "f32", stale=3.0)
    kn, vn = new_rows(rng, N, 200, 1, 4, "f32")
    n_new = [int(n) for n in rng.integers(0, 201, N)]
    need = sum(po.pages_of(n + m, 4) - po.pages_of(n, 4) for n, m in zip(c["lens"], n_new))
    named = {p for row in c["table"] for p in row if p >= 0}
    others = np.array([p for p in rng.permutation(P) if p not in named])
    free = [int(p) for p in others[: need + spare]]
    assert hold(rng, c, free) == need + spare and need > 400
    assert all(sum(lo <= p < lo + 16384 for p in free) < need / 2 for lo in range(0, P, 16384)) and max(free) >= 3 * 16384
    run_append(c, "f32", kn, vn, slots=[int(s) for s in rng.permutation(N)], n_new=n_new)


@pytest.mark.parametrize("spare", [500, -200])
def test_more_pages_than_lds_holds(spare):
    rng = np.random.default_rng(103)
    N = 64
    lens = [int(n) for n in rng.integers(0, 20, N)]
    need = sum(po.pages_of(n + 300, 4) - po.pages_of(n, 4) for n in lens)
    assert need + min(spare, 0) > 4096 + 200
    c = make(rng, lens, 4, 80, need + spare + sum(po.pages_of(n, 4) for n in lens), 1, 4, "f32", stale=3.0)
    run_append(c, "f32", *new_rows(rng, N, 300, 1, 4, "f32"))
    # rows given up make room for the ones that come; shared pages are copied; and what is taken lies in several trips' counts
    c = po.fork(c, [1, 2, 3], [0, 0, 0], [3, 2, 1])
    run_append(c, "f32", *new_rows(rng, N, 300, 1, 4, "f32"), pos=[int(p) for p in rng.integers(0, 9, N)], n_new=[int(n) for n in rng.integers(0, 301, N)])


def many_slots(rng, P):
    """1400 slots, some of them forks of others that share a page in part."""
    N = 1400
    c = make(rng, [int(n) for n in rng.integers(0, 14, N)], 4, 5, P, 1, 4, "f32", stale=3.0)
    to = [int(s) for s in rng.permutation(N)[:400]]
    return po.fork(c, to, [int(s) for s in rng.integers(0, N, 400)], [int(n) for n in rng.integers(0, 14, 400)])


@pytest.mark.parametrize("free", [4000, 300])
@pytest.mark.parametrize("B", [1025, 2500])
def test_more_entries_than_threads(free, B):
    """Duplicates, slots that are none, rows given up, shared pages kept in part, more rows than a slot holds, and (300 free ones) too few pages."""
    rng = np.random.default_rng(B + free)
    c = many_slots(rng, 6000)
    spare = [p for p in rng.permutation(6000) if c["refs"][p] <= 0]
    for p in spare[free:]:
        c["refs"][p] = 1                                  # (held by somebody else)
    slots = [int(s) for s in rng.integers(-2, 1403, B)]
    slots[7], slots[1024] = 2 ** 31 - 1, -2 ** 31
    pos = [int(p) for p in rng.integers(-1, 16, B)]
    n_new = [int(n) for n in rng.integers(-1, 9, B)]
    kn, vn = new_rows(rng, B, 7, 1, 4, "f32")
    ref, _ = run_append(c, "f32", kn, vn, slots=slots, pos=pos, n_new=n_new, rope=100.0)
    assert len(set(slots)) < B - 50 and sum(0 <= s < 1400 for s in slots) < B
    ref["k"] = stored(ref["k"], "f32")                    # (the oracle's rotated rows are not rounded)
    run_append(ref, "f32", *new_rows(rng, B, 2, 1, 4, "f32"), slots=slots)        # and again, behind what is there


BIG = [3 * 700 + 1, 0, 1700, 5 * 900 - 1, 1]


@pytest.mark.parametrize("dtype,G,d", [("f32", 1, 4), ("bf16", 1, 128)])
def test_compaction_of_two_launches(dtype, G, d):
    rng = np.random.default_rng(107)
    W = po.pages_of(max(BIG), 4) + 3
    c = make(rng, BIG, 4, W, 5000, G, d, dtype, stale=4.0)
    c = po.fork(c, [1], [3], [1501])                       # shared, the last page in part
    live = sum(r > 0 for r in c["refs"])

    def blank(P, width):
        return dict(make(rng, [0] * 5, 4, width, P, G, d, dtype, stale=9.0), lens=[5] * 5, refs=[3] * P)

    run_compact(c, blank(6000, W), dtype)                  # larger
    run_compact(c, blank(live, W), dtype)                  # exactly the live pages
    run_compact(c, blank(live - 1, W), dtype)              # one page short
    run_compact(c, blank(700, W), dtype)                   # far too small: every long sequence is cut
    run_compact(c, blank(6000, 300), dtype)                # a narrower table
    run_compact(c, blank(live, W + 700), dtype)            # a wider one
    run_compact(c, blank(900, 300), dtype)                 # both too small
    c["table"][3][400], c["table"][0][7], c["table"][2][0] = -1, 5000, 2 ** 31 - 1        # lost pages cut, the first one to nothing
    run_compact(c, blank(6000, W), dtype)
    run_compact(c, blank(1000, 500), dtype)
    free = [p for p in range(5000) if c["refs"][p] <= 0]
    c["table"][0][3] = free[0]                             # a page that nobody counts did not move
    run_compact(c, blank(6000, W), dtype)


def test_compaction_of_more_pages_than_a_trip_numbers():
    rng = np.random.default_rng(109)
    c = make(rng, [int(n) for n in rng.integers(0, 1200, 60)], 4, 300, 40000, 1, 4, "f32", stale=0.0)
    c = po.fork(c, [3, 9], [4, 4], [700, 33])
    run_compact(c, dict(make(rng, [0] * 60, 4, 310, 20000, 1, 4, "f32", stale=0.0)), "f32")
    run_compact(c, dict(make(rng, [0] * 60, 4, 300, 2500, 1, 4, "f32", stale=0.0)), "f32")
    empty = make(rng, [0] * 60, 4, 300, 5000, 1, 4, "f32", stale=0.0)
    run_compact(empty, dict(make(rng, [0] * 60, 4, 10, 8, 1, 4, "f32", stale=1.0), lens=[3] * 60, refs=[1] * 8), "f32")


@pytest.mark.parametrize("M,window", [(1, 0), (9, 0), (2, 100)])
def test_more_entries_than_lanes(M, window):
    """Long entries among many short and empty ones, cut or whole, in the first, a middle and the last group of 64."""
    rng = np.random.default_rng(113 + M)
    lens = [int(n) for n in rng.integers(0, 120, 200)]
    lens[5], lens[100], lens[199], lens[64], lens[63] = 2500, 1300, 900, 0, 1
    c = make(rng, lens, 16, 160, sum(po.pages_of(n, 16) for n in lens) + 1, 2, 128, "bf16")
    check_attend(c, queries(rng, 200, M, 8, 128, "bf16"), "bf16", window=window, sinks=3 if window else 0)


def test_many_entries_share_few_slots():
    rng = np.random.default_rng(127)
    c = make(rng, [777, 3, 0, 130], 16, 60, 70, 1, 128, "bf16")
    slots = [int(s) for s in rng.integers(-1, 5, 300)]
    check_attend(c, queries(rng, 300, 1, 4, 128, "bf16"), "bf16", slots=slots, n_true=[int(n) for n in rng.integers(0, 800, 300)],
                 tree=rng.random((300, 1, 70)) < 0.5)


@pytest.mark.parametrize("dtype,d", [("bf16", 128), ("f32", 64)])
def test_a_sequence_alone_and_in_a_batch(dtype, d):
    """Where an entry is cut depends on the others, so the order of its sums does: equal to rounding, not bit by bit (a batch
    repeated is)."""
    rng = np.random.default_rng(131)
    lens = [6000, 10, 2500]
    c = make(rng, lens, 64, 100, 150, 2, d, dtype)
    q = queries(rng, 3, 4, 8, d, dtype)
    o, lse = check_attend(c, q, dtype)
    _, _, spread, _ = po.attend(c, q)
    for b in range(3):
        o1, lse1 = attend(c, q[b:b + 1], dtype, slots=[b])
        again, lse2 = attend(c, q[b:b + 1], dtype, slots=[b])
        assert torch.equal(o1, again) and torch.equal(lse1, lse2)
        # two float evaluations with the same scores and weights: sums of lens + 64 terms each, and both results round
        half = 2.0 ** -8 if dtype == "bf16" else 2.0 ** -24
        tol = 2 * half * np.abs(host(o1)[0]) * (1 + half) + 2 * (lens[b] + 64) * 2.0 ** -23 * spread[b]
        assert (np.abs(host(o)[b] - host(o1)[0]) <= tol).all()
        assert np.abs(host(lse)[b] - host(lse1)[0]).max() <= 2 * (lens[b] + 64) * 2.0 ** -23
