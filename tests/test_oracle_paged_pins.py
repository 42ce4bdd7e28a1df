"""Pins of the paged cache's oracle: hand-written bookkeeping, and attention over pages against the contiguous oracle."""
import numpy as np
import pytest

from oracle import beagle_oracle as orc
from oracle import paged_oracle as po


def _cache(P, page, N, W, G=2, d=8, seed=0):
    rng = np.random.default_rng(seed)
    return dict(k=rng.standard_normal((P, page, G, d)), v=rng.standard_normal((P, page, G, d)), table=[[-1] * W for _ in range(N)],
                lens=[0] * N, refs=[0] * P)


def test_append_fork_and_trim_by_hand():
    c = _cache(6, 4, 3, 4)
    x = np.arange(2 * 6 * 2 * 8, dtype=float).reshape(2, 6, 2, 8)
    c, short = po.append(c, x, -x, slots=[2, 0], n_new=[6, 3])
    assert short == 0 and c["lens"] == [3, 0, 6] and c["table"] == [[2, -1, -1, -1], [-1] * 4, [0, 1, -1, -1]] and c["refs"] == [1, 1, 1, 0, 0, 0]
    assert np.array_equal(c["k"][1, 1], x[0, 5]) and np.array_equal(c["v"][2, 0], -x[1, 0])
    c = po.fork(c, [1], [2], [5])                     # shares page 1 in part
    assert c["refs"] == [2, 2, 1, 0, 0, 0] and c["table"][1] == [0, 1, -1, -1] and c["lens"][1] == 5
    kept = c["k"][1].copy()
    c2, short = po.append(c, x[:1, :1], x[:1, :1], slots=[1])
    assert short == 0 and c2["table"][1] == [0, 3, -1, -1] and c2["refs"] == [2, 1, 1, 1, 0, 0] and np.array_equal(c2["k"][1], kept)
    assert np.array_equal(c2["k"][3, 0], kept[0]) and np.array_equal(c2["k"][3, 1], x[0, 0])
    c3 = po.fork(c2, [2, 0], [-1, 2])                 # frees slot 2; slot 0 takes what slot 2 was
    assert c3["lens"] == [6, 6, 0] and c3["refs"] == [2, 1, 0, 1, 0, 0]
    c4, short = po.append(c2, x, x, slots=[0, 1], pos=[1, 4], n_new=[6, 6])
    assert short == 0 and c4["lens"] == [7, 10, 6] and c4["table"][0] == [2, 3, -1, -1] and c4["table"][1] == [0, 4, 5, -1]
    c5, short = po.append(c2, np.repeat(x, 3, 1), np.repeat(x, 3, 1), slots=[1, 0], n_new=[1, 13])
    assert short == 1 and c5["lens"][0] == 3 and c5["lens"][1] == 7


def test_compact_by_hand():
    c = _cache(6, 4, 2, 3)
    c.update(table=[[4, 1, -1], [4, 5, 3]], lens=[7, 9], refs=[0, 1, 0, 1, 2, 1])
    big, short = po.compact(c, _cache(8, 4, 2, 3, seed=1))
    assert short == 0 and big["table"] == [[2, 0, -1], [2, 3, 1]] and big["refs"] == [1, 1, 2, 1, 0, 0, 0, 0] and big["lens"] == [7, 9]
    assert np.array_equal(big["k"][2], c["k"][4])
    small, short = po.compact(c, _cache(3, 4, 2, 3, seed=1))
    assert short == 1 and small["table"] == [[2, 0, -1], [2, -1, -1]] and small["lens"] == [7, 4] and small["refs"] == [1, 0, 2]


@pytest.mark.parametrize("n,n_true", [(9, 9), (13, 9), (4, 0)])
def test_attention_over_pages_is_attention_over_rows(n, n_true):
    rng = np.random.default_rng(3)
    c = _cache(9, 4, 2, 4)
    c["table"][1], c["lens"] = [7, 2, 5, 0], [0, n]
    q = rng.standard_normal((1, 3, 4, 8))
    tree = rng.random((1, 3, n - n_true)) < 0.5
    o, lse, _, _ = po.attend(c, q, slots=[1], n_true=[n_true], tree=tree)
    rows = np.array([c["k"][p, r] for p, r in po.rows_of(c, 1, n)]), np.array([c["v"][p, r] for p, r in po.rows_of(c, 1, n)])
    eye = np.eye(32)
    ref = orc.draft_step_tree(q[0].reshape(3, 32), rows[0], rows[1], eye, eye, n_true=n_true, tree_mask=tree[0], n_q_heads=4, n_kv_heads=2)
    assert np.allclose(o[0].reshape(3, 32), ref["y"], atol=1e-12) and np.allclose(lse[0], ref["lse"], atol=1e-12)


def test_window_and_sinks_by_hand():
    c = _cache(4, 4, 1, 4)
    c["table"][0], c["lens"] = [3, 1, 0, 2], [14]
    q = np.random.default_rng(4).standard_normal((1, 1, 2, 8))
    o, _, _, _ = po.attend(c, q, window=5, sinks=2)
    short = dict(c, k=np.zeros((4, 4, 2, 8)), v=np.zeros((4, 4, 2, 8)), table=[[0, 1, 2, 3]], lens=[7])
    for i, j in enumerate([0, 1, 9, 10, 11, 12, 13]):
        (p, r), (a, b) = po.rows_of(c, 0, 14)[j], divmod(i, 4)
        short["k"][a, b], short["v"][a, b] = c["k"][p, r], c["v"][p, r]
    assert np.allclose(o, po.attend(short, q)[0], atol=1e-13)


def test_rotation_keeps_lengths_and_composes():
    x = np.random.default_rng(5).standard_normal((2, 8))
    assert np.allclose(po.rotate(po.rotate(x, 3, 100.0), 4, 100.0), po.rotate(x, 7, 100.0)) and np.allclose(po.rotate(x, 0, 100.0), x)
