"""What the paged attention computes with: probabilities and scale of 24 bits, infinities in rows that are seen.

Every tolerance counts the roundings of the case at hand, in units u = 2^-24 of a float; bf16 results round by 2^-8 of themselves."""
import numpy as np
import pytest
import torch

from oracle import paged_oracle as po
from test_gpu_paged import attend, host, make, pytestmark, queries, stored  # noqa: F401

U = 2.0 ** -24


@pytest.mark.parametrize("M", [1, 64])                   # an entry for each query (one tile), or all in one entry (two tiles)
@pytest.mark.parametrize("W", [1, 40])                   # a workgroup an entry, or equal runs
def test_probabilities_have_all_their_bits(M, W):
    """Two rows of scores 0 and -t, t another for every query.  Channel m holds a and -b with a / b next to exp(-t) of query m, so the terms
    of o = (a - b exp(-t)) / (1 + exp(-t)) all but cancel and the probability's error is what remains.

    The probability is off by 4 u of itself: two roundings of the scaled score (below 1.45, in log2 units: 2 u) and the hardware's exp2
    (one unit in the last place, 2 u).  Products of bf16 numbers are exact in float; a sum of four terms, cut off at worst, is off by 4 * 2 u
    of the sum of magnitudes.  Half of that sum is the probability's: 8 u + 4 u / 2 = 10 u in all."""
    t = stored(np.linspace(0.26, 0.99, 64), "bf16")
    assert len(set(t)) == 64
    p = np.exp(-t)
    b = np.arange(128, 256)
    off = np.abs(np.rint(p[:, None] * b) - p[:, None] * b)
    b = b[off.argmin(1)]
    a = np.rint(p * b)
    assert (np.abs(a - p * b) <= 2.0 ** -5).all()
    c = dict(k=np.zeros((3, 16, 1, 128)), v=np.zeros((3, 16, 1, 128)), table=[[1] + [-1] * (W - 1)], lens=[2], refs=[0, 1, 0])
    c["k"][1, 1, 0, 0] = -1.0
    c["v"][1, 0, 0, :64], c["v"][1, 1, 0, :64] = a, -b
    q = np.zeros((64 // M, M, 1, 128))
    q[..., 0, 0] = t.reshape(64 // M, M)
    o, lse = attend(c, q, "bf16", slots=[0] * (64 // M), scale=1.0)
    got = host(o).reshape(64, 128)[np.arange(64), np.arange(64)]
    ref, spread = (a - p * b) / (1 + p), (a + p * b) / (1 + p)
    far = np.abs(got - ref) - 2.0 ** -8 * np.abs(ref)
    assert (far <= 10 * U * spread).all(), (far / spread / U).max()
    assert np.abs(host(lse).reshape(64) - np.log1p(p)).max() <= 16 * U


@pytest.mark.parametrize("dtype,d", [("bf16", 128), ("f32", 64)])
@pytest.mark.parametrize("W", [1, 40])
def test_scale_has_all_its_bits(dtype, d, W):
    """A sequence of one row: lse is the score, scale * <q, k> with <q, k> = 1024, whose products are exact.  The scales (0.6932 .. 0.697) are
    those at which scale * log2(e) is a fifth of a float's step (2 u) or less below a float: the score in log2 units rounds by 0.4 u,
    its product with ln 2 by half of a step, 0.73 u, and the float ln 2 is off by 0.05 u: 1.2 u in all.  The float below would be
    1.6 u or more off."""
    scales = np.float32(0.6932) + np.arange(1 << 16) * 2.0 ** -24
    c2 = scales * 1.44269504088896340736
    step = (c2 - 1) * 2.0 ** 23 % 1
    scales = scales[step > 0.8][::800]
    assert len(scales) >= 12 and c2.min() > 1 and (np.float32(scales) == scales).all()
    c = dict(k=np.zeros((3, 16, 1, d)), v=np.zeros((3, 16, 1, d)), table=[[1] + [-1] * (W - 1)], lens=[1], refs=[0, 1, 0])
    c["k"][1, 0, 0, 0] = 32.0
    q = np.zeros((1, 1, 1, d))
    q[..., 0] = 32.0
    for scale in scales:
        lse = attend(c, q, dtype, scale=float(scale))[1]
        assert abs(host(lse).item() / (1024 * scale) - 1) <= 1.2 * U, scale


def with_infinities(rng, lens, page, W, d, dtype):
    """Channel c of the sequences' rows: c % 8 == 0 an infinity in one row, 1 a negative one, 2 the same in every row, 3 both signs, 4 no number,
    5 next to the largest number of bf16; the others ordinary."""
    c = make(rng, lens, page, W, sum(po.pages_of(n, page) for n in lens) + 2, 2, d, dtype)
    for s, n in enumerate(lens):
        place = po.rows_of(c, s, n)
        at = [place[int(i)] for i in rng.integers(0, n, 2)]
        c["v"][at[0]][:, 0::8], c["v"][at[0]][:, 1::8], c["v"][at[0]][:, 4::8] = np.inf, -np.inf, np.nan
        c["v"][at[0]][:, 3::8] = np.inf
        c["v"][at[1]][:, 3::8] = -np.inf
        c["v"][at[1]][:, 5::8] = -3.3e38 if dtype == "f32" else -(2.0 ** 127) * 1.984375
        for p in place:
            c["v"][p][:, 2::8] = np.inf
    return c


@pytest.mark.parametrize("dtype,d", [("bf16", 128), ("f32", 64), ("f32", 100)])
@pytest.mark.parametrize("lens,W,window", [([1, 2, 37, 300], 20, 0), ([1, 2, 37, 300], 400, 0), ([3000, 5, 777], 400, 0), ([900, 40], 400, 64)])
@pytest.mark.parametrize("M", [1, 11])
def test_infinities_in_rows_that_are_seen(dtype, d, lens, W, window, M):
    """Where a query sees an infinite value the result is that infinity, as the definition says: every score is finite, so every weight
    is above zero.  The other channels are as ever: half a step of the result, and per term the weight's error and float sums."""
    rng = np.random.default_rng(len(lens) + M)
    c = with_infinities(rng, lens, 16, W, d, dtype)
    if window:
        inside = {p for s, n in enumerate(lens) for p in po.rows_of(c, s, n)[max(0, n - window):]}
        for s, n in enumerate(lens):
            for p in po.rows_of(c, s, n):
                c["v"][p][:, 7::8] = 1.0 if p in inside else np.inf          # (not seen)
    q = queries(rng, len(lens), M, 8, d, dtype)
    o, lse = attend(c, q, dtype, window=window)
    with np.errstate(invalid="ignore", over="ignore"):
        ref, rlse, spread, err = po.attend(c, q, window=window)
    got = host(o)
    assert np.array_equal(np.isnan(got), np.isnan(ref)), (np.isnan(got).sum(), np.isnan(ref).sum())
    assert np.array_equal(got[np.isinf(ref)], ref[np.isinf(ref)])
    fine = np.isfinite(ref)
    half, e = 2.0 ** -8 if dtype == "bf16" else U, err.transpose(0, 2, 1)[..., None]
    tol = half * np.abs(ref) + spread * (1 + half) * (2 * e + (max(lens) + 64) * 2.0 ** -23) + 1e-37
    assert np.isfinite(got[fine]).all() and (np.abs(got[fine] - ref[fine]) <= tol[fine]).all()
    assert np.isinf(ref).any() and np.isnan(ref).any() and fine.any()


@pytest.mark.parametrize("dtype,d", [("bf16", 128), ("f32", 64)])
@pytest.mark.parametrize("M,W", [(18, 10), (18, 1000), (6, 10), (6, 1000)])
def test_a_value_is_worth_the_same_in_a_true_and_in_a_drafted_row(dtype, d, M, W):
    """The same rows, all seen: as true rows, and as true and drafted ones under a tree that lets everybody see everything."""
    rng = np.random.default_rng(M)
    lens = [90, 33]
    c = with_infinities(rng, lens, 16, W, d, dtype)
    q = queries(rng, 2, M, 4, d, dtype)
    tree = np.ones((2, M, 60), bool)
    a, la = attend(c, q, dtype)
    b, lb = attend(c, q, dtype, n_true=[40, 0], tree=tree)
    a, b = host(a), host(b)
    assert np.array_equal(np.isnan(a), np.isnan(b)) and np.array_equal(a[np.isinf(a)], b[np.isinf(a)])
    assert np.array_equal(np.isfinite(a), np.isfinite(b)) and np.isinf(a).any()
    assert (np.abs(host(la) - host(lb)) <= 64 * U * np.maximum(1, np.abs(host(la)))).all()
