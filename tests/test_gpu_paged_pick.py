"""Page selection on the GPU where the picking has most to decide: the last page picked with a score below zero (keys that lean against the
queries), pages in doubt around it, over several turns of a workgroup, from scores in LDS and in memory.  Pages have to be equal."""
import numpy as np
import pytest

from test_gpu_paged import make, queries, stored
from test_gpu_paged_context import check_select

pytestmark = pytest.mark.gpu

# entries, heads, pages of four rows; with them one launch or two, scores in LDS or in memory
SIZES = [(9, 8, 620), (2, 1, 1500), (1, 1, 8400)]
KINDS = [("bf16", 128), ("f32", 20)]


def leaning(rng, B, G, pages, d, dtype):
    """A cache, queries and bounds of which every product is below zero: (c, q [B, 1, G, d], bounds)."""
    c = make(rng, [4 * pages + 1 - 4 * b for b in range(B)], 4, pages + 2, B * (pages + 2), G, d, dtype)
    q = stored(np.abs(queries(rng, B, 1, G, d, dtype)) + 0.125, dtype)
    hi = -1.0 - np.abs(rng.standard_normal((len(c["refs"]), G, d)))
    return c, q, stored(np.stack((hi - np.abs(rng.standard_normal(hi.shape)), hi), 2), dtype)


def in_doubt(rng, c, q, b, n_select, many):
    """`many` pages more take the bounds of one that is picked, but for a channel that moves their scores by less than can be told."""
    for e in range(q.shape[0]):
        for g in range(q.shape[2]):
            q[e, 0, g, 0] = 2.0 ** -10
            table = np.array(c["table"][e][: c["lens"][e] // 4])
            order = table[np.argsort(-(b[table, g, 1] @ q[e, 0, g]), kind="stable")]
            like = order[max(n_select - many // 3, 0)]
            alike = rng.permutation(order[n_select + 1:])[:many]
            b[alike, g] = b[like, g]
            b[alike, g, 1, 0] = b[like, g, 1, 0] * (1 + 2.0 ** -7 * rng.integers(-8, 9, len(alike)))


@pytest.mark.parametrize("dtype,d", KINDS)
@pytest.mark.parametrize("B,G,pages", SIZES)
def test_scores_below_zero(B, G, pages, dtype, d):
    rng = np.random.default_rng(pages)
    c, q, b = leaning(rng, B, G, pages, d, dtype)
    for n_select in (1, pages // 3, pages - 9):
        check_select(c, q, b, 0, 0, n_select, dtype)
    for n_select, many in ((40, 12), (pages // 3, 70)):
        q2, b2 = q.copy(), b.copy()
        in_doubt(rng, c, q2, b2, n_select, many)
        check_select(c, stored(q2, dtype), stored(b2, dtype), 0, 0, n_select, dtype)


@pytest.mark.parametrize("dtype,d", KINDS)
@pytest.mark.parametrize("B,G,pages", SIZES[1:])
def test_many_in_doubt(B, G, pages, dtype, d):
    """More pages in doubt than a list holds: equal scores on both sides of the last one picked, and what takes the error's bound away."""
    rng = np.random.default_rng(pages + 1)
    c, q, b = leaning(rng, B, G, pages, d, dtype)
    kinds = b[rng.integers(0, 17, len(b))]                   # seventeen scores below zero, hundreds of pages of each
    for n_select in (1, pages // 17, pages // 2, pages - 3):
        check_select(c, q, kinds, 0, 0, n_select, dtype)
    check_select(c, q, np.zeros_like(b), 8, 4, pages // 3, dtype)
    check_select(c, -q, kinds, 0, 0, pages // 2, dtype)
    odd = b.copy()
    odd[::401, :, 0, 3] = -np.inf                            # (a least value that no query above zero meets)
    for n_select in (5, pages // 3):
        check_select(c, q, odd, 0, 0, n_select, dtype)
    odd[::7, :, 1, 2], odd[1::5, :, 1, 0], odd[2::9, :, 1] = np.nan, np.inf, np.nan
    c["table"][0][11], c["table"][0][pages - 20] = -1, 1 << 20
    for n_select in (pages // 9, pages - 30):
        check_select(c, q, odd, 0, 0, n_select, dtype)
