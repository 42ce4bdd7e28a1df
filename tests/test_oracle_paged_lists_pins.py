"""What pins the oracle of listed pages (CPU): whatever a list holds, no row counts more than once."""
import numpy as np
import pytest

from oracle import paged_context_oracle as pc
from test_oracle_paged_context_pins import alike, make


@pytest.mark.parametrize("odd,clean", [([5, 3, 5], [5]), ([5, -1, 5], [5]), ([2, 7, 99, 7], [2, 7]), ([3, 5, 4, 5, 6], [3, 5, 6]),
                                       ([6, 2, 4, 7], [6, 7]), ([99, 2, 4, 4], [4]), ([2, 2, 3, 2, 3, 4], [2, 3, 4])])
def test_a_page_counts_once(odd, clean):
    rng = np.random.default_rng(1)
    c = make(rng, [40], 4, 10, 1, 4)
    q = rng.standard_normal((1, 1, 1, 4))
    alike(pc.attend_blocks(c, q, [[odd]], 4, 4), pc.attend_blocks(c, q, [[clean]], 4, 4))


def test_weights_of_lists_of_any_content_add_up_row_by_row():
    """With values that are 1 in one page's rows and 0 elsewhere the result is that page's weight: at most one row's share times its rows."""
    rng = np.random.default_rng(2)
    c = make(rng, [80], 4, 20, 1, 4)
    c["k"][:] = 0.0                                          # every row has the same score
    q = rng.standard_normal((1, 1, 1, 4))
    for _ in range(100):
        listed = rng.integers(-2, 22, 12)
        weights = []
        for page in c["table"][0]:
            c["v"][:] = 0.0
            c["v"][page] = 1.0
            weights.append(pc.attend_blocks(c, q, [[listed]], 6, 3)[0][0, 0, 0, 0])
        seen = sum(w > 0 for w in weights)
        assert all(w == 0 or abs(w * seen - 1) < 1e-12 for w in weights), (listed, weights)
