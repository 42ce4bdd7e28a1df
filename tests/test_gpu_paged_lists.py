"""Attention over listed pages on the GPU where lists are not ascending: no page counts more than once, wherever a workgroup begins with the
list and however many page numbers it holds at a time."""
import numpy as np
import pytest

from oracle import paged_oracle as po
from test_gpu_paged import make, queries
from test_gpu_paged_context import check_blocks

pytestmark = pytest.mark.gpu


def wandering(rng, shape, pages):
    """Numbers that mostly go up, sometimes down or back to one that was there."""
    steps = rng.integers(1, max(2 * pages // shape[-1], 3), shape)
    back = rng.random(shape) < 0.1
    steps[back] = -rng.integers(0, max(pages // 3, 2), back.sum())
    return np.cumsum(steps, -1) % (pages + 3) - 1


@pytest.mark.parametrize("dtype,H,G,d", [("bf16", 4, 2, 128), ("f32", 4, 2, 64), ("f32", 2, 2, 100)])
def test_repeated_pages(dtype, H, G, d):
    rng = np.random.default_rng(1)
    c = make(rng, [300, 290], 8, 40, 90, G, d, dtype)
    lists = np.array([[[5, 3, 5, 7, 5, 7, 9, 9], [5, -1, 5, -1, 6, 1 << 30, 6, 7]], [[20, 3, 4, 5, 20, 21, 20, 21], [33, 34, 2, 3, 4, 33, 34, 34]]])
    check_blocks(c, queries(rng, 2, 2, H, d, dtype), lists, 20, 9, dtype)
    for n in (12, 30, 35):
        check_blocks(c, queries(rng, 2, 3, H, d, dtype), wandering(rng, (2, G, n), 37), 20, 9, dtype)


@pytest.mark.parametrize("dtype,H,G,d,B,M", [("bf16", 4, 4, 128, 1, 1), ("bf16", 8, 2, 128, 7, 1), ("bf16", 4, 1, 128, 3, 10), ("f32", 4, 1, 64, 2, 1)])
def test_repeated_pages_of_long_lists(dtype, H, G, d, B, M):
    """Lists that several workgroups share, and of more numbers than one holds."""
    rng = np.random.default_rng(2)
    n = 9000 if B == 1 else 5200
    lens = [n - 700 * i for i in range(B)]
    c = make(rng, lens, 4, n // 4, sum(lens) // 4 + 20, G, d, dtype)
    q = queries(rng, B, M, H, d, dtype)
    for many in (70, 300, 1100):
        check_blocks(c, q, wandering(rng, (B, G, many), n // 4), 500, 5, dtype)
    once = np.arange(600) * 2 + 2
    again = np.concatenate((once, once - 1, once))           # the second third lists one page in two once more, or between
    check_blocks(c, q, np.broadcast_to(again, (B, G, len(again))), 500, 5, dtype)


def test_repeated_pages_of_a_tree():
    rng = np.random.default_rng(3)
    c = make(rng, [400, 301, 150], 16, 30, 90, 2, 128, "bf16")
    tree = rng.random((3, 6, 40)) < 0.4
    n_true = [360, 301, 110]
    assert po.pages_of(400, 16) == 25
    for n in (8, 20):
        check_blocks(c, queries(rng, 3, 6, 8, 128, "bf16"), wandering(rng, (3, 2, n), 22), 33, 4, "bf16", n_true=n_true, tree=tree)
