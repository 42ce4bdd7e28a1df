"""What the paged attention asks for as workspace, and that it does with it where a kv head has one worker (CPU, and one GPU test)."""
import numpy as np
import pytest

from paper_2505_24544_amd import binding as bx
from test_paged_abi import _cache, _desc


def _bytes(**kw):
    return bx.beagle_xattn_paged_workspace_bytes(_desc(**kw), _cache(N=64), bx.BEAGLE_WS_PAGED_ATTEND)


@pytest.mark.parametrize("B,M,H,G,dtype,d", [(1, 4096, 32, 32, bx.BEAGLE_BF16, 128), (7, 4096, 32, 8, bx.BEAGLE_BF16, 128), (3, 160, 64, 64, bx.BEAGLE_F32, 4)])
def test_many_query_rows_need_no_sums_of_parts(B, M, H, G, dtype, d):
    """One worker a kv head and row block takes every entry whole: what is left is a note of 8 bytes for each entry."""
    assert 8 * B <= _bytes(B=B, M=M, H=H, G=G, dtype=dtype, d=d) <= 256


@pytest.mark.parametrize("B,M,H,G", [(1, 1, 32, 32), (48, 1, 32, 8), (12, 10, 32, 8), (4, 1, 40, 40), (1, 256, 32, 32)])
def test_cut_entries_have_room_for_their_parts(B, M, H, G):
    """Two rows of 130 floats for every worker, kv head and query row of a kv head."""
    rows = M * H // G
    blocks = -(-(-(-rows // 16)) // 2)
    workers = 512 // (G * blocks)
    want = 2 * workers * G * rows * 130 * 4 + 8 * B if workers > 1 else 8 * B
    assert want <= _bytes(B=B, M=M, H=H, G=G) < want + 256


@pytest.mark.gpu
@pytest.mark.parametrize("n_true", [None, [290, 0, 64]])
def test_one_worker_a_head(n_true):
    from test_gpu_paged import check_attend, make, queries
    rng = np.random.default_rng(67)
    c = make(rng, [300, 0, 70], 16, 40, 26, 64, 4, "f32")
    tree = None if n_true is None else rng.random((3, 160, 10)) < 0.5
    check_attend(c, queries(rng, 3, 160, 64, 4, "f32"), "f32", n_true=n_true, tree=tree)
