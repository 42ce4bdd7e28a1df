"""The paged draft step's rotated queries: how often they round."""
import numpy as np
import pytest
import torch

from oracle import paged_oracle as po
from paper_2505_24544_amd import binding as bx
from test_gpu_paged import DEV, desc_for, dev, host, ints, on_gpu, pytestmark, stored, workspace  # noqa: F401


def rotated_queries(B, M, D, H, given, seed):
    """One row in every sequence, a 1 in channel 13 b of it: with a scale of 1 the lse of entry b is channel 13 b of its rotated queries.
    Returns those, by the library and in float64, and the pair's other channel."""
    rng = np.random.default_rng(seed)
    c = dict(k=np.zeros((B, 4, 1, 128)), v=np.zeros((B, 4, 1, 128)), table=[[b] for b in range(B)], lens=[1] * B, refs=[1] * B)
    ch = [13 * b % 128 for b in range(B)]
    for b in range(B):
        c["k"][b, 0, 0, ch[b]] = 1.0
    t, handle = on_gpu(c, "bf16")
    x, wq = stored(rng.standard_normal((B, M, D)), "bf16"), stored(0.05 * rng.standard_normal((D, H * 128)), "bf16")
    wo = torch.zeros(H * 128, D, dtype=torch.bfloat16, device=DEV)
    pos = rng.integers(0, 100000, (B, M))
    at = ints([int(p) for p in pos.reshape(-1)]) if given else None
    if not given:
        pos = np.ones((B, M), int)                        # the rows that a slot holds
    desc = desc_for(B, M, H, 1, 128, "bf16", hidden=D, flags=bx.BEAGLE_FLAG_ROPE, rope_positions=at, softmax_scale=1.0)
    y = torch.empty(B, M, D, dtype=torch.bfloat16, device=DEV)
    lse = torch.full((B, H, M), float("nan"), dtype=torch.float32, device=DEV)
    print("rotated queries", B, M, D, H, given, flush=True)
    bx.beagle_xattn_draft_step_paged(desc, handle, dev(x, "bf16"), dev(wq, "bf16"), wo, None, None, None, 0, 0, 0, y, lse,
                                     workspace(desc, handle, bx.BEAGLE_WS_PAGED_DRAFT))
    torch.cuda.synchronize()
    assert not host(y).any()
    q, size = (x.reshape(-1, D) @ wq).reshape(B, M, H, 128), (np.abs(x).reshape(-1, D) @ np.abs(wq)).reshape(B, M, H, 128)
    want, sums = np.zeros((B, H, M)), np.zeros((B, H, M))
    for b in range(B):
        for m in range(M):
            want[b, :, m] = po.rotate(q[b, m], pos[b, m], 10000.0)[:, ch[b]]
            sums[b, :, m] = size[b, m][:, [ch[b], (ch[b] + 64) % 128]].sum(-1)
    return host(lse), want, sums


@pytest.mark.parametrize("B,M", [(1, 1), (9, 3), (16, 4), (13, 5), (12, 10), (16, 8)])
@pytest.mark.parametrize("given", [False, True])
def test_rotated_queries_round_once(B, M, given):
    """Half a step of the stored value (steps are 2^-7 of the power of two below it), the product's float sums (1024 terms in blocks of 32
    and their slices: at most 64 roundings of the magnitudes), and 9 * 2^-24 of the value: the rotation's two products and sum, and
    score and lse."""
    got, want, sums = rotated_queries(B, M, 1024, 4, given, B + M)
    step = 2.0 ** (np.floor(np.log2(np.abs(want))) - 7)
    off = 64 * 2.0 ** -24 * sums
    assert (np.abs(got - want) <= step / 2 + off + 9 * 2.0 ** -24 * np.abs(want)).all(), (np.abs(got - want) / step).max()


def test_rotated_queries_of_many_rows_round_twice():
    """Past 128 rows the product is stored and rotated in place: half a step of either channel of the pair, and of the result
    (values here stay below 6)."""
    got, want, sums = rotated_queries(43, 3, 256, 2, True, 5)
    assert np.abs(got - want).max() <= 2.0 ** -8 * (1 + 2 ** 0.5) * 6
    assert np.isfinite(got).all() and np.abs(want).max() < 6
