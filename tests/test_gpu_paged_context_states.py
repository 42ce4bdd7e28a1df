"""The draft steps on shared and on long contexts, from states: they are their projections and the calls that they are made of."""
import numpy as np
import pytest
import torch

from oracle import paged_context_oracle as pc
from paper_2505_24544_amd import binding as bx
from test_gpu_paged import DEV, desc_for, dev, host, ints, on_gpu, pack, pytestmark, queries, stored, tdt, workspace  # noqa: F401
from test_gpu_paged_context import blocks, bounds_of, branches, outputs, select, shared


@pytest.mark.parametrize("dtype,H,G,d,M", [("bf16", 4, 2, 128, 1), ("bf16", 4, 4, 128, 10), ("f32", 4, 2, 64, 2), ("bf16", 4, 1, 128, 40)])
@pytest.mark.parametrize("rope", [False, True])
def test_steps_are_what_they_are_made_of(dtype, H, G, d, M, rope):
    """Weights of ones and zeros project without a rounding, and a rotation by no angle turns nothing: the same bits."""
    rng = np.random.default_rng(M)
    c, first, n = branches(rng, [200, 90], [3, 2], [40, 70, 39, 130, 55], 16, G, d, dtype)
    T, D = 30, H * d
    tree = rng.random((5, M, T)) < 0.5
    n_true = [x - T for x in c["lens"]]
    q = queries(rng, 5, M, H, d, dtype)
    t, handle = on_gpu(c, dtype)
    kw = dict(flags=bx.BEAGLE_FLAG_ROPE, rope_positions=torch.zeros(5 * M, dtype=torch.int32, device=DEV)) if rope else {}
    desc = desc_for(5, M, H, G, d, dtype, hidden=D, **kw)
    eye, x = dev(np.eye(D), dtype), dev(q.reshape(5, M, D), dtype)
    bits, words = pack(tree)

    y, lse = outputs(5, M, H, d, dtype)
    bx.beagle_xattn_draft_step_paged_shared(desc, handle, x, eye, eye, None, ints(first), ints(n), 2, ints(n_true), bits, words, y, lse,
                                            workspace(desc, handle, bx.BEAGLE_WS_PAGED_DRAFT_SHARED))
    torch.cuda.synchronize()
    o, want = shared(c, q, first, n, dtype, n_true=n_true, tree=tree)
    assert torch.equal(y, o) and torch.equal(lse, want)

    b = bounds_of(c)
    pages = torch.zeros(5, G, 4, dtype=torch.int32, device=DEV)
    y, lse = outputs(5, M, H, d, dtype)
    bx.beagle_xattn_draft_step_paged_blocks(desc, handle, x, eye, eye, None, ints(n_true), bits, words, dev(b, dtype), 33, 4, 4, pages, y, lse,
                                            workspace(desc, handle, bx.BEAGLE_WS_PAGED_DRAFT_BLOCKS))
    torch.cuda.synchronize()
    assert torch.equal(pages, select(c, q, b, 33, 4, 4, dtype, n_true=n_true))
    assert np.array_equal(pages.cpu().numpy(), pc.select(c, q, b, 33, 4, 4, n_true=n_true))
    o, want = blocks(c, q, pages.cpu().numpy(), 33, 4, dtype, n_true=n_true, tree=tree)
    assert torch.equal(y, o) and torch.equal(lse, want)


@pytest.mark.parametrize("dtype,H,G,d", [("bf16", 8, 2, 128), ("f32", 4, 2, 64)])
@pytest.mark.parametrize("M", [2, 30])
def test_rotated_steps_agree_with_the_step_on_all_rows(dtype, H, G, d, M):
    """With every page listed, and with the rows that branches have in common, the rows seen are those of the plain paged step, on the same
    projected and rotated queries.  Outputs o round to half a step each (2^-8 of at most 6, 2^-24), y sums H d = 1024 (256) of them by weights of
    at most 0.25 and rounds again; float sums are off by less than that."""
    rng = np.random.default_rng(M)
    c, first, n = branches(rng, [200, 90], [3, 2], [40, 70, 39, 130, 55], 16, G, d, dtype)
    B, D = 5, 512
    t, handle = on_gpu(c, dtype)
    x = dev(stored(rng.standard_normal((B, M, D)), dtype), dtype)
    wq, wo = (dev(np.clip(0.05 * rng.standard_normal(s), -0.25, 0.25), dtype) for s in ((D, H * d), (H * d, D)))
    desc = desc_for(B, M, H, G, d, dtype, hidden=D, flags=bx.BEAGLE_FLAG_ROPE)
    out = []
    for _ in range(3):
        out.append((torch.full((B, M, D), float("nan"), dtype=tdt(dtype), device=DEV), torch.full((B, H, M), float("nan"), device=DEV)))
    bx.beagle_xattn_draft_step_paged(desc, handle, x, wq, wo, None, None, None, 0, 0, 0, *out[0], workspace(desc, handle, bx.BEAGLE_WS_PAGED_DRAFT))
    bx.beagle_xattn_draft_step_paged_shared(desc, handle, x, wq, wo, None, ints(first), ints(n), 2, None, None, 0, *out[1],
                                            workspace(desc, handle, bx.BEAGLE_WS_PAGED_DRAFT_SHARED))
    pages = torch.zeros(B, G, 40, dtype=torch.int32, device=DEV)
    bx.beagle_xattn_draft_step_paged_blocks(desc, handle, x, wq, wo, None, None, None, 0, dev(bounds_of(c), dtype), 0, 0, 40, pages, *out[2],
                                            workspace(desc, handle, bx.BEAGLE_WS_PAGED_DRAFT_BLOCKS))
    torch.cuda.synchronize()
    half = 2.0 ** -8 if dtype == "bf16" else 2.0 ** -24
    want, lse = host(out[0][0]), host(out[0][1])
    most = host(torch.cat([t["v"][p].flatten() for p in range(len(c["refs"])) if c["refs"][p]]).nan_to_num(0.0)).__abs__().max()
    weight = np.abs(host(wo)).sum(0).max()
    for y, l in out[1:]:
        # two stored o's that each are half a step from nearly the same number, two y's likewise; float sums: 512 roundings
        tol = 2 * half * most * weight + 2 * half * np.abs(want) + 512 * 2.0 ** -24 * most * weight
        assert (np.abs(host(y) - want) <= tol).all() and np.isfinite(host(y)).all()
        assert np.abs(host(l) - lse).max() <= 512 * 2.0 ** -24 * (1 + np.abs(lse).max())
