"""GPU parity of the paged cache against its float64 oracle.

Tolerances count roundings.  A score is off by at most err (oracle: (d + 4) 2^-24 sum |q k| scale + 2^-22 |s|), a probability by
2 err of itself, a float sum of n terms by (n + 64) 2^-24 of the sum of magnitudes, a probability stored as two bf16 numbers by
2^-16 of itself; the result rounds once, by 2^-8 (bf16) or 2^-24 (float) of itself.  Rows that are only moved have to be equal,
rotated ones within the rounding of two products and a sum (3 * 2^-24) and of the result."""
import copy

import numpy as np
import pytest
import torch

from oracle import beagle_oracle as orc
from oracle import paged_oracle as po
from paper_2505_24544_amd import binding as bx
from paper_2505_24544_amd import synth

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def tdt(dtype):
    return torch.bfloat16 if dtype == "bf16" else torch.float32


def stored(a, dtype):
    a = np.asarray(a, np.float32)
    return (synth.round_to_bf16(a) if dtype == "bf16" else a).astype(np.float64)


def dev(a, dtype):
    return torch.from_numpy(np.ascontiguousarray(a, np.float32)).to(tdt(dtype)).to(DEV).contiguous()


def ints(v):
    return None if v is None else torch.tensor(v, dtype=torch.int32, device=DEV)


def host(t):
    return t.detach().cpu().double().numpy()


def make(rng, lens, page, W, P, G, d, dtype, stale=np.nan):
    """An oracle cache whose slots hold `lens` rows in random pages; rows that nobody holds are `stale`."""
    k, v = (np.full((P, page, G, d), stale) for _ in range(2))
    c = dict(k=k, v=v, table=[[-1] * W for _ in lens], lens=list(lens), refs=[0] * P)
    order = [int(p) for p in rng.permutation(P)]
    for s, n in enumerate(lens):
        for i in range(po.pages_of(n, page)):
            c["table"][s][i] = order.pop()
            c["refs"][c["table"][s][i]] = 1
        for p, r in po.rows_of(c, s, n):
            k[p, r], v[p, r] = stored(1.28 * rng.standard_normal((G, d)), dtype), stored(rng.standard_normal((G, d)), dtype)
    return c


def on_gpu(c, dtype):
    t = dict(k=dev(c["k"], dtype), v=dev(c["v"], dtype), table=ints(c["table"]), lens=ints(c["lens"]), refs=ints(c["refs"]))
    return t, bx.make_paged_cache(t["k"], t["v"], t["table"], t["lens"], t["refs"])


def desc_for(B, M, H, G, d, dtype, rows=1 << 20, **kw):
    return bx.make_desc(batch=B, seq_q=M, seq_kv=rows, hidden=kw.pop("hidden", 512), n_q_heads=H, n_kv_heads=G, head_dim=d,
                        io_dtype=bx.BEAGLE_BF16 if dtype == "bf16" else bx.BEAGLE_F32, **kw)


def workspace(desc, handle, which):
    n = bx.beagle_xattn_paged_workspace_bytes(desc, handle, which)
    assert n > 0
    return torch.full((n,), 0xFF, dtype=torch.uint8, device=DEV)          # (nan, whatever it is read as)


def pack(tree):
    """bool [B, M, T] -> int32 words"""
    B, M, T = tree.shape
    words = max(1, -(-T // 32))
    bits = np.zeros((B, M, words * 32), np.uint32)
    bits[:, :, :T] = tree
    w = (bits.reshape(B, M, words, 32) << np.arange(32, dtype=np.uint32)).sum(-1, dtype=np.uint32)
    return torch.from_numpy(w.view(np.int32).copy()).to(DEV), words


def attend(c, q, dtype, *, slots=None, n_true=None, tree=None, window=0, sinks=0, scale=0.0, rows=1 << 20):
    B, M, H, d = q.shape
    t, handle = on_gpu(c, dtype)
    desc = desc_for(B, M, H, c["k"].shape[2], d, dtype, rows, softmax_scale=scale)
    o = torch.full((B, M, H, d), float("nan"), dtype=tdt(dtype), device=DEV)
    lse = torch.full((B, H, M), float("nan"), dtype=torch.float32, device=DEV)
    bits, words = (None, 0) if tree is None else pack(tree)
    bx.beagle_xattn_paged_attend(desc, handle, dev(q, dtype), ints(slots), ints(n_true), bits, words, window, sinks, o, lse,
                                 workspace(desc, handle, bx.BEAGLE_WS_PAGED_ATTEND))
    torch.cuda.synchronize()
    return o, lse


def check_attend(c, q, dtype, **kw):
    print("attend", dtype, q.shape, c["k"].shape, {k: v for k, v in kw.items() if k != "tree"}, flush=True)
    o, lse = attend(c, q, dtype, **kw)
    ref, rlse, spread, err = po.attend(c, q, slots=kw.get("slots"), n_true=kw.get("n_true"), tree=kw.get("tree"), window=kw.get("window", 0),
                                       sinks=kw.get("sinks", 0), scale=kw.get("scale") or None, bound=kw.get("rows"))
    n = max(c["lens"]) + 64
    e = err.transpose(0, 2, 1)[..., None]
    half = 2.0 ** -8 if dtype == "bf16" else 2.0 ** -24
    tol = half * np.abs(ref) + spread * (1 + half) * (2 * e + n * 2.0 ** -23 + (2.0 ** -16 if dtype == "bf16" else 0)) + 1e-37
    got, glse = host(o), host(lse)
    assert np.isfinite(got).all()
    assert (np.abs(got - ref) <= tol).all(), (np.abs(got - ref) / tol).max()
    seen = np.isfinite(rlse)
    assert np.array_equal(np.isneginf(glse), ~seen)
    far = np.abs(glse - np.where(seen, rlse, 0))[seen]
    assert (far <= (2 * err + n * 2.0 ** -23 + 2.0 ** -22 * np.abs(np.where(seen, rlse, 0)))[seen]).all(), far.max()
    return o, lse


def queries(rng, B, M, H, d, dtype, std=1.0):
    return stored(std * rng.standard_normal((B, M, H, d)), dtype)


# ------------------------------------------------------------------ attention
HEADS = [("bf16", 4, 4, 128), ("bf16", 8, 2, 128), ("bf16", 5, 1, 128), ("f32", 4, 2, 64), ("f32", 3, 3, 128), ("f32", 6, 2, 20), ("f32", 2, 1, 4), ("f32", 4, 1, 100)]


@pytest.mark.parametrize("dtype,H,G,d", HEADS)
@pytest.mark.parametrize("M,page,lens", [(1, 16, [1, 0, 31, 33, 700]), (3, 4, [129, 2, 64]), (7, 64, [65, 1000, 5, 128])])
@pytest.mark.parametrize("room", [1, 1000])              # short sequences by what a slot can hold, or not: another launch
def test_lengths_heads_and_pages(dtype, H, G, d, M, page, lens, room):
    rng = np.random.default_rng(hash((H, G, d, M)) % 1000)
    W = po.pages_of(max(lens), page) + room
    c = make(rng, lens, page, W, sum(po.pages_of(n, page) for n in lens) + 3, G, d, dtype)
    check_attend(c, queries(rng, len(lens), M, H, d, dtype), dtype)


@pytest.mark.parametrize("dtype,H,G,d", [("bf16", 8, 2, 128), ("f32", 4, 2, 64)])
@pytest.mark.parametrize("window,sinks", [(1, 0), (1, 1), (32, 4), (33, 32), (100, 0), (100, 33), (500, 7), (5000, 4), (40, 300), (64, 1000)])
def test_window_and_sinks(dtype, H, G, d, window, sinks):
    rng = np.random.default_rng(window + sinks)
    lens = [900, 0, 3, 32, 65, 301, 133]
    c = make(rng, lens, 16, 64, 110, G, d, dtype)
    check_attend(c, queries(rng, 7, 2, H, d, dtype), dtype, window=window, sinks=sinks)


@pytest.mark.parametrize("dtype,H,G,d", [("bf16", 8, 2, 128), ("f32", 4, 4, 64), ("f32", 2, 2, 100)])
@pytest.mark.parametrize("M,T,window", [(5, 40, 0), (10, 3, 50), (1, 33, 0), (20, 64, 20)])
@pytest.mark.parametrize("W", [96, 1000])
def test_drafted_rows_under_a_tree(dtype, H, G, d, M, T, window, W):
    rng = np.random.default_rng(M + T)
    true = [300, 0, 31, 64, 700]
    c = make(rng, [n + T for n in true], 8, W, 220, G, d, dtype)
    tree = rng.random((5, M, T)) < 0.4
    tree[1, 0] = False                                    # with no true row: sees nothing at all
    tree[3] = False
    check_attend(c, queries(rng, 5, M, H, d, dtype), dtype, n_true=true, tree=tree, window=window, sinks=3 if window else 0)


@pytest.mark.parametrize("dtype,d", [("bf16", 128), ("f32", 64)])
@pytest.mark.parametrize("M,W", [(18, 10), (18, 1000), (6, 10), (6, 1000)])
def test_drafted_rows_that_are_no_numbers_reach_only_who_sees_them(dtype, d, M, W):
    rng = np.random.default_rng(17)
    T = 20
    c = make(rng, [90 + T, 33 + T], 16, W, 20, 2, d, dtype)
    for s, n in ((0, 90), (1, 33)):
        place = po.rows_of(c, s, n + T)
        c["v"][place[n + 2]][0, ::3] = np.inf
        c["v"][place[n + 5]] = np.nan
        c["k"][place[n + 7]] = np.nan
    tree = rng.random((2, M, T)) < 0.5
    tree[:, ::2, [2, 5, 7]] = False
    tree[:, 1, [2, 5, 7]] = True
    q = queries(rng, 2, M, 4, d, dtype)
    o, lse = attend(c, q, dtype, n_true=[90, 33], tree=tree)
    clean = copy.deepcopy(c)
    for name in ("k", "v"):
        clean[name] = np.where(np.isfinite(clean[name]), clean[name], 0.0)
    o2, lse2 = check_attend(clean, q, dtype, n_true=[90, 33], tree=tree)
    spared = ~tree[:, :, [2, 5, 7]].any(-1)
    assert spared.sum() >= M
    a, b = host(o)[spared], host(o2)[spared]
    assert np.isfinite(a).all() and np.abs(a - b).max() <= (2 ** -7 if dtype == "bf16" else 2 ** -20) * np.abs(b).max()
    assert np.array_equal(host(lse).transpose(0, 2, 1)[spared], host(lse2).transpose(0, 2, 1)[spared])
    assert np.isnan(host(o)[:, 1]).all()


@pytest.mark.parametrize("dtype,H,G,d", [("bf16", 32, 8, 128), ("f32", 8, 2, 64), ("f32", 8, 2, 128)])
@pytest.mark.parametrize("W", [9, 100])
def test_more_rows_than_one_tile(dtype, H, G, d, W):
    rng = np.random.default_rng(23)
    c = make(rng, [260, 31], 32, W, 12, G, d, dtype)
    check_attend(c, queries(rng, 2, 25, H, d, dtype), dtype)                # 100 rows a kv head: tiles of 32, the last ragged


def test_shared_slots_ragged_order_and_scale():
    rng = np.random.default_rng(29)
    c = make(rng, [700, 40, 1], 16, 50, 60, 2, 128, "bf16")
    q = queries(rng, 6, 2, 8, 128, "bf16")
    check_attend(c, q, "bf16", slots=[2, 0, 0, 1, 2, 0], scale=0.3)
    check_attend(c, q, "bf16", slots=[0, -1, 3, 1, 2 ** 31 - 1, -2 ** 31])      # slots that are none
    check_attend(c, q, "bf16", slots=[2, 0, 0, 1, 2, 0], rows=333)              # rows behind the bound


def test_peaked_scores_and_their_order():
    """One key far above the rest, at the start, in the middle and at the end, so that running maxima change late or at once."""
    for dtype, d in (("bf16", 128), ("f32", 64)):
        rng = np.random.default_rng(31)
        c = make(rng, [1500, 1500, 1500], 16, 100, 300, 1, d, dtype)
        q = queries(rng, 3, 2, 2, d, dtype, std=3.0)
        for s, at in ((0, 0), (1, 777), (2, 1499)):
            c["k"][po.rows_of(c, s, 1500)[at]] = stored(q[s, 0, 0], dtype) * 4
        check_attend(c, q, dtype)


def test_pages_that_are_none_hide_their_rows():
    for dtype, d in (("bf16", 128), ("f32", 32)):
        rng = np.random.default_rng(37)
        c = make(rng, [200, 90, 64], 16, 16, 40, 2, d, dtype)
        c["table"][0][3], c["table"][0][12], c["table"][1][0], c["table"][2][:4] = -1, 40, 2 ** 31 - 1, [-2 ** 31] * 4
        check_attend(c, queries(rng, 3, 3, 4, d, dtype), dtype)
        c["lens"] = [10 ** 9, -5, 64]                     # lengths that no slot can have
        c["table"][0] = [-1] * 16
        check_attend(c, queries(rng, 3, 3, 4, d, dtype), dtype)


def test_split_sequences_are_reproducible_and_do_not_depend_on_the_batch():
    rng = np.random.default_rng(41)
    lens = [6000, 10, 2500]
    c = make(rng, lens, 64, 100, 150, 2, 128, "bf16")
    q = queries(rng, 3, 4, 8, 128, "bf16")
    o1, l1 = check_attend(c, q, "bf16")
    o2, l2 = attend(c, q, "bf16")
    assert torch.equal(o1.view(torch.int16), o2.view(torch.int16)) and torch.equal(l1.view(torch.int32), l2.view(torch.int32))


@pytest.mark.parametrize("lens,W", [([900, 700, 500, 300], 100), ([900, 700, 500, 300], 57), ([2000, 1800, 100, 5], 130), ([400, 0, 333, 1], 100)])
def test_how_entries_are_cut(lens, W):
    """16 workers a head: runs of eight blocks each, whole entries, equal runs of all, runs of four."""
    rng = np.random.default_rng(sum(lens) + W)
    c = make(rng, lens, 16, W, sum(-(-n // 16) for n in lens) + 1, 32, 128, "bf16")
    check_attend(c, queries(rng, 4, 1, 32, 128, "bf16"), "bf16", rows=2000)


def test_more_entries_than_workers_and_than_a_wave_has_lanes():
    rng = np.random.default_rng(44)
    lens = [int(n) for n in rng.integers(0, 300, 70)]
    c = make(rng, lens, 16, 200, 1400, 8, 4, "f32")
    check_attend(c, queries(rng, 70, 2, 16, 4, "f32"), "f32")


def test_many_entries():
    """More entries than a wave looks at once."""
    rng = np.random.default_rng(43)
    lens = [int(n) for n in rng.integers(0, 90, 150)]
    lens[77] = 3000
    c = make(rng, lens, 16, 200, 1000, 1, 64, "f32")
    check_attend(c, queries(rng, 150, 1, 2, 64, "f32"), "f32")


def test_pool_past_32_bit_offsets():
    """A pool of more than 4 GiB per tensor, pages at both ends; and the same rows in a small pool give the same bits."""
    P, page, G, d = 36000, 64, 8, 128                      # 4.7 GB each
    rng = np.random.default_rng(47)
    small = make(rng, [600, 65], page, 10, 14, G, d, "bf16")
    q = queries(rng, 2, 2, 16, d, "bf16")
    o1, l1 = check_attend(small, q, "bf16")
    to = [int(v) for v in rng.permutation(14)]
    far = [i if i < 5 else P - 14 + i for i in to]
    k, v = (torch.empty(P, page, G, d, dtype=torch.bfloat16, device=DEV) for _ in range(2))
    for i, p in enumerate(far):
        k[p], v[p] = dev(small["k"][i], "bf16"), dev(small["v"][i], "bf16")
    table = ints([[far[p] if p >= 0 else -1 for p in row] for row in small["table"]])
    lens, refs = ints(small["lens"]), torch.zeros(P, dtype=torch.int32, device=DEV)
    for p in far:
        refs[p] = 1
    handle = bx.make_paged_cache(k, v, table, lens, refs)
    desc = desc_for(2, 2, 16, G, d, "bf16")
    o, lse = torch.empty_like(o1), torch.empty_like(l1)
    bx.beagle_xattn_paged_attend(desc, handle, dev(q, "bf16"), None, None, None, 0, 0, 0, o, lse, workspace(desc, handle, bx.BEAGLE_WS_PAGED_ATTEND))
    assert torch.equal(o.view(torch.int16), o1.view(torch.int16)) and torch.equal(lse, l1)
    # appending at the far end, and moving it all into a small pool
    refs.fill_(1)
    refs[P - 1] = 0
    held = {p for p in far}
    if P - 1 in held:
        refs[P - 1] = 1
        refs[P - 20] = 0
    new = torch.randn(2, 64, G, d, device=DEV).to(torch.bfloat16)
    d2 = desc_for(2, 64, G, G, d, "bf16")
    short = torch.zeros(1, dtype=torch.int32, device=DEV)
    bx.beagle_xattn_paged_append(d2, handle, None, None, ints([0, 64]), new, -new, short, workspace(d2, handle, bx.BEAGLE_WS_PAGED_APPEND))
    assert short.item() == 0 and lens.tolist() == [600, 129]
    p = table[1, 2].item()
    assert p in (P - 1, P - 20)
    rows = torch.cat([k[table[1, 1].item(), 1:], k[p, :1]])
    assert torch.equal(rows, new[1])


# ------------------------------------------------------------------ what changes a cache
def whole(c, t, dtype, rotated=()):
    """The tensors hold the oracle's state: equal, but for the rotated K rows (page, row)."""
    assert t["lens"].tolist() == c["lens"] and t["refs"].tolist() == c["refs"] and t["table"].tolist() == c["table"]
    k, v = host(t["k"]), host(t["v"])
    assert np.array_equal(v, c["v"], equal_nan=True)
    at = np.zeros(c["k"].shape[:2], bool)
    for p, r in rotated:
        at[p, r] = True
    assert np.array_equal(k[~at], c["k"][~at], equal_nan=True)
    if at.any():
        want, half = c["k"][at], 2.0 ** -8 if dtype == "bf16" else 2.0 ** -24
        d = want.shape[-1]
        size = np.sqrt(want[..., : d // 2] ** 2 + want[..., d // 2:] ** 2)       # of the pair: both products are below it
        size = np.concatenate([size, size], -1)
        assert (np.abs(k[at] - want) <= half * np.abs(want) + 5 * 2.0 ** -24 * size).all()


def run_append(c, dtype, k_new, v_new, *, slots=None, pos=None, n_new=None, rope=None, positions=None):
    B, M, G, d = k_new.shape
    print("append", dtype, k_new.shape, c["k"].shape, slots, pos, n_new, rope, flush=True)
    t, handle = on_gpu(c, dtype)
    at = ints(positions)
    desc = desc_for(B, M, G, G, d, dtype, flags=bx.BEAGLE_FLAG_ROPE if rope else 0, rope_base=rope or 0.0, rope_positions=at)
    short = torch.full((1,), -7, dtype=torch.int32, device=DEV)
    bx.beagle_xattn_paged_append(desc, handle, ints(slots), ints(pos), ints(n_new), dev(k_new, dtype), dev(v_new, dtype), short,
                                 workspace(desc, handle, bx.BEAGLE_WS_PAGED_APPEND))
    torch.cuda.synchronize()
    ref, missing = po.append(c, k_new, v_new, slots=slots, pos=pos, n_new=n_new, rope_base=rope, positions=positions)
    assert short.item() == missing
    rotated = []
    if rope:
        for b in range(B):
            s = b if slots is None else slots[b]
            if 0 <= s < len(ref["lens"]) and s not in [b2 if slots is None else slots[b2] for b2 in range(b)]:
                had = po.length(c, s)
                at0 = had if pos is None else min(max(pos[b], 0), had)
                rotated += po.rows_of(ref, s, ref["lens"][s])[at0:]
    whole(ref, t, dtype, rotated)
    return ref, t


def new_rows(rng, B, M, G, d, dtype):
    return stored(rng.standard_normal((B, M, G, d)), dtype), stored(rng.standard_normal((B, M, G, d)), dtype)


ROWS = [("bf16", 2, 128), ("bf16", 5, 128), ("f32", 2, 64), ("f32", 1, 12), ("f32", 3, 128), ("f32", 2, 4)]


@pytest.mark.parametrize("dtype,G,d", ROWS)
@pytest.mark.parametrize("page", [4, 16, 64])
@pytest.mark.parametrize("rope", [None, 10000.0])
def test_append(dtype, G, d, page, rope):
    rng = np.random.default_rng(G + d + page)
    lens = [0, 5, 16, 100, 63, 64]
    c = make(rng, lens, page, 240 // page, 6 * (240 // page), G, d, dtype, stale=7.0)
    for M, pos, n_new in ((1, None, None), (9, [0, 3, 16, 64, 50, 1], [9, 0, 4, 9, 1, 20]), (70, [5, 99, -3, 31, 63, 0], None)):
        kn, vn = new_rows(rng, 6, M, G, d, dtype)
        run_append(c, dtype, kn, vn, slots=[3, 0, 5, 2, 1, 4], pos=pos, n_new=n_new, rope=rope)


def test_append_given_positions_and_slots_that_do_not_count():
    rng = np.random.default_rng(3)
    c = make(rng, [10, 20, 30], 8, 10, 24, 2, 128, "bf16", stale=0.5)
    kn, vn = new_rows(rng, 6, 3, 2, 128, "bf16")
    positions = [[int(v) for v in rng.integers(0, 100000, 3)] for _ in range(6)]
    run_append(c, "bf16", kn, vn, slots=[1, -1, 1, 3, 0, 1], pos=[20, 0, 0, 0, 3, 5], rope=500.0, positions=positions)


def test_append_copies_shared_pages_and_only_those():
    for dtype, d in (("bf16", 128), ("f32", 16)):
        rng = np.random.default_rng(5)
        c = make(rng, [37, 0, 0, 50, 0], 16, 8, 20, 2, d, dtype, stale=2.0)
        c = po.fork(c, [1, 2, 4], [0, 0, 3], [37, 32, 45])
        kn, vn = new_rows(rng, 5, 20, 2, d, dtype)
        run_append(c, dtype, kn, vn, slots=[1, 0, 2, 3, 4], n_new=[1, 2, 20, 0, 5], rope=100.0)      # 0 and 1 part, 3 keeps the shared page
        run_append(c, dtype, kn, vn, slots=[4, 3, 2, 1, 0], pos=[33, 32, 5, 16, 15], n_new=[3, 3, 3, 3, 0])
        run_append(c, dtype, kn, vn, pos=[20, 20, 20, 20, 20])


def test_append_copies_large_pages_of_many_entries():
    """More to copy of each page than the workgroups of an entry take at once."""
    rng = np.random.default_rng(6)
    c = make(rng, [255] + [0] * 127, 256, 2, 260, 2, 128, "f32", stale=2.0)
    c = po.fork(c, list(range(1, 128)), [0] * 127, [int(n) for n in rng.integers(1, 256, 127)])
    kn, vn = new_rows(rng, 128, 2, 2, 128, "f32")
    run_append(c, "f32", kn, vn, n_new=[int(n) for n in rng.integers(0, 3, 128)])


def test_append_to_a_full_pool():
    rng = np.random.default_rng(7)
    c = make(rng, [10, 10, 10, 10, 8], 8, 6, 12, 1, 64, "f32", stale=1.0)       # 9 of 12 pages held
    kn, vn = new_rows(rng, 5, 20, 1, 64, "f32")
    run_append(c, "f32", kn, vn, n_new=[6, 7, 14, 1, 20])                      # the third and the last go without
    run_append(c, "f32", kn, vn, pos=[2, 10, 0, 10, 8], n_new=[20, 20, 0, 0, 20])
    run_append(c, "f32", kn, vn, pos=[0, 0, 0, 0, 0], n_new=[20] * 5)
    big = new_rows(rng, 5, 50, 1, 64, "f32")
    run_append(c, "f32", *big, n_new=[1, 38, 39, 50, 0])                        # more than a slot holds: 38 is what fits
    c["table"][0][1] = -1                                                       # the page to write into is none
    c["refs"] = [int(any(p in row for row in c["table"])) for p in range(12)]
    run_append(c, "f32", kn, vn, n_new=[3, 0, 0, 0, 0])


def test_append_long_and_wide():
    rng = np.random.default_rng(11)
    c = make(rng, [130, 0], 32, 60, 100, 8, 128, "bf16", stale=0.0)
    kn, vn = new_rows(rng, 2, 1500, 8, 128, "bf16")
    run_append(c, "bf16", kn, vn, rope=10000.0)


def test_many_slots_and_pages():
    """More entries than the planning workgroup has threads, more pages than it looks at once, most of them held."""
    rng = np.random.default_rng(13)
    N, P = 1500, 9000
    c = make(rng, [int(n) for n in rng.integers(0, 9, N)], 4, 4, P, 1, 4, "f32", stale=3.0)
    for p in rng.permutation(P)[:4000]:
        c["refs"][p] = max(c["refs"][p], 1)
    kn, vn = new_rows(rng, N, 5, 1, 4, "f32")
    run_append(c, "f32", kn, vn, slots=[int(s) for s in rng.permutation(N)], n_new=[int(n) for n in rng.integers(0, 6, N)])


def run_fork(c, dst, src, rows=None):
    t, handle = on_gpu(c, "f32")
    desc = desc_for(len(dst), 1, 1, 1, c["k"].shape[3], "f32")
    bx.beagle_xattn_paged_fork(desc, handle, ints(dst), ints(src), ints(rows), workspace(desc, handle, bx.BEAGLE_WS_PAGED_FORK))
    torch.cuda.synchronize()
    ref = po.fork(c, dst, src, rows)
    whole(ref, t, "f32")
    return ref


def test_fork():
    rng = np.random.default_rng(19)
    c = make(rng, [50, 0, 17, 16, 1, 200], 8, 30, 60, 1, 4, "f32", stale=1.0)
    c = run_fork(c, [1], [0])
    c = run_fork(c, [3, 4], [0, 2], [33, 100])                     # what 3 and 4 held is given up
    c = run_fork(c, [0, 1, 2, 3, 4, 5], [5, 0, 1, 2, 3, 4])        # a cycle: everybody takes the old state of another
    c = run_fork(c, [0, 1, 2], [2, 2, 2], [9, 200, 0])             # one survivor takes over
    c = run_fork(c, [4, 4, 4], [4, 5, -1], [3, 1, 1])              # the first entry counts: shortened
    c = run_fork(c, [0, -1, 6, 2 ** 31 - 1, 1], [1, 0, 0, 0, 99])  # targets that are none; a source that is none frees
    c = run_fork(c, list(range(6)), [-1] * 6)
    assert c["refs"] == [0] * 60 and c["lens"] == [0] * 6
    c["table"][2], c["lens"][2] = [60, -7, 3] + [-1] * 27, 20      # pages that are none are passed on, and counted nowhere
    run_fork(c, [2, 0], [2, 2], [10, 20])


def test_fork_of_more_than_one_workgroup_takes():
    rng = np.random.default_rng(23)
    N = 300
    c = make(rng, [int(n) for n in rng.integers(0, 120, N)], 4, 40, 12000, 1, 4, "f32", stale=0.0)
    order = [int(s) for s in rng.permutation(N)]
    c = run_fork(c, order + order[:20], [int(s) for s in rng.integers(-1, N, N + 20)], [int(n) for n in rng.integers(0, 130, N + 20)])
    run_fork(c, list(range(N)), order)                             # a permutation


def run_compact(c, into, dtype):
    t, handle = on_gpu(c, dtype)
    u, target = on_gpu(into, dtype)
    desc = desc_for(1, 1, 1, c["k"].shape[2], c["k"].shape[3], dtype) if c["k"].shape[2] == 1 else \
        desc_for(1, 1, c["k"].shape[2], c["k"].shape[2], c["k"].shape[3], dtype)
    short = torch.full((1,), -7, dtype=torch.int32, device=DEV)
    bx.beagle_xattn_paged_compact(desc, handle, target, short, workspace(desc, handle, bx.BEAGLE_WS_PAGED_COMPACT))
    torch.cuda.synchronize()
    ref, missing = po.compact(c, into)
    assert short.item() == missing
    whole(ref, u, dtype)
    whole(c, t, dtype)
    return ref


@pytest.mark.parametrize("dtype,G,d,page", [("bf16", 2, 128, 16), ("f32", 1, 12, 4), ("f32", 3, 64, 64)])
def test_compact(dtype, G, d, page):
    rng = np.random.default_rng(G + d)
    lens = [3 * page + 1, 0, page, 5 * page - 1, 1]
    c = make(rng, lens, page, 6, 40, G, d, dtype, stale=4.0)
    c = po.fork(c, [1], [3], [2 * page + 1])
    blank = lambda P, W: dict(make(rng, [0] * 5, page, W, P, G, d, dtype, stale=9.0), lens=[5] * 5, refs=[3] * P)      # noqa: E731
    run_compact(c, blank(60, 6), dtype)                    # larger
    run_compact(c, blank(po.pages_of(3 * page + 1, page) + 7, 5), dtype)        # exactly the live pages
    run_compact(c, blank(6, 6), dtype)                     # too small
    run_compact(c, blank(60, 3), dtype)                    # a narrower table
    run_compact(blank(5, 4) | dict(lens=[0] * 5, refs=[0] * 5), blank(3, 3), dtype)         # nothing to move
    c["table"][3][1] = -1                                  # a sequence that a lost page cuts
    run_compact(c, blank(60, 6), dtype)


def test_compact_many_pages():
    rng = np.random.default_rng(2)
    c = make(rng, [int(n) for n in rng.integers(0, 60, 300)], 4, 16, 6000, 1, 8, "f32", stale=0.0)
    run_compact(c, dict(make(rng, [0] * 300, 4, 16, 4000, 1, 8, "f32", stale=0.0)), "f32")


# ------------------------------------------------------------------ together, as a program uses them
def test_a_drafting_loop_and_its_graph():
    """Prompts in, sequences forked, a depth of drafted rows appended behind the true ones and attended under a tree, the
    accepted states in their place; eager against the oracle, then the depth captured and replayed between eager work."""
    dtype, H, G, d, page, B = "bf16", 8, 2, 128, 16, 4
    rng = np.random.default_rng(53)
    c = make(rng, [0] * 6, page, 20, 90, G, d, dtype, stale=0.0)
    t, handle = on_gpu(c, dtype)
    slots, true = [0, 1, 4, 5], [100, 33, 70, 33]

    def put(c, kn, vn, desc, ws, **kw):
        bx.beagle_xattn_paged_append(desc, handle, *(ints(kw.get(n)) for n in ("slots", "pos", "n_new")), dev(kn, dtype), dev(vn, dtype), None, ws)
        return po.append(c, kn, vn, **kw)[0]

    d100, d5 = desc_for(2, 100, H, G, d, dtype), desc_for(B, 5, H, G, d, dtype)
    kn, vn = new_rows(rng, 2, 100, G, d, dtype)
    c = put(c, kn, vn, d100, workspace(d100, handle, bx.BEAGLE_WS_PAGED_APPEND), slots=[0, 1], n_new=[100, 33])
    dd = desc_for(2, 1, H, G, d, dtype)
    bx.beagle_xattn_paged_fork(dd, handle, ints([4, 5]), ints([0, 1]), ints([70, 33]), workspace(dd, handle, bx.BEAGLE_WS_PAGED_FORK))
    c = po.fork(c, [4, 5], [0, 1], [70, 33])
    whole(c, t, dtype)
    ws_a, ws_t = workspace(d5, handle, bx.BEAGLE_WS_PAGED_APPEND), workspace(d5, handle, bx.BEAGLE_WS_PAGED_ATTEND)
    sl, nt = ints(slots), ints(true)
    kd, vd = (torch.empty(B, 5, G, d, dtype=torch.bfloat16, device=DEV) for _ in range(2))
    qd, o = (torch.empty(B, 5, H, d, dtype=torch.bfloat16, device=DEV) for _ in range(2))
    lse = torch.empty(B, H, 5, dtype=torch.float32, device=DEV)
    tree = np.tril(np.ones((5, 5), bool))[None].repeat(B, 0)
    bits, words = pack(tree)

    def depth():
        bx.beagle_xattn_paged_append(d5, handle, sl, nt, None, kd, vd, None, ws_a)
        bx.beagle_xattn_paged_attend(d5, handle, qd, sl, nt, bits, words, 0, 0, o, lse, ws_t)

    def step(run):
        nonlocal c
        kn, vn = new_rows(rng, B, 5, G, d, dtype)
        q = queries(rng, B, 5, H, d, dtype)
        kd.copy_(dev(kn, dtype)); vd.copy_(dev(vn, dtype)); qd.copy_(dev(q, dtype))
        o.fill_(float("nan")); lse.fill_(float("nan"))
        run()
        torch.cuda.synchronize()
        c = po.append(c, kn, vn, slots=slots, pos=true)[0]
        whole(c, t, dtype)
        ref, rlse, spread, err = po.attend(c, q, slots=slots, n_true=true, tree=tree)
        assert (np.abs(host(o) - ref) <= 2.0 ** -8 * np.abs(ref) + spread * (2 * err.transpose(0, 2, 1)[..., None] + 2.0 ** -14)).all()
        assert np.abs(host(lse) - rlse).max() <= 1e-4

    step(depth)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        depth()
    for _ in range(3):
        step(graph.replay)
        step(depth)
    # the accepted states take the drafted ones' place
    kn, vn = new_rows(rng, B, 5, G, d, dtype)
    c = put(c, kn, vn, d5, ws_a, slots=slots, pos=true, n_new=[2, 5, 0, 1])
    whole(c, t, dtype)
    true[:] = [102, 38, 70, 34]
    nt.copy_(ints(true))
    step(graph.replay)                                     # the graph reads lengths and positions as they are now


def test_calls_on_two_streams_with_a_workspace_each():
    rng = np.random.default_rng(59)
    c = make(rng, [3000, 1700], 16, 200, 310, 2, 128, "bf16")
    t, handle = on_gpu(c, "bf16")
    desc = desc_for(2, 3, 8, 2, 128, "bf16")
    qs = [dev(queries(rng, 2, 3, 8, 128, "bf16"), "bf16") for _ in range(2)]
    outs = []
    for _ in range(2):
        streams = [torch.cuda.Stream() for _ in range(2)]
        got = []
        torch.cuda.synchronize()
        for q, s in zip(qs, streams):
            with torch.cuda.stream(s):
                o, lse, ws = torch.empty_like(q), torch.empty(2, 8, 3, device=DEV), workspace(desc, handle, bx.BEAGLE_WS_PAGED_ATTEND)
                for _ in range(3):
                    bx.beagle_xattn_paged_attend(desc, handle, q, None, None, None, 0, 0, 0, o, lse, ws)       # the current stream
                got.append((o, lse, ws))
        torch.cuda.synchronize()
        outs.append(got)
    for (a, la, _), (b, lb, _) in zip(*outs):
        assert torch.equal(a.view(torch.int16), b.view(torch.int16)) and torch.equal(la, lb)


def contiguous(c, slot, n):
    place = po.rows_of(c, slot, n)
    return np.array([c["k"][p] for p in place]), np.array([c["v"][p] for p in place])


@pytest.mark.parametrize("dtype,M,B,d,H,G,D", [("bf16", 4, 3, 128, 4, 2, 512), ("bf16", 40, 2, 128, 4, 4, 512), ("f32", 3, 2, 64, 4, 2, 256)])
@pytest.mark.parametrize("rope", [False, True])
def test_draft_step_from_states(dtype, M, B, d, H, G, D, rope):
    """From states: appended by the projections, attended, projected; the oracle's draft step per sequence on the rows as they are stored."""
    rng = np.random.default_rng(M + B + D)
    c = make(rng, [0] * B, 16, 20, 20 * B, G, d, dtype, stale=0.0)
    t, handle = on_gpu(c, dtype)
    w = {n: stored(0.05 * rng.standard_normal(s), dtype) for n, s in (("wq", (D, H * d)), ("wk", (D, G * d)), ("wv", (D, G * d)), ("wo", (H * d, D)))}
    wd = {n: dev(a, dtype) for n, a in w.items()}
    flags = bx.BEAGLE_FLAG_ROPE if rope else 0
    n, T = [150, 40, 9][:B], 6
    x = stored(rng.standard_normal((B, 150, D)), dtype)
    da = desc_for(B, 150, H, G, d, dtype, hidden=D, flags=flags)
    bx.beagle_xattn_kv_append_paged(da, handle, dev(x, dtype), wd["wk"], wd["wv"], None, None, ints(n), None, workspace(da, handle, bx.BEAGLE_WS_PAGED_KV_APPEND))
    torch.cuda.synchronize()
    assert t["lens"].tolist() == n
    c = dict(k=host(t["k"]), v=host(t["v"]), table=t["table"].tolist(), lens=n, refs=t["refs"].tolist())
    half = 2.0 ** -8 if dtype == "bf16" else 2.0 ** -22
    for b in range(B):
        kr, vr = contiguous(c, b, n[b])
        want_v, want_k = (x[b, : n[b]] @ w["wv"]).reshape(n[b], G, d), (x[b, : n[b]] @ w["wk"]).reshape(n[b], G, d)
        if rope:
            want_k = np.stack([po.rotate(want_k[j], j, 10000.0) for j in range(n[b])])
        # bf16: the projection rounds, and the rotation rounds again (of either channel of a pair: sqrt 2)
        for got, want, size in ((vr, want_v, 1), (kr, want_k, 1 + 2 ** 0.5 if rope else 1)):
            assert np.abs(got - want).max() <= half * size * np.abs(want).max() * 1.01 + D * 2.0 ** -23
    xd = stored(rng.standard_normal((B, M, D)), dtype)
    dq = desc_for(B, M, H, G, d, dtype, hidden=D, flags=flags)
    n_true = [v - T for v in n]
    tree = rng.random((B, M, T)) < 0.5
    bits, words = pack(tree)
    y = torch.full((B, M, D), float("nan"), dtype=tdt(dtype), device=DEV)
    lse = torch.full((B, H, M), float("nan"), dtype=torch.float32, device=DEV)
    bx.beagle_xattn_draft_step_paged(dq, handle, dev(xd, dtype), wd["wq"], wd["wo"], None, ints(n_true), bits, words, 0, 0, y, lse,
                                     workspace(dq, handle, bx.BEAGLE_WS_PAGED_DRAFT))
    torch.cuda.synchronize()
    for b in range(B):
        q = (xd[b] @ w["wq"]).reshape(M, H, d)
        if rope:
            q = np.stack([po.rotate(q[m], n[b], 10000.0) for m in range(M)])
        kr, vr = contiguous(c, b, n[b])
        # the definition on the rows as stored: identity projections
        eye = np.eye(H * d)
        ref = orc.draft_step_tree(q.reshape(M, H * d), kr, vr, eye, w["wo"], n_true=n_true[b], tree_mask=tree[b], n_q_heads=H, n_kv_heads=G)
        # a score moves by what q's roundings (one, or two with the rotation) make of it
        move = np.abs(q).max() * half * (1 + 2 ** 0.5 if rope else 1) * np.abs(kr).sum(-1).max() * d ** -0.5
        assert np.abs(host(lse)[b] - ref["lse"]).max() <= move + 1e-4
        fro = np.linalg.norm(host(y)[b] - ref["y"]) / np.linalg.norm(ref["y"])
        assert fro <= (2e-2 if dtype == "bf16" else 1e-5), fro
