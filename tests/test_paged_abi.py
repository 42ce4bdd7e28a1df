"""Host side of the paged-cache entry points (CPU only): what is refused, with which status, before anything is enqueued,
and what the Python layer refuses by itself."""
import pytest
import torch

from paper_2505_24544_amd import binding as bx

A, WS = 4096, 1 << 40          # an aligned address that nothing reads; plenty of workspace


def _desc(B=2, M=3, H=4, G=2, d=128, dtype=bx.BEAGLE_BF16, hidden=512, **kw):
    return bx.make_desc(batch=B, seq_q=M, seq_kv=kw.pop("rows", 100), hidden=hidden, n_q_heads=H, n_kv_heads=G, head_dim=d, io_dtype=dtype, **kw)


def _cache(P=10, page=16, N=4, W=8, k=A, v=A, table=A, lens=A, refs=A, size=None, reserved=0):
    import ctypes as C
    return bx.beagle_paged_cache(C.sizeof(bx.beagle_paged_cache) if size is None else size, P, page, N, W, reserved, k, v, table, lens, refs)


def _far_cache():
    """Another pool, far enough from the first that their memory does not meet."""
    return _cache(k=1 << 30, v=1 << 31, table=1 << 32, lens=1 << 33, refs=1 << 34)


def _calls(desc, cache, ws=A, nbytes=WS):
    kw = dict(stream=0, workspace_bytes=nbytes, check=False)
    return {
        "attend": bx.beagle_xattn_paged_attend(desc, cache, A, A, A, A, 1, 0, 0, A, A, ws, **kw),
        "append": bx.beagle_xattn_paged_append(desc, cache, A, A, A, A, A, A, ws, **kw),
        "fork": bx.beagle_xattn_paged_fork(desc, cache, A, A, A, ws, **kw),
        "compact": bx.beagle_xattn_paged_compact(desc, cache, _far_cache(), A, ws, **kw),
        "draft": bx.beagle_xattn_draft_step_paged(desc, cache, A, A, A, A, A, A, 1, 0, 0, A, A, ws, **kw),
        "kv_append": bx.beagle_xattn_kv_append_paged(desc, cache, A, A, A, A, A, A, A, ws, **kw),
    }


BAD_DESC = [(dict(B=0), 2), (dict(M=0), 2), (dict(H=3), 2), (dict(rows=0), 2), (dict(softmax_scale=-1.0), 2), (dict(softmax_scale=float("nan")), 2),
            (dict(d=64), 3), (dict(dtype=5), 3), (dict(B=8193), 3), (dict(M=1 << 28), 3), (dict(flags=bx.BEAGLE_FLAG_NEED_DXKV), 3),
            (dict(flags=1 << 9), 3), (dict(d=6, dtype=bx.BEAGLE_F32), 3), (dict(d=132, dtype=bx.BEAGLE_F32), 3),
            (dict(cu_seqlens_q=A, cu_seqlens_kv=A, total_q=2, total_kv=2), 3), (dict(flags=bx.BEAGLE_FLAG_ROPE, rope_positions=2), 5),
            (dict(flags=bx.BEAGLE_FLAG_ROPE, rope_base=-2.0), 2), (dict(H=1 << 20, G=1 << 20), 3)]


@pytest.mark.parametrize("kw,status", BAD_DESC)
def test_bad_descriptors(kw, status):
    got = _calls(_desc(**kw), _cache())
    assert set(got.values()) == {status}, got
    for which in range(6):
        assert bx.beagle_xattn_paged_workspace_bytes(_desc(**kw), _cache(), which) == 0


BAD_CACHE = [(dict(P=0), 2), (dict(page=0), 2), (dict(N=0), 2), (dict(W=0), 2), (dict(size=8), 2), (dict(reserved=1), 2),
             (dict(page=24), 3), (dict(page=2), 3), (dict(page=8192), 3), (dict(N=8193), 3), (dict(page=4096, W=(1 << 16) + 1), 3),
             (dict(P=(1 << 28) + 1), 3),
             (dict(k=None), 1), (dict(v=None), 1), (dict(table=None), 1), (dict(lens=None), 1), (dict(refs=None), 1),
             (dict(k=A + 8), 5), (dict(v=A + 2), 5), (dict(table=A + 2), 5), (dict(lens=A + 1), 5), (dict(refs=A + 3), 5)]


@pytest.mark.parametrize("kw,status", BAD_CACHE)
def test_bad_caches(kw, status):
    got = _calls(_desc(), _cache(**kw))
    assert set(got.values()) == {status}, got
    assert bx.beagle_xattn_paged_workspace_bytes(_desc(), _cache(**kw), 0) == 0
    into = bx.beagle_xattn_paged_compact(_desc(), _far_cache(), _cache(**kw), None, A, stream=0, workspace_bytes=WS, check=False)
    assert into == status


def test_workspaces_pointers_and_alignment():
    d, c = _desc(), _cache()
    assert set(_calls(d, c, ws=None).values()) == {1}
    assert set(_calls(d, c, ws=A + 16).values()) == {5}
    assert set(_calls(d, c, nbytes=0).values()) == {4}
    for i, call in enumerate(("attend", "append", "fork", "compact", "draft", "kv_append")):
        need = bx.beagle_xattn_paged_workspace_bytes(d, c, i)
        assert need > 0 and _calls(d, c, nbytes=need - 1)[call] == 4
    assert bx.beagle_xattn_paged_workspace_bytes(d, c, 6) == 0 and bx.beagle_xattn_paged_workspace_bytes(d, c, -1) == 0
    kw = dict(stream=0, workspace_bytes=WS, check=False)
    for i in (0, 7, 8):                      # q, o, lse
        args = [A, A, A, A, 1, 0, 0, A, A]
        args[i] = None
        assert bx.beagle_xattn_paged_attend(d, c, *args, A, **kw) == 1
        args[i] = A + 8
        assert bx.beagle_xattn_paged_attend(d, c, *args, A, **kw) == 5
    for i in (1, 2, 3):                      # slots, n_true, the tree
        args = [A, A, A, A, 1, 0, 0, A, A]
        args[i] = A + 2
        assert bx.beagle_xattn_paged_attend(d, c, *args, A, **kw) == 5
    assert bx.beagle_xattn_paged_attend(d, c, A, A, A, None, 1, 0, 0, A, A, A, **kw) == 1
    for bad in ((-1, 0, 0), (0, -1, 0), (0, (1 << 28) + 1, 0), (0, 0, -1), (0, 0, (1 << 28) + 1)):
        assert bx.beagle_xattn_paged_attend(d, c, A, A, A, A, *bad, A, A, A, **kw) == 2
        assert bx.beagle_xattn_draft_step_paged(d, c, A, A, A, A, A, A, *bad, A, A, A, **kw) == 2
    for i in range(6):
        args = [A] * 6
        args[i] = A + 2
        assert bx.beagle_xattn_paged_append(d, c, *args, A, **kw) == 5
    for i in (3, 4):
        args = [A] * 6
        args[i] = None
        assert bx.beagle_xattn_paged_append(d, c, *args, A, **kw) == 1
    assert bx.beagle_xattn_paged_fork(d, c, None, A, A, A, **kw) == 1 and bx.beagle_xattn_paged_fork(d, c, A, None, A, A, **kw) == 1
    assert bx.beagle_xattn_paged_fork(d, c, A, A, A + 1, A, **kw) == 5
    for i in range(3):
        args = [A] * 3
        args[i] = None
        assert bx.beagle_xattn_kv_append_paged(d, c, *args, A, A, A, A, A, **kw) == 1
        assert bx.beagle_xattn_draft_step_paged(d, c, *args, A, A, A, 1, 0, 0, A, A, A, **kw) == 1
    # states: the products' limits
    assert bx.beagle_xattn_draft_step_paged(_desc(hidden=200), c, *[A] * 6, 1, 0, 0, A, A, A, **kw) == 3
    assert bx.beagle_xattn_kv_append_paged(_desc(hidden=0), c, *[A] * 7, A, **kw) == 2
    # null structures
    import ctypes as C
    L = bx.lib()
    assert L.beagle_xattn_paged_fork(None, C.byref(c), A, A, A, A, WS, 0) == 1
    assert L.beagle_xattn_paged_fork(C.byref(d), None, A, A, A, A, WS, 0) == 1
    assert L.beagle_xattn_paged_compact(C.byref(d), C.byref(c), None, A, A, WS, 0) == 1


def test_pools_that_a_compaction_cannot_join():
    d, c, kw = _desc(), _far_cache(), dict(stream=0, workspace_bytes=WS, check=False)
    for other in (_cache(page=32), _cache(N=5), _far_cache(), _cache(refs=(1 << 34) + 16), _cache(table=(1 << 30) + 4)):
        assert bx.beagle_xattn_paged_compact(d, c, other, None, A, **kw) == 2
    assert bx.beagle_xattn_paged_compact(d, c, _cache(), A + 2, A, **kw) == 5


def test_the_python_layer_refuses_what_it_can_see():
    i32, bf = torch.int32, torch.bfloat16
    k, table, lens, refs = torch.zeros(6, 16, 2, 128, dtype=bf), torch.zeros(4, 8, dtype=i32), torch.zeros(4, dtype=i32), torch.zeros(6, dtype=i32)
    ok = bx.make_paged_cache(k, k.clone(), table, lens, refs)
    assert (ok.n_pages, ok.page_rows, ok.n_slots, ok.slot_pages) == (6, 16, 4, 8)
    for bad in ((k, k[:5], table, lens, refs), (k, k.float(), table, lens, refs), (k[0], k[0], table, lens, refs), (k, k, table, lens[:3], refs),
                (k, k, table, lens, refs[:5]), (k, k, table.long(), lens, refs), (k, k, table, lens.float(), refs), (k, k, table[:, ::2], lens, refs),
                (k[:, :, :, :64], k[:, :, :, :64], table, lens, refs)):
        with pytest.raises(ValueError):
            bx.make_paged_cache(*bad)
    d = _desc()
    q, lse = torch.zeros(2, 3, 4, 128, dtype=bf), torch.zeros(2, 4, 3)
    args = dict(q=q, slots=lens[:2], n_true=None, tree_mask=None, mask_words=0, window=0, sinks=0, o=q, lse=lse, workspace=None)
    for bad in (dict(q=q.float()), dict(q=q[:1]), dict(slots=lens), dict(slots=lens[:2].long()), dict(lse=lse.double()), dict(lse=lse[:1]),
                dict(tree_mask=table, mask_words=1), dict(q=q.transpose(1, 2)), {}):          # ({}: on the CPU)
        with pytest.raises(ValueError):
            bx.beagle_xattn_paged_attend(d, ok, **dict(args, **bad))
    with pytest.raises(ValueError):                        # rows of another shape than the descriptor's
        bx.beagle_xattn_paged_fork(_desc(G=4), ok, A, A, None, A, stream=0, workspace_bytes=WS)
