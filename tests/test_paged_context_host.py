"""Host side of the calls for shared and long contexts (CPU only): what is refused, with which status, before anything is enqueued;
their checks and layouts under UndefinedBehaviorSanitizer; and their index code under sanitizers against plain loops."""
import os
import random
import shutil
import subprocess
import sys
import textwrap

import pytest
import torch

from paper_2505_24544_amd import binding as bx
from test_paged_abi import BAD_CACHE, BAD_DESC, A, WS, _cache, _desc
from test_paged_host_sanitized import ROOT, sanitized_lib  # noqa: F401

HERE = os.path.dirname(os.path.abspath(__file__))
KW = dict(stream=0, check=False)


def _calls(desc, cache, ws=A, nbytes=WS):
    kw = dict(KW, workspace_bytes=nbytes)
    return {
        8: bx.beagle_xattn_paged_attend_shared(desc, cache, A, A, A, A, 2, A, A, 1, A, A, ws, **kw),
        9: bx.beagle_xattn_paged_select(desc, cache, A, A, A, A, 0, 0, 3, A, ws, **kw),
        10: bx.beagle_xattn_paged_attend_blocks(desc, cache, A, A, A, A, 1, 0, 0, A, 3, A, A, ws, **kw),
        11: bx.beagle_xattn_draft_step_paged_shared(desc, cache, A, A, A, A, A, A, 2, A, A, 1, A, A, ws, **kw),
        12: bx.beagle_xattn_draft_step_paged_blocks(desc, cache, A, A, A, A, A, A, 1, A, 0, 0, 3, A, A, A, ws, **kw),
    }


@pytest.mark.parametrize("kw,status", BAD_DESC)
def test_bad_descriptors(kw, status):
    got = _calls(_desc(**kw), _cache())
    assert set(got.values()) == {status}, got
    assert bx.beagle_xattn_paged_bounds(_desc(**kw), _cache(), A, A, A, **KW) == status
    for which in got:
        assert bx.beagle_xattn_paged_workspace_bytes(_desc(**kw), _cache(), which) == 0


@pytest.mark.parametrize("kw,status", BAD_CACHE)
def test_bad_caches(kw, status):
    got = _calls(_desc(), _cache(**kw))
    assert set(got.values()) == {status}, got
    assert bx.beagle_xattn_paged_bounds(_desc(), _cache(**kw), A, A, A, **KW) == status


def test_workspaces():
    d, c = _desc(), _cache()
    assert set(_calls(d, c, ws=None).values()) == {1}
    assert set(_calls(d, c, ws=A + 16).values()) == {5}
    assert set(_calls(d, c, nbytes=0).values()) == {4}
    for which in _calls(d, c, nbytes=0):
        need = bx.beagle_xattn_paged_workspace_bytes(d, c, which)
        assert need > 0 and need % 256 == 0 and _calls(d, c, nbytes=need - 1)[which] == 4
    assert [bx.beagle_xattn_paged_workspace_bytes(d, c, w) for w in (6, 7, 13)] == [0, 0, 0]


def _each(call, args, places, values, status):
    for i in places:
        for v in values:
            bad = list(args)
            bad[i] = v
            assert call(*bad) == status, (call, i, v)


def test_pointers_and_sizes():
    d, c, kw = _desc(), _cache(), dict(KW, workspace_bytes=WS)
    attend = lambda *a: bx.beagle_xattn_paged_attend_shared(d, c, *a, A, **kw)                        # noqa: E731
    ok = (A, A, A, A, 2, A, A, 1, A, A)
    _each(attend, ok, (0, 8, 9), (None,), 1)
    _each(attend, ok, (0, 8, 9), (A + 8,), 5)
    _each(attend, ok, (2, 3), (None,), 1)
    _each(attend, ok, (1, 2, 3, 5, 6), (A + 2,), 5)
    _each(attend, ok, (4,), (0, -1, 3), 2)                    # B = 2
    _each(attend, ok, (7,), (-1,), 2)
    assert attend(A, A, A, A, 2, A, None, 1, A, A) == 1
    bounds = lambda *a: bx.beagle_xattn_paged_bounds(d, c, *a, **KW)                                  # noqa: E731
    _each(bounds, (A, A, A), (2,), (None,), 1)
    _each(bounds, (A, A, A), (2,), (A + 8,), 5)
    _each(bounds, (A, A, A), (0, 1), (A + 1,), 5)
    select = lambda *a: bx.beagle_xattn_paged_select(d, c, *a, A, **kw)                               # noqa: E731
    ok = (A, A, A, A, 0, 0, 3, A)
    _each(select, ok, (0, 3, 7), (None,), 1)
    _each(select, ok, (0, 3), (A + 8,), 5)
    _each(select, ok, (1, 2, 7), (A + 2,), 5)
    _each(select, ok, (4, 5), (-1, (1 << 28) + 1), 2)
    _each(select, ok, (6,), (0, -1, (1 << 26) + 1), 2)
    blocks = lambda *a: bx.beagle_xattn_paged_attend_blocks(d, c, *a, A, **kw)                        # noqa: E731
    ok = (A, A, A, A, 1, 0, 0, A, 3, A, A)
    _each(blocks, ok, (0, 7, 9, 10), (None,), 1)
    _each(blocks, ok, (0, 9, 10), (A + 8,), 5)
    _each(blocks, ok, (1, 2, 3, 7), (A + 2,), 5)
    _each(blocks, ok, (5, 6), (-1, (1 << 28) + 1), 2)
    _each(blocks, ok, (8,), (0, -1, (1 << 26) + 1), 2)
    shared = lambda *a: bx.beagle_xattn_draft_step_paged_shared(d, c, *a, A, **kw)                    # noqa: E731
    ok = (A, A, A, A, A, A, 2, A, A, 1, A, A)
    _each(shared, ok, (0, 1, 2, 4, 5, 10, 11), (None,), 1)
    _each(shared, ok, (0, 1, 2, 10, 11), (A + 8,), 5)
    _each(shared, ok, (3, 4, 5, 7, 8), (A + 2,), 5)
    _each(shared, ok, (6,), (0, 3), 2)
    step = lambda *a: bx.beagle_xattn_draft_step_paged_blocks(d, c, *a, A, **kw)                      # noqa: E731
    ok = (A, A, A, A, A, A, 1, A, 0, 0, 3, A, A, A)
    _each(step, ok, (0, 1, 2, 7, 11, 12, 13), (None,), 1)
    _each(step, ok, (0, 1, 2, 7, 12, 13), (A + 8,), 5)
    _each(step, ok, (3, 4, 5, 11), (A + 2,), 5)
    _each(step, ok, (8, 9), (-1, (1 << 28) + 1), 2)
    _each(step, ok, (10,), (0,), 2)


def test_query_rows_that_are_not_counted():
    many = _desc(B=8192, M=2048, H=64, G=1)                   # 2^30 query rows of the kv head
    got = _calls(many, _cache())
    assert got[8] == 3 and bx.beagle_xattn_paged_workspace_bytes(many, _cache(), 8) == 0
    assert bx.beagle_xattn_paged_workspace_bytes(many, _cache(), 9) > 0


def test_the_python_layer_refuses_what_it_can_see():
    i32, bf = torch.int32, torch.bfloat16
    k, table, lens, refs = torch.zeros(6, 16, 2, 128, dtype=bf), torch.zeros(4, 8, dtype=i32), torch.zeros(4, dtype=i32), torch.zeros(6, dtype=i32)
    c, d = bx.make_paged_cache(k, k.clone(), table, lens, refs), _desc()
    q, lse, two, three = torch.zeros(2, 3, 4, 128, dtype=bf), torch.zeros(2, 4, 3), torch.zeros(2, dtype=i32), torch.zeros(3, dtype=i32)
    bnd, pages = torch.zeros(6, 2, 2, 128, dtype=bf), torch.zeros(2, 2, 5, dtype=i32)
    shared = dict(q=q, slots=two, group_first=three, n_shared=two, n_groups=2, n_true=None, tree_mask=None, mask_words=0, o=q, lse=lse, workspace=None)
    for bad in (dict(group_first=two), dict(n_shared=three), dict(group_first=three.long()), dict(n_groups=1), dict(q=q.float()), dict(lse=lse[:1]), {}):
        with pytest.raises(ValueError):                       # ({}: on the CPU)
            bx.beagle_xattn_paged_attend_shared(d, c, **dict(shared, **bad))
    for bad in (dict(bounds=bnd.float()), dict(bounds=bnd[:5]), dict(first=three), {}):
        with pytest.raises(ValueError):
            bx.beagle_xattn_paged_bounds(d, c, **dict(dict(slots=two, first=two, bounds=bnd), **bad))
    select = dict(q=q, slots=two, n_true=two, bounds=bnd, window=0, sinks=0, n_select=5, pages=pages, workspace=None)
    for bad in (dict(pages=pages[:1]), dict(n_select=4), dict(pages=pages.long()), dict(bounds=bnd.transpose(1, 2)), {}):
        with pytest.raises(ValueError):
            bx.beagle_xattn_paged_select(d, c, **dict(select, **bad))
    blocks = dict(q=q, slots=two, n_true=None, tree_mask=None, mask_words=0, window=0, sinks=0, pages=pages, n_select=5, o=q, lse=lse, workspace=None)
    for bad in (dict(pages=pages[:, :1]), dict(n_select=6), dict(o=q[:1]), {}):
        with pytest.raises(ValueError):
            bx.beagle_xattn_paged_attend_blocks(d, c, **dict(blocks, **bad))


SWEEP = textwrap.dedent('''
    import itertools, sys, ctypes as C
    sys.path.insert(0, sys.argv[2])
    import paper_2505_24544_amd.binding as bx
    bx.LIB_PATH = sys.argv[1]
    L = bx.lib()
    EDGE = (-2**31, -1, 0, 1, 3, 4, 8, 64, 128, 4096, 8192, 8193, 2**20 + 1, 2**24, 2**26, 2**28, 2**30 + 1, 2**31 - 1)
    n = 0

    def poke(d, c, k=3):
        global n
        n += 1
        for w in range(8, 14):
            L.beagle_xattn_paged_workspace_bytes(C.byref(d), C.byref(c), w)
        kw = dict(check=False, workspace_bytes=1 << 60, stream=0)
        z, a = None, 4096
        # everything but the workspace is there: no call gets to a launch
        bx.beagle_xattn_paged_attend_shared(d, c, a, a, a, a, k, a, a, 1, a, a, z, **kw)
        bx.beagle_xattn_paged_bounds(d, c, a, a, z, check=False, stream=0)
        bx.beagle_xattn_paged_select(d, c, a, a, a, a, k, k, k, a, z, **kw)
        bx.beagle_xattn_paged_attend_blocks(d, c, a, a, a, a, 1, k, k, a, k, a, a, z, **kw)
        bx.beagle_xattn_draft_step_paged_shared(d, c, a, a, a, a, a, a, k, a, a, 1, a, a, z, **kw)
        bx.beagle_xattn_draft_step_paged_blocks(d, c, a, a, a, a, a, a, 1, a, k, k, k, a, a, a, z, **kw)

    def desc(**kw):
        return bx.make_desc(**dict(dict(batch=2, seq_q=3, seq_kv=64, hidden=256, n_q_heads=4, n_kv_heads=2, head_dim=128,
                                        io_dtype=bx.BEAGLE_BF16), **kw))

    def cache(P=10, page=16, N=4, W=8, at=4096):
        return bx.beagle_paged_cache(C.sizeof(bx.beagle_paged_cache), P, page, N, W, 0, *[at + 4096 * i for i in range(5)])

    for dtype in (bx.BEAGLE_BF16, bx.BEAGLE_F32):
        for flags in (0, bx.BEAGLE_FLAG_ROPE, 0xffffffff):
            for field in ("batch", "seq_q", "seq_kv", "hidden", "n_q_heads", "n_kv_heads", "head_dim"):
                for v in EDGE:
                    poke(desc(io_dtype=dtype, flags=flags, **{field: v}), cache())
    for v in EDGE:
        poke(desc(), cache(), v)
    for field in ("P", "page", "N", "W"):
        for v in EDGE:
            poke(desc(), cache(**{field: v}))
    big = (1, 4096, 8192, 2**24, 2**28, 2**31 - 1)
    for a, b, c in itertools.product(big, big, big):
        poke(desc(batch=a, seq_q=b, n_q_heads=c, n_kv_heads=c), cache())
        poke(desc(seq_q=a, n_q_heads=b, n_kv_heads=1, hidden=c if c % 64 == 0 else 256), cache())
        poke(desc(batch=a, seq_kv=c), cache(P=b, W=c, page=4))
        poke(desc(), cache(P=a, page=4096, N=b if b < 8193 else 8192, W=c))
    print("swept:", n)
''')


def test_sweep_under_ubsan(sanitized_lib, tmp_path):  # noqa: F811
    script = tmp_path / "sweep.py"
    script.write_text(SWEEP)
    r = subprocess.run([sys.executable, str(script), sanitized_lib, ROOT], capture_output=True, text=True, timeout=600)
    assert r.returncode == 0, "the sweep died (a trap is an undefined-behaviour report):\n%s\n%s" % (r.stdout[-2000:], r.stderr[-4000:])
    assert "swept:" in r.stdout


# ------------------------------------------------------------------ index code
@pytest.fixture(scope="module")
def driver(tmp_path_factory):
    cxx = shutil.which("g++") or shutil.which("c++")
    if cxx is None:
        pytest.skip("no host C++ compiler")
    exe = str(tmp_path_factory.mktemp("san") / "paged_pick_driver")
    r = subprocess.run([cxx, "-std=c++17", "-O1", "-g", "-fsanitize=address,undefined", "-fno-sanitize-recover=all",
                        os.path.join(HERE, "paged_pick_driver.cpp"), "-o", exe], capture_output=True, text=True)
    assert r.returncode == 0, r.stderr

    def run(lines):
        env = dict(os.environ)
        env.pop("LD_PRELOAD", None)       # the sanitizer runtime must come first in the driver's own process
        r = subprocess.run([exe], input="\n".join(lines) + "\n", capture_output=True, text=True, env=env, timeout=120)
        assert r.returncode == 0, "sanitizer or driver failure:\n" + r.stderr[-4000:]
        return [[int(v) for v in ln.split()] for ln in r.stdout.splitlines()]
    return run


def test_pages_seen_count_as_one_sequence(driver):
    rng = random.Random(1)
    cases = []
    for _ in range(600):
        shift = rng.choice((2, 3, 5))
        page = 1 << shift
        n = rng.choice((0, 1, page, rng.randrange(40 * page)))
        nt = rng.choice((n, n, rng.randrange(-3, n + 5)))
        window, sinks = rng.choice((0, rng.randrange(1, 20 * page))), rng.choice((0, 1, page, rng.randrange(10 * page)))
        list_ = sorted(rng.randrange(-2, 45) for _ in range(rng.randrange(1, 20)))
        if rng.random() < 0.5:
            rng.shuffle(list_)
        cases.append((n, nt, window, sinks, shift, list_, [rng.randrange(-1, 60) for _ in range(-(-n // page) or 1)]))
    out = driver(["pick %d %d %d %d %d %d 50 %s | %s" % (n, nt, w, s, len(l), sh, " ".join(map(str, l)), " ".join(map(str, t)))
                  for n, nt, w, s, sh, l, t in cases])
    for (n, nt, w, s, sh, l, table), got in zip(cases, out):
        page = 1 << sh
        nt = min(max(nt, 0), n)
        lead = -(-s // page)
        tail = max(lead, max(nt - w, 0) // page)
        count = min(tail - lead, len(l))
        assert got[:3] == [lead, count, tail - lead - count]
        hidden = (tail - lead - count) * page
        assert got[3:5] == [n - hidden, max(nt - hidden, 0)]
        pages = -(-n // page)
        want, before = [], -1
        for i in range(min(lead, pages)):
            want.append(table[i])
        for i in range(count):
            want.append(table[l[i]] if l[i] > before and lead <= l[i] < tail else -1)
            before = l[i]
        want += [table[i] for i in range(tail, pages)]
        assert got[5:] == [p if 0 <= p < 50 else -1 for p in want], (n, nt, w, s, l)
    big = 1 << 28
    got = driver(["pick %d %d %d %d %d 2 10 " % c for c in ((big, big, 0, 0, 1 << 26), (big, 2 ** 31 - 1, big, big, 5), (big, big, 1, big, 1),
                                                           (big, big, 0, 0, 1), (0, -(2 ** 31), big, 0, 1))])
    assert got == [[0, 1 << 26, 0, big, big], [1 << 26, 0, 0, big, big], [1 << 26, 0, 0, big, big], [0, 1, (1 << 26) - 1, 4, 4], [0, 0, 0, 0, 0]]


def test_own_rows(driver):
    rng = random.Random(2)
    cases = [(n, nt, f) for n in (0, 1, 31, 32, 33, 200) for nt in (-1, 0, 1, 32, n) for f in (-5, 0, 1, 31, 32, 64, n, 1000)]
    cases += [(rng.randrange(1500), rng.randrange(-3, 1600), rng.randrange(1600)) for _ in range(300)]
    for (n, nt, f), got in zip(cases, driver(["from %d %d %d" % c for c in cases])):
        nt = min(max(nt, 0), n)
        f = min(max(f, 0), nt)
        for j, v in enumerate(got[1:]):
            assert v % 2 == (f <= j < n), (n, nt, f, j)
            assert v // 2 <= 1 and (v // 2 == 1 or not v % 2), (n, nt, f, j)      # a row that is seen is walked, once
        assert got[0] == max(-(-n // 32) - f // 32, 0)
    assert [g[0] for g in driver(["from %d %d %d" % c for c in ((2 ** 28, 2 ** 28, 0), (2 ** 28, 2 ** 31 - 1, 2 ** 28), (2 ** 28, 5, 2 ** 31 - 1))])] == [
        2 ** 23, 0, 2 ** 23]
