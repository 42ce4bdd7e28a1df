"""The picking of pages (CPU): its code in a host build, where a workgroup's waves run in any order between two barriers, against a
plain ranking.  An order that changes the pages, waves that meet at different barriers and writes outside the list all show."""
import os
import random
import shutil
import struct
import subprocess

import pytest

HERE = os.path.dirname(os.path.abspath(__file__))
ORDERS = (-1, -2, 1)                       # the first wave first, the last one, any


@pytest.fixture(scope="module")
def pick(tmp_path_factory):
    cxx = shutil.which("g++") or shutil.which("c++")
    if cxx is None:
        pytest.skip("no host C++ compiler")
    exe = str(tmp_path_factory.mktemp("pick") / "paged_pick_order_driver")
    r = subprocess.run([cxx, "-std=c++17", "-O1", "-g", "-fsanitize=undefined", "-fno-sanitize-recover=all", "-Wno-unknown-pragmas",
                        os.path.join(HERE, "paged_pick_order_driver.cpp"), "-o", exe], capture_output=True, text=True)
    assert r.returncode == 0, r.stderr

    def run(n_select, off, scores, truth, *, lead=3, rows=2, memory=0, order=-1):
        text = "%d %d %d %d %d %d %r\n" % (len(scores), n_select, lead, rows, memory, order, off)
        text += "\n".join("%r %r" % p for p in zip(scores, truth))
        env = dict(os.environ)
        env.pop("LD_PRELOAD", None)
        r = subprocess.run([exe], input=text + "\n", capture_output=True, text=True, env=env, timeout=120)
        assert r.returncode == 0, r.stderr[-4000:]
        assert not r.stdout.startswith("wrong"), r.stdout
        return [int(v) for v in r.stdout.split()]
    return run


def f32(x):
    return struct.unpack("f", struct.pack("f", x))[0]


def ranked(truth, n_select, lead=3):
    return sorted(i + lead for i in sorted(range(len(truth)), key=lambda i: (-truth[i], i))[:n_select])


def near(rng, truth, off):
    """Scores that are off by less than `off`."""
    return [f32(t + 0.9 * off * rng.uniform(-1, 1)) for t in truth]


def check(pick, truth, scores, n_select, off, **kw):
    for order in ORDERS:
        assert pick(n_select, off, scores, truth, order=order, **kw) == ranked(truth, n_select), (n_select, off, kw, order)


@pytest.mark.parametrize("memory", [0, 1])
@pytest.mark.parametrize("n,n_select", [(2, 1), (65, 64), (513, 40), (3001, 700)])
def test_the_largest_scores(pick, memory, n, n_select):
    rng = random.Random(n)
    truth = [f32(rng.uniform(1, 9)) for _ in range(n)]
    check(pick, truth, near(rng, truth, 0.01), n_select, 0.01, memory=memory)
    check(pick, truth, truth, n_select, 1e-6, memory=memory, rows=1)


@pytest.mark.parametrize("memory", [0, 1])
@pytest.mark.parametrize("n,n_select,doubt", [(600, 100, 3), (2000, 333, 40), (9000, 700, 150), (700, 690, 8)])
def test_scores_below_zero(pick, memory, n, n_select, doubt):
    """The last page picked has a score below zero, and some before and behind it are in doubt."""
    rng = random.Random(n + doubt)
    truth = [f32(-100.0 + rng.uniform(0, 90)) for _ in range(n)]
    order = sorted(range(n), key=lambda i: -truth[i])
    for k in order[max(n_select - doubt // 2, 0): n_select + doubt - doubt // 2]:      # closer to each other than can be told
        truth[k] = f32(truth[order[n_select]] + rng.uniform(-1e-3, 1e-3))
    for off in (2e-3, 1e-6):
        check(pick, truth, near(rng, truth, off), n_select, off, memory=memory)


@pytest.mark.parametrize("memory", [0, 1])
@pytest.mark.parametrize("n,n_select,alike", [(300, 50, 241), (1000, 400, 1000), (1200, 700, 600), (9000, 300, 2500)])
def test_many_in_doubt(pick, memory, n, n_select, alike):
    """More pages in doubt than a list holds: equal scores, an error without a bound, scores below zero and of both signs."""
    rng = random.Random(n + alike)
    for low, high in ((1, 9), (-9, -1), (-5, 5)):
        truth = [f32(rng.uniform(low, high)) for _ in range(n)]
        check(pick, truth, near(rng, truth, 0.5), n_select, float("inf"), memory=memory, rows=1)
        at = sorted(truth, reverse=True)[n_select - 1]
        for i in rng.sample(range(n), alike):
            truth[i] = at
        check(pick, truth, near(rng, truth, 1e-4), n_select, 1e-4, memory=memory, rows=1)


@pytest.mark.parametrize("memory", [0, 1])
def test_no_scores_at_all(pick, memory):
    none = [float("-inf")] * 700
    check(pick, none, none, 300, 1e-3, memory=memory)
    check(pick, none, none, 300, float("inf"), memory=memory)
    some = none[:]
    some[5], some[650], some[651] = -3.0, -2.0, float("inf")
    check(pick, some, some, 2, float("inf"), memory=memory)
    some[651] = -4.0
    check(pick, some, some, 300, 1e-3, memory=memory)
