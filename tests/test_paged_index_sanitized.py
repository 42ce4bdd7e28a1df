"""The paged cache's index code (csrc/paged_index.h) compiled for the HOST with AddressSanitizer and
UndefinedBehaviorSanitizer: which rows a window shows, which blocks are walked, how workers share them, and what hostile slot
numbers, lengths and page numbers turn into.  CPU only."""
import os
import random
import shutil
import subprocess

import pytest

HERE = os.path.dirname(os.path.abspath(__file__))
INT32_MAX = 2 ** 31 - 1


@pytest.fixture(scope="module")
def driver(tmp_path_factory):
    cxx = shutil.which("g++") or shutil.which("c++")
    if cxx is None:
        pytest.skip("no host C++ compiler")
    exe = str(tmp_path_factory.mktemp("san") / "paged_index_driver")
    r = subprocess.run([cxx, "-std=c++17", "-O1", "-g", "-fsanitize=address,undefined", "-fno-sanitize-recover=all",
                        os.path.join(HERE, "paged_index_driver.cpp"), "-o", exe], capture_output=True, text=True)
    assert r.returncode == 0, r.stderr

    def run(lines):
        env = dict(os.environ)
        env.pop("LD_PRELOAD", None)       # the sanitizer runtime must come first in the driver's own process
        r = subprocess.run([exe], input="\n".join(lines) + "\n", capture_output=True, text=True, env=env, timeout=120)
        assert r.returncode == 0, "sanitizer or driver failure:\n" + r.stderr[-4000:]
        return [[int(v) for v in ln.split()] for ln in r.stdout.splitlines()]
    return run


def test_rows_that_a_window_shows_and_the_blocks_that_hold_them(driver):
    rng = random.Random(5)
    cases = [(n, nt, w, s) for n in (0, 1, 31, 32, 33, 200) for nt in (0, 1, 32, n) for w in (0, 1, 31, 32, 64, 1000) for s in (0, 1, 4, 33)]
    cases += [(rng.randrange(1500), rng.randrange(-3, 1600), rng.choice((0, rng.randrange(1, 700))), rng.randrange(300)) for _ in range(300)]
    for (n, nt, w, s), got in zip(cases, driver(["rows %d %d %d %d" % c for c in cases])):
        nt = min(max(nt, 0), n)
        seen = [j < n and (j >= nt or w == 0 or j < s or j >= nt - w) for j in range(n + 40)]
        assert 1 <= got[0] <= max(1, -(-n // 32))
        for j, v in enumerate(got[1:]):
            held, sees, whole = v // 4, bool(v & 2), bool(v & 1)
            assert sees == seen[j] and held <= 1, (n, nt, w, s, j)
            assert held == 1 or not seen[j], (n, nt, w, s, j)         # a row that is seen is walked, once
            first = j // 32 * 32
            full = first + 32 <= nt and all(seen[first: first + 32])
            assert not whole or full, (n, nt, w, s, j)                # (a block of sinks and window rows together may be missed)
    big = [(2 ** 28, 2 ** 28, 0, 0), (2 ** 28, INT32_MAX, 2 ** 28, 2 ** 28), (2 ** 28, 2 ** 28, 1, 0)]
    assert [g[0] for g in driver(["rows %d %d %d %d" % c for c in big])] == [2 ** 23, 2 ** 23, 1]


def test_workers_share_all_blocks_evenly(driver):
    rng = random.Random(6)
    cases = [(rng.choice((1, 4, 25, 64, 512)), rng.choice((2, 3)), [max(1, int(2 ** rng.uniform(0, 9)) * rng.choice((0, 1, 1)))
                                                                  for _ in range(rng.choice((1, 2, 7, 64, 65, 150)))]) for _ in range(200)]
    cases.append((512, 3, [2 ** 23] * 300))
    for (target, longest, blocks), got in zip(cases, driver(["workers %d %d %s" % (t, k, " ".join(map(str, n))) for t, k, n in cases])):
        n, run, ends = got[0], got[1], got[len(got) - 2 * len(blocks):]
        shares = [got[i: i + 4] for i in range(2, len(got) - len(ends), 4)]
        fits = [r for r in (4, 8) if r <= 1 << longest and sum(-(-size // r) for size in blocks) <= target
                and (r == 4 or (r - 5) * target <= sum(blocks))]
        assert run == (fits[0] if fits else 0)
        assert 1 <= n <= target and n == (sum(-(-size // run) for size in blocks) if run else min(target, -(-sum(blocks) // 4)))
        parts = {}
        for w, e, a, b in shares:
            parts.setdefault(e, []).append((w, a, b))
        even = sum(blocks) / n
        work = [0] * n
        for e, size in enumerate(blocks):
            at = 0
            for w, a, b in parts[e]:                    # in order, without a gap, from the first worker to the last
                assert a == at
                at, work[w] = b, work[w] + b - a
            assert at == size
            if size <= (run or 4):
                assert len(parts[e]) == 1 and parts[e][0][0] == ends[2 * e]
            else:
                assert [p[0] for p in parts[e]] == list(range(ends[2 * e], ends[2 * e + 1] + 1))
        assert max(work) <= (run or even + 1 + 4)
        if run:                              # a worker for every run: nobody has two entries
            assert sorted(v for v, e, a, b in shares) == list(range(n))
        for w in range(n):                              # at most one entry gone on with and one begun in part: two places for sums
            part = [(a, b, e) for v, e, a, b in shares if v == w and b - a < blocks[e]]
            assert sum(a > 0 for a, b, e in part) <= 1 and sum(a == 0 for a, b, e in part) <= 1


def test_hostile_numbers(driver):
    t = [5, -1, INT32_MAX, -2 ** 31, 9, 10]
    lines = ["page 10 2 %d 1 %s" % (row, " ".join(map(str, t))) for row in range(24)] + ["page 10 2 %d 0 %s" % (10 ** 6, " ".join(map(str, t)))]
    assert [g[0] for g in driver(lines)] == [5] * 4 + [-1] * 12 + [9] * 4 + [-1] * 4 + [-1]
    got = driver(["slot %d 8 %d 4 3" % (s, n) for s in (-1, 0, 7, 8, INT32_MAX, -2 ** 31) for n in (-5, 0, 9, 32, INT32_MAX)])
    for (s, n), g in zip([(s, n) for s in (-1, 0, 7, 8, INT32_MAX, -2 ** 31) for n in (-5, 0, 9, 32, INT32_MAX)], got):
        n = min(max(n, 0), 32)
        assert g == [s if 0 <= s < 8 else -1, n, -(-n // 8)]
