"""The host side of the paged-cache entry points (csrc/api_paged.hip: descriptor and cache checks, workspace layouts) rebuilt with
UndefinedBehaviorSanitizer in trap mode on the host pass and swept with fields across the whole int32 range, one at a time and
in large combinations; a trap kills the sweeping process.  Tensor arguments are NULL, so that no call gets to a launch: CPU only."""
import os
import subprocess
import sys
import textwrap

import pytest

HERE = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(HERE)


@pytest.fixture(scope="module")
def sanitized_lib(tmp_path_factory):
    from paper_2505_24544_amd import build as bld
    bdir = os.path.join(bld.CSRC, "_build")
    others = [s for s in bld.sources() if s != "api_paged.hip"]
    if not all(os.path.exists(os.path.join(bdir, s.replace(".hip", ".o"))) for s in others):
        bld.build(verbose=False)
    out = tmp_path_factory.mktemp("ubsan_paged")
    obj, lib = str(out / "api_paged.o"), str(out / "libbeagle_xattn_ubsan.so")
    flags = [f for f in bld.FLAGS if f != "-O3"] + ["-O1", "-g"]
    san = ["-Xarch_host", "-fsanitize=undefined", "-Xarch_host", "-fsanitize-trap=undefined"]
    r = subprocess.run([bld.HIPCC, *flags, *san, "-c", os.path.join(bld.CSRC, "api_paged.hip"), "-o", obj], capture_output=True, text=True)
    assert r.returncode == 0, r.stderr[-3000:]
    objs = [os.path.join(bdir, s.replace(".hip", ".o")) for s in others] + [obj]
    r = subprocess.run([bld.HIPCC, "--offload-arch=gfx950", "-shared", "-fPIC", "-fno-gpu-rdc", *objs, "-o", lib], capture_output=True, text=True)
    assert r.returncode == 0, r.stderr[-3000:]
    return lib


SWEEP = textwrap.dedent('''
    import itertools, sys, ctypes as C
    sys.path.insert(0, sys.argv[2])
    import paper_2505_24544_amd.binding as bx
    bx.LIB_PATH = sys.argv[1]
    L = bx.lib()
    EDGE = (-2**31, -1, 0, 1, 3, 4, 8, 64, 128, 4096, 8192, 8193, 2**20 + 1, 2**24, 2**28, 2**30 + 1, 2**31 - 1)
    n = 0

    def poke(d, c):
        global n
        n += 1
        for w in range(-1, 8):
            L.beagle_xattn_paged_workspace_bytes(C.byref(d), C.byref(c), w)
        kw = dict(check=False, workspace_bytes=1 << 50, stream=0)
        z = None
        bx.beagle_xattn_paged_attend(d, c, z, z, z, z, 0, 0, 0, z, z, z, **kw)
        bx.beagle_xattn_paged_append(d, c, z, z, z, z, z, z, z, **kw)
        bx.beagle_xattn_paged_fork(d, c, z, z, z, z, **kw)
        bx.beagle_xattn_paged_compact(d, c, c, z, z, **kw)
        bx.beagle_xattn_paged_compact(d, c, cache(at=1 << 45), z, z, **kw)
        bx.beagle_xattn_draft_step_paged(d, c, z, z, z, z, z, z, 0, 0, 0, z, z, z, **kw)
        bx.beagle_xattn_kv_append_paged(d, c, z, z, z, z, z, z, z, z, **kw)

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
    for field in ("P", "page", "N", "W"):
        for v in EDGE:
            poke(desc(), cache(**{field: v}))
    big = (1, 4096, 8192, 2**24, 2**28, 2**31 - 1)
    for a, b, c in itertools.product(big, big, big):
        poke(desc(batch=a, seq_q=b, n_q_heads=c, n_kv_heads=c), cache())
        poke(desc(seq_q=a, n_q_heads=b, n_kv_heads=1, hidden=c if c % 64 == 0 else 256), cache())
        poke(desc(batch=a), cache(P=b, W=c, page=4))
        poke(desc(), cache(P=a, page=4096, N=b if b < 8193 else 8192, W=c))
    print("swept:", n)
''')


def test_sweep_under_ubsan(sanitized_lib, tmp_path):
    script = tmp_path / "sweep.py"
    script.write_text(SWEEP)
    r = subprocess.run([sys.executable, str(script), sanitized_lib, ROOT], capture_output=True, text=True, timeout=600)
    assert r.returncode == 0, "the sweep died (a trap is an undefined-behaviour report):\n%s\n%s" % (r.stdout[-2000:], r.stderr[-4000:])
    assert "swept:" in r.stdout
