"""The planning workgroups of the paged cache as they are compiled: where one wave's stores and count changes are read by another, every
wave has waited for its own before the barrier (a barrier does not wait for memory), and the vector cache is emptied behind it; and
the one-launch fork has all that it reads before any of its waves writes.
Read from the built library's own code objects."""
import os
import re
import shutil

import pytest

from paper_2505_24544_amd import build
from test_mfma_in_place import LLVM, _out, pytestmark  # noqa: F401

HANDOVERS = {"paged_append_plan_kernel": 2, "paged_compact_kernel": 1}
KERNELS = (*HANDOVERS, "paged_fork_kernel")
MEMORY = re.compile(r"(global|flat|buffer|scratch)_(load|store|atomic)")


@pytest.fixture(scope="module")
def kernels(tmp_path_factory):
    """{kernel: its instructions' text in order}"""
    if not os.path.exists(build.OUT):
        build.build(verbose=False)
    tmp = str(tmp_path_factory.mktemp("co"))
    shutil.copy(build.OUT, os.path.join(tmp, "lib.so"))
    _out(LLVM + "llvm-objdump", "--offloading", "lib.so", cwd=tmp)
    found = {}
    for f in sorted(os.listdir(tmp)):
        if not f.endswith("gfx950"):
            continue
        if not any(k in _out(LLVM + "llvm-readelf", "--notes", f, cwd=tmp) for k in KERNELS):
            continue
        code = None
        for line in _out(LLVM + "llvm-objdump", "-d", "--mcpu=gfx950", f, cwd=tmp).splitlines():
            m = re.match(r"[0-9a-f]+ <(\S+)>:", line)
            if m:
                name = next((k for k in KERNELS if k in m[1]), None)
                code = found.setdefault(name, []) if name else None
            elif code is not None and (m := re.match(r"\s+(\S.*?)\s*//", line)):
                code.append(m[1])
    return found


@pytest.mark.parametrize("name", HANDOVERS)
def test_memory_is_waited_for_before_the_barrier(kernels, name):
    code = kernels[name]
    at = [n for n, i in enumerate(code) if i.startswith("buffer_inv")]
    assert len(at) == HANDOVERS[name]
    for n in at:
        barrier = max(k for k in range(n) if code[k].startswith("s_barrier"))
        assert not any(MEMORY.match(i) for i in code[barrier:n])
        waited = max((k for k in range(barrier) if re.match(r"s_waitcnt\b.*vmcnt\(0\)", code[k])), default=-1)
        between = code[waited + 1:barrier]
        assert waited >= 0 and not any(MEMORY.match(i) or i.startswith(("s_cbranch", "s_branch", "s_barrier")) for i in between), code[barrier - 12:n + 1]


def test_a_fork_has_read_everything_before_it_writes(kernels):
    code = kernels["paged_fork_kernel"]
    first = min(n for n, i in enumerate(code) if re.match(r"global_(store|atomic)", i))
    last = max(n for n in range(first) if re.match(r"global_load", code[n]))
    assert not any(re.match(r"global_load", i) for i in code[first:])
    waited = [n for n in range(last, first) if re.match(r"s_waitcnt\b.*vmcnt\(0\)", code[n])]
    assert waited and any(i.startswith("s_barrier") for i in code[waited[0]:first])
