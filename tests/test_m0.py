"""Requests into LDS that are written out set m0, and say so to the compiler, which keeps the address of its own ones there: read from the
compiled form of its request, one that is written out, and its request again."""
import os
import re
import subprocess

import pytest

from paper_2505_24544_amd import build

SOURCE = """
#include "paged_attend.h"
#include "attn_tiles.h"
namespace beagle {
__global__ void between(const char* p, uint32_t other) {
  __shared__ __attribute__((aligned(1024))) char rows[4096];
  typedef const __attribute__((address_space(1))) uint32_t* from_t;
  typedef __attribute__((address_space(3))) uint32_t* into_t;
  __builtin_amdgcn_global_load_lds((from_t)(p + threadIdx.x * 16), (into_t)rows, 16, 0, 0);
  load_to_lds((addr_t)p + 4096 + threadIdx.x * 16, other);
  __builtin_amdgcn_global_load_lds((from_t)(p + 8192 + threadIdx.x * 16), (into_t)rows, 16, 0, 0);
}
}
"""


def test_m0_is_set_again_behind_a_request_that_is_written_out(tmp_path):
    if not os.path.exists(build.HIPCC):
        pytest.skip("no hipcc")
    (tmp_path / "between.hip").write_text(SOURCE)
    out = tmp_path / "between.txt"
    r = subprocess.run([build.HIPCC, *build.FLAGS, "--cuda-device-only", "-S", "-I", build.CSRC, str(tmp_path / "between.hip"), "-o", str(out)],
                       capture_output=True, text=True)
    assert r.returncode == 0, r.stderr
    code = [ln.strip() for ln in out.read_text().splitlines()]
    code = code[next(n for n, ln in enumerate(code) if re.match(r"_ZN6beagle7between\S*:", ln)):]
    ops = ["set" if re.match(r"s_\w+ m0,", ln) else "load" for ln in code if re.match(r"s_\w+ m0,|global_load_lds", ln)]
    assert ops == ["set", "load"] * 3, ops
