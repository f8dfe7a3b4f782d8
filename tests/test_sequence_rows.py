"""CPU-only: which rows the attention's kernels may address from a chunk's first token with 32 bits (csrc/seq_geom.h, compiled for the host)."""
import os
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2311_09445_amd", "csrc")
CHUNK = 32      # tokens: the last one's offset is 31 strides

PROGRAM = r"""
#include "seq_geom.h"
#include <cstdio>
#include <cstdlib>
int main(int, char** argv) {
  const unsigned long heads = strtoul(argv[2], nullptr, 10), width = strtoul(argv[3], nullptr, 10);
  per::SeqRows r;
  if (argv[1][0] == 'p') r = per::packed(nullptr, 64, heads, width, 1);
  else r = per::rows(per_seq_rows{nullptr, 0, (int64_t)(heads * width), (int64_t)width}, argv[1][0] == 'b' ? PER_SEQ_BF16 : PER_SEQ_F32, 1);
  printf("%lld %u %u\n", (long long)r.token, r.wide, r.near);
}
"""


@pytest.fixture(scope="module")
def program(tmp_path_factory):
    at = tmp_path_factory.mktemp("rows")
    (at / "rows.cpp").write_text(PROGRAM)
    exe = at / "rows"
    subprocess.check_call(["g++", "-std=c++17", "-D__HIP_PLATFORM_AMD__=1", "-isystem", "/opt/rocm/include", "-I", CSRC, str(at / "rows.cpp"), "-o", str(exe)])
    return str(exe)


@pytest.mark.parametrize("kind", ["packed", "b", "f"])
@pytest.mark.parametrize("heads,width", [(1, 4), (8, 64), (1, 128), (131071, 128), (131072, 128), (1 << 19, 128), (1 << 21, 128), ((1 << 22) - 1, 4), (1 << 20, 12)])
def test_wide_rows_are_near(program, kind, heads, width):
    """Wide rows go the way that forms 31 strides, in bytes of up to four an element, in 32 bits."""
    token, wide, near = map(int, subprocess.check_output([program, kind, str(heads), str(width)], text=True).split())
    assert token == heads * width
    if wide or near:
        assert (CHUNK - 1) * token * 4 + width * 4 < 1 << 32
    if heads * width < 1 << 24 and (heads * width) % 8 == 0 and width % 8 == 0:
        assert wide and near
