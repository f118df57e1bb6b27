"""Launches of the cache's operators, on the CPU: a small host program against the library's own helpers."""
import os
import subprocess

import pytest

from paper_2512_17917_amd import build as B

PROBE = r"""
#include <cstdio>
#include "kvr_launch.h"
// g n -> workgroups a row, rows
int main() {
  char kind;
  while (std::scanf(" %c", &kind) == 1) {
    long long n;
    if (kind == 'g') {
      if (std::scanf("%lld", &n) != 1) return 1;
      const kvr::GridRows r = kvr::grid_rows(n);
      std::printf("%u %u\n", r.x, r.rows);
    }
  }
}
"""


@pytest.fixture(scope="module")
def ask(tmp_path_factory):
    d = tmp_path_factory.mktemp("launch")
    src, exe = str(d / "probe.hip"), str(d / "probe")
    open(src, "w").write(PROBE)
    subprocess.run([B._hipcc(), "--offload-host-only", "-std=c++17", "-I", B.CSRC, src, "-L", os.path.dirname(B.OUT),
                    "-l:" + os.path.basename(B.OUT), f"-Wl,-rpath,{os.path.dirname(B.OUT)}", "-o", exe], check=True, capture_output=True)

    def run(lines):
        out = subprocess.run([exe], input="\n".join(lines) + "\n", capture_output=True, text=True, check=True).stdout
        return [tuple(map(int, x.split())) for x in out.splitlines()]
    return run


def test_no_dimension_of_a_launch_wraps(ask):
    """Every workgroup is there, in dimensions that hold them with 512 threads each."""
    cases = [1, 2, 255, 1 << 22, (1 << 22) + 1, 1 << 24, (1 << 24) + 3, (1 << 27) + 65535, 1 << 31]
    for n, (x, rows) in zip(cases, ask([f"g {n}" for n in cases])):
        assert x * 512 < 1 << 32 and rows <= 65535 and n <= x * rows < n + (1 << 22)
        assert rows == 1 or n > 1 << 22
