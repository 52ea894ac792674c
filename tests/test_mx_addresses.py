"""Address arithmetic of the cache in microscaling formats, run on the host: rows are counted with all 32 bits, and a lane's
register, from which the kernels take a row, reads as an int."""
import os
import shutil
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
PROGRAM = r"""
#include <stdio.h>
#include "ss_mx.h"
int main() {
  const long long rows[] = {0, 1, (1LL << 31) - 1, 1LL << 31, (1LL << 31) + 77, (1LL << 32) - 1};
  const int bytes[] = {2, 4, 32, 64, 128};
  for (long long r : rows)
    for (int b : bytes) {
      const int lane = (int)(unsigned)r;  // what __builtin_amdgcn_readlane returns
      printf("%lld %d %llu\n", r, b, (unsigned long long)ss::mx_row_at(lane, b));
    }
  return 0;
}
"""


def test_rows_beyond_31_bits(tmp_path):
    hipcc = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
    if not (os.path.exists(hipcc) or shutil.which(hipcc)):
        pytest.skip("hipcc not found")
    src, exe = tmp_path / "rows.hip", str(tmp_path / "rows")
    src.write_text(PROGRAM)
    csrc = os.path.join(ROOT, "paper_2402_11131_amd", "csrc")
    r = subprocess.run([hipcc, "--offload-arch=gfx950", "--offload-host-only", "-O1", "-std=c++17", "-I", os.path.join(ROOT, "include"), "-I", csrc,
                        str(src), "-o", exe], stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True, timeout=300)
    assert r.returncode == 0, r.stdout[-3000:]
    lines = subprocess.run([exe], stdout=subprocess.PIPE, text=True, timeout=60, check=True).stdout.split("\n")[:-1]
    assert len(lines) == 30
    for line in lines:
        row, size, at = map(int, line.split())
        assert at == row * size, line
