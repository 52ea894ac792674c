"""AddressSanitizer + UndefinedBehaviorSanitizer build of the host side of the calls on a cache in a microscaling format: queries over
their whole ranges and refusals.  GPU code is not sanitized (not available here)."""
import os
import shutil

import pytest

from test_sanitizers import ENV, ROOT, SAN, _run


def test_host_side_under_asan_ubsan(tmp_path):
    hipcc = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
    if not (os.path.exists(hipcc) or shutil.which(hipcc)):
        pytest.skip("hipcc not found")
    exe = str(tmp_path / "mx_driver")
    csrc = os.path.join(ROOT, "paper_2402_11131_amd", "csrc")
    # the sanitizers go to the host pass only; the device pass is compiled as always
    cmd = [hipcc, "--offload-arch=gfx950", "-O1", "-g", "-std=c++17", "-Xarch_host", "-fsanitize=address", "-Xarch_host",
           "-fsanitize=undefined", "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
           "-Wno-unused-command-line-argument", "-parallel-jobs=4", "-I", os.path.join(ROOT, "include"), "-I", csrc,
           *(os.path.join(csrc, f) for f in ("ss_api.hip", "ss_kv_mx.hip", "ss_msa_mx.hip", "ss_msa_mx_rows.hip")), os.path.join(SAN, "mx_driver.cpp"),
           "-o", exe]
    r = _run(cmd, timeout=600)
    assert r.returncode == 0, r.stdout[-4000:]
    r = _run([exe], env=dict(ENV, ASAN_OPTIONS="detect_leaks=0"), timeout=120)
    assert r.returncode == 0 and "mx driver done" in r.stdout and "ERROR: AddressSanitizer" not in r.stdout and "runtime error" not in r.stdout, r.stdout
