"""The paged cache's host-side validation under AddressSanitizer and UndefinedBehaviorSanitizer, against stub launchers: a host-only build
made here, nothing touches a GPU."""
import os
import shutil
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
SAN = os.path.join(ROOT, "tests", "sanitize")
CSRC = os.path.join(ROOT, "paper_2601_01298_amd", "csrc")
ENV = dict(os.environ, ASAN_OPTIONS="detect_leaks=0:verify_asan_link_order=0", UBSAN_OPTIONS="print_stacktrace=1")


def run(cmd, **kw):
    r = subprocess.run(cmd, capture_output=True, text=True, timeout=600, **kw)
    return r.returncode, "\n".join(l for l in (r.stdout + r.stderr).splitlines() if "not a recognized feature" not in l)


def test_paged_validation_under_sanitizers(tmp_path):
    hipcc, clang = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc"), "/opt/rocm/bin/amdclang"
    if shutil.which(hipcc) is None or not os.path.exists(clang):
        pytest.skip("no hipcc on this host")
    san = ["-Xarch_host", "-fsanitize=address", "-Xarch_host", "-fsanitize=undefined", "-Xarch_host", "-fno-sanitize-recover=all"]
    objs = []
    for src in (os.path.join(CSRC, "api.hip"), os.path.join(CSRC, "paged_api.hip"), os.path.join(SAN, "api_stubs.cpp"), os.path.join(SAN, "paged_stubs.cpp")):
        objs.append(str(tmp_path / (os.path.basename(src) + ".o")))
        rc, out = run([hipcc, "--offload-arch=gfx950", "-O1", "-g", "-std=c++17"] + san + ["-x", "hip", "-c", src, "-o", objs[-1]])
        assert rc == 0, out
    drv = str(tmp_path / "driver.o")
    rc, out = run([clang, "-O1", "-g", "-fsanitize=address,undefined", "-fno-sanitize-recover=all", "-c", os.path.join(SAN, "paged_driver.c"), "-o", drv])
    assert rc == 0, out
    exe = str(tmp_path / "checks")
    rc, out = run([hipcc, "--offload-arch=gfx950", "-fsanitize=address,undefined"] + objs + [drv, "-lm", "-o", exe])
    assert rc == 0, out
    rc, out = run([exe], env=ENV)
    assert rc == 0 and "all checks passed" in out, out
