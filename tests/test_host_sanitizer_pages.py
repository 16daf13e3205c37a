"""The host code of the operators on a cache in pages under AddressSanitizer and UndefinedBehaviorSanitizer, as
test_host_sanitizer.py does it for the others (tests/host_sanitizer/pages_harness.cpp)."""
import os
import shutil
import subprocess

import pytest

from paper_2604_16855_amd import build as B

HERE = os.path.dirname(os.path.abspath(__file__))
SOURCES = ["tdq_api.hip", "tdq_cache.hip", "tdq_paged.hip"]       # (the harness calls nothing of the others)


@pytest.mark.skipif(shutil.which("hipcc") is None and not os.path.exists("/opt/rocm/bin/hipcc"), reason="hipcc not found")
def test_paged_host_code_under_sanitizers(tmp_path):
    hipcc = B.hipcc()
    flags = ["--offload-arch=gfx950", "--cuda-host-only", "-O1", "-g", "-std=c++17", "-fno-omit-frame-pointer",
             "-fsanitize=address,undefined", "-fno-sanitize-recover=undefined",
             "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops", "-Wno-unknown-warning-option",
             "-I", os.path.join(B.ROOT, "include"), "-I", B.CSRC]
    objs, jobs = [], []
    for src in [os.path.join(B.CSRC, s) for s in SOURCES] + [os.path.join(HERE, "host_sanitizer", "pages_harness.cpp")]:
        obj = str(tmp_path / (os.path.basename(src) + ".o"))
        jobs.append(subprocess.Popen([hipcc, *flags, "-x", "hip", "-c", src, "-o", obj], stderr=subprocess.PIPE, text=True))
        objs.append(obj)
    for j in jobs:
        err = j.communicate()[1]
        assert j.returncode == 0, err
    exe = str(tmp_path / "pages_harness")
    # (without the device images, and what the other sources define: see test_host_sanitizer.py)
    linker = next((c for c in (os.path.join(os.path.dirname(hipcc), "amdclang++"), "/opt/rocm/lib/llvm/bin/clang++",
                               "/opt/rocm/llvm/bin/clang++", shutil.which("clang++")) if c and os.path.exists(c)), None)
    if linker is None:
        pytest.skip("no clang++ of the ROCm toolchain to link the host-only objects with")
    r = subprocess.run([linker, "-fsanitize=address,undefined", *objs, "-o", exe, "-Wl,--unresolved-symbols=ignore-all"],
                       capture_output=True, text=True)
    assert r.returncode == 0, r.stderr
    env = dict(os.environ, ASAN_OPTIONS="detect_leaks=0:abort_on_error=0", UBSAN_OPTIONS="print_stacktrace=1")
    env.pop("LD_PRELOAD", None)
    r = subprocess.run([exe], capture_output=True, text=True, env=env, timeout=300)
    assert r.returncode == 0, r.stdout[-2000:] + r.stderr[-6000:]
    assert "0 failures" in r.stdout and int(r.stdout.split()[0]) > 300, r.stdout
