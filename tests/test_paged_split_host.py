"""The paged attention's plan with the real split rule (zsa_paged_split.cpp)
under AddressSanitizer and UndefinedBehaviorSanitizer, host-only; the launches
are stand-ins that record the jobs."""
import os
import shutil
import subprocess
import tempfile

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
HIPCC = "/opt/rocm/bin/hipcc"
CLANG = "/opt/rocm/llvm/bin/clang++"
# the sanitizers go to the host compilation only (each flag behind -Xarch_host)
SAN = ["-Xarch_host", "-fsanitize=address", "-Xarch_host", "-fsanitize=undefined",
       "-Xarch_host", "-fno-sanitize-recover=undefined"]
CSRC = os.path.join(ROOT, "paper_2509_01190_amd", "csrc")
SOURCES = [os.path.join(CSRC, "zsa_paged.cpp"), os.path.join(CSRC, "zsa_paged_split.cpp"),
           os.path.join(ROOT, "tests", "host", "paged_split_driver.cpp")]


@pytest.mark.skipif(not (os.path.exists(HIPCC) and os.path.exists(CLANG)), reason="ROCm compilers not installed")
def test_split_rule_under_sanitizers():
    tmp = tempfile.mkdtemp(prefix="zsa_split_")
    try:
        objs = []
        for src in SOURCES:
            obj = os.path.join(tmp, os.path.basename(src) + ".o")
            subprocess.run([HIPCC, "-x", "hip", "--cuda-host-only", "--offload-arch=gfx950", "-std=c++17", "-O1", "-g",
                            "-fno-omit-frame-pointer", *SAN, "-c", src, "-o", obj],
                           check=True, capture_output=True, text=True, timeout=300)
            objs.append(obj)
        exe = os.path.join(tmp, "paged_split_driver")
        subprocess.run([CLANG, "-fsanitize=address,undefined", *objs, "-o", exe],
                       check=True, capture_output=True, text=True, timeout=300)
        env = dict(os.environ, ASAN_OPTIONS="detect_leaks=1:abort_on_error=0",
                   UBSAN_OPTIONS="print_stacktrace=1:halt_on_error=1")
        r = subprocess.run([exe], capture_output=True, text=True, timeout=300, env=env)
        assert r.returncode == 0, r.stdout + r.stderr
        assert r.stdout.startswith("ok ") and int(r.stdout.split()[1]) > 100000, r.stdout
        assert "runtime error" not in r.stderr, r.stderr
    finally:
        shutil.rmtree(tmp, ignore_errors=True)
