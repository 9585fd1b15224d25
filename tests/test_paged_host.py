"""The host code of the paged cache's entry points under AddressSanitizer and
UndefinedBehaviorSanitizer, host-only, with device-side stand-ins that record
what a call launches: over random calls the jobs cover every key and their
parts stay inside the workspace."""
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
SOURCES = [os.path.join(ROOT, "paper_2509_01190_amd", "csrc", "zsa_paged.cpp"),
           os.path.join(ROOT, "tests", "host", "paged_driver.cpp")]


@pytest.mark.skipif(not (os.path.exists(HIPCC) and os.path.exists(CLANG)), reason="ROCm compilers not installed")
def test_paged_calls_under_sanitizers():
    tmp = tempfile.mkdtemp(prefix="zsa_paged_")
    try:
        objs = []
        for src in SOURCES:
            obj = os.path.join(tmp, os.path.basename(src) + ".o")
            subprocess.run([HIPCC, "-x", "hip", "--cuda-host-only", "--offload-arch=gfx950", "-O1", "-g",
                            "-fno-omit-frame-pointer", *SAN, "-c", src, "-o", obj],
                           check=True, capture_output=True, text=True, timeout=300)
            objs.append(obj)
        exe = os.path.join(tmp, "paged_driver")
        subprocess.run([CLANG, "-fsanitize=address,undefined", *objs, "-o", exe],
                       check=True, capture_output=True, text=True, timeout=300)
        env = dict(os.environ, ASAN_OPTIONS="detect_leaks=1:abort_on_error=0",
                   UBSAN_OPTIONS="print_stacktrace=1:halt_on_error=1")
        r = subprocess.run([exe], capture_output=True, text=True, timeout=300, env=env)
        assert r.returncode == 0, r.stdout + r.stderr
        assert r.stdout.startswith("ok ") and int(r.stdout.split()[1]) > 10000, r.stdout
        assert "runtime error" not in r.stderr, r.stderr
    finally:
        shutil.rmtree(tmp, ignore_errors=True)
