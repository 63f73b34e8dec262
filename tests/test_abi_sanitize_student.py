"""The host code of the recurrence, the distillation and the verification, and of the vocabulary's calls, under AddressSanitizer and UndefinedBehaviorSanitizer:
tests/host/abi_sanitize_student.c walks through their argument checks and size queries, up to the largest descriptors.  No GPU is needed."""
import os
import shutil
import subprocess

import pytest

from test_abi_sanitize import CLANG, ROOT


def _library():
    """The instrumented library, built unless it is newer than everything that it is built from."""
    from paper_1805_08899_amd import build
    parts = [os.path.join(d, f) for d in (build.CSRC, os.path.join(ROOT, "include")) for f in os.listdir(d)] + [build.__file__]
    if os.path.exists(build.SAN_LIB) and os.path.getmtime(build.SAN_LIB) > max(map(os.path.getmtime, parts)):
        return build.SAN_LIB
    return build.build_library(sanitize=True, verbose=False)


@pytest.mark.skipif(not os.path.exists(CLANG) or shutil.which("hipcc") is None, reason="needs ROCm's clang and hipcc")
def test_host_side_of_the_students_calls_under_sanitizers(tmp_path):
    lib = _library()
    symbols = subprocess.run(["nm", "-D", lib], capture_output=True, text=True).stdout
    assert "__asan_" in symbols and "__ubsan_" in symbols, "the host code is not instrumented"
    runtime = os.path.dirname(subprocess.run([CLANG, "-print-file-name=libclang_rt.asan-x86_64.so"], capture_output=True, text=True).stdout.strip())
    exe = str(tmp_path / "abi_sanitize_student")
    r = subprocess.run([CLANG, "-std=c99", "-g", "-Wall", "-Werror", "-fsanitize=address,undefined", "-fno-sanitize-recover=undefined", "-shared-libsan",
                        "-I", os.path.join(ROOT, "include"), os.path.join(ROOT, "tests", "host", "abi_sanitize_student.c"), "-o", exe,
                        "-L", os.path.dirname(lib), "-lechoattn_san", f"-Wl,-rpath,{os.path.dirname(lib)}", f"-Wl,-rpath,{runtime}"],
                       capture_output=True, text=True)
    assert r.returncode == 0, r.stderr
    env = dict(os.environ, ASAN_OPTIONS="verify_asan_link_order=0:detect_leaks=0:abort_on_error=0", UBSAN_OPTIONS="print_stacktrace=1:halt_on_error=1")
    r = subprocess.run([exe], capture_output=True, text=True, env=env, timeout=120)
    assert r.returncode == 0 and r.stdout.strip() == "ok", (r.stdout, r.stderr)
    assert "AddressSanitizer" not in r.stderr and "runtime error" not in r.stderr, r.stderr
