"""The argument checks of the operators between a decoder's projections under AddressSanitizer and UndefinedBehaviorSanitizer (host
code only; every call returns before anything is enqueued)."""
import os
import shutil

import pytest

from test_sanitizers import ENV, ROOT, run


@pytest.mark.skipif(shutil.which("hipcc") is None, reason="needs hipcc to build the library's host code")
def test_argument_checks_under_asan_and_ubsan(tmp_path):
    from paper_2601_22813_amd import build
    lib = build.build_sanitized(str(tmp_path))
    exe = str(tmp_path / "decode_abi_check")
    clang = os.path.join(os.path.dirname(os.path.realpath(shutil.which("hipcc"))), "..", "lib", "llvm", "bin", "clang")
    if not os.path.exists(clang):
        clang = "/opt/rocm/lib/llvm/bin/clang"
    b = run([clang, "-O1", "-g", "-std=c11", "-fsanitize=address,undefined", "-fno-sanitize-recover=all", "-shared-libsan",
             os.path.join(ROOT, "tests", "sanitize", "decode_abi_check.c"), lib, f"-Wl,-rpath,{tmp_path}", "-o", exe])
    assert b.returncode == 0, b.stdout
    rt = run([clang, "-print-file-name=libclang_rt.asan-x86_64.so"]).stdout.strip()
    env = dict(ENV)
    if os.path.sep in rt:
        env["LD_LIBRARY_PATH"] = os.path.dirname(rt) + os.pathsep + env.get("LD_LIBRARY_PATH", "")
    r = run([exe], env=env, timeout=300)
    assert r.returncode == 0 and "decode abi: ok" in r.stdout, r.stdout
    assert "runtime error" not in r.stdout and "AddressSanitizer" not in r.stdout, r.stdout
