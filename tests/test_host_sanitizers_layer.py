"""The host side of the operators around the recurrence (csrc/kla_layer_api.hip: validation, offsets, workspace plans, dispatch) built with clang's
AddressSanitizer and UndefinedBehaviorSanitizer, device code not instrumented, under tests/test_layer_abi.py: every refusal and every
workspace query.  CPU only; runs when KLA_RUN_SANITIZERS=1 is set, like the recurrence's (tests/host_sanitizers.py)."""
import glob
import os
import subprocess
import sys
from concurrent.futures import ThreadPoolExecutor

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.mark.skipif(os.environ.get("KLA_RUN_SANITIZERS") != "1", reason="set KLA_RUN_SANITIZERS=1 (compiles the library once more)")
def test_host_sanitizers_layer(tmp_path):
    from paper_2605_08587_amd import build
    hipcc = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
    flags = [f for f in build.FLAGS if f != "-shared"]
    san = ["-Xarch_host", "-fsanitize=address", "-Xarch_host", "-fsanitize=undefined", "-Xarch_host", "-fno-sanitize-recover=all", "-Xarch_host", "-g"]

    def compile_one(src):
        obj = str(tmp_path / (src + ".o"))
        subprocess.check_call([hipcc, *flags, *(san if src == "kla_layer_api.hip" else []), "-c", os.path.join(build.CSRC, src), "-o", obj],
                              stderr=subprocess.DEVNULL)
        return obj
    with ThreadPoolExecutor(max_workers=8) as pool:
        objs = list(pool.map(compile_one, build.SOURCES))
    lib = str(tmp_path / "libkla_san.so")
    # host-only link of the sanitizer runtimes (no -Xarch_ option on this line, device sanitizers explicitly off)
    subprocess.check_call([hipcc, "--offload-arch=gfx950", "-shared", "-fPIC", "-fno-gpu-sanitize", "-fsanitize=address", "-fsanitize=undefined",
                           "-shared-libsan", "-o", lib, *objs])
    runtime = glob.glob("/opt/rocm/lib/llvm/lib/clang/*/lib/linux/libclang_rt.asan-x86_64.so")
    assert runtime, "clang's shared AddressSanitizer runtime not found"
    pre = os.environ.get("LD_PRELOAD", "")
    env = dict(os.environ, ASAN_OPTIONS="detect_leaks=0:abort_on_error=1:halt_on_error=1", UBSAN_OPTIONS="halt_on_error=1:print_stacktrace=1",
               KLA_LIBRARY=lib, LD_PRELOAD=runtime[0] + (":" + pre if pre else ""))
    subprocess.check_call([sys.executable, "-m", "pytest", "-x", "-q", "-m", "not gpu", os.path.join(ROOT, "tests", "test_layer_abi.py")], env=env,
                          cwd=ROOT)
