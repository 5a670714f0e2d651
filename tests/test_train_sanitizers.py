"""The host code of the operators of a training step (gated layouts, launch
planning, gradient lists, argument checks; capi_train.cpp) built with the address and
undefined-behaviour sanitizers and driven by tests/sanitize/train_abi_check.cpp.  CPU
only: the kernel launchers are stubs."""
import os
import shutil
import subprocess

import pytest

from tests.test_host_sanitizers import CSRC, FLAGS, ROCM, SAN

SOURCES = [os.path.join(CSRC, f) for f in ("layout.cpp", "capi.cpp", "capi_train.cpp")] + [
    os.path.join(SAN, f) for f in ("kernel_stubs.cpp", "train_kernel_stubs.cpp", "train_abi_check.cpp")]


def test_train_abi_under_sanitizers(tmp_path):
    if shutil.which("g++") is None or not os.path.isdir(f"{ROCM}/include/hip"):
        pytest.skip("needs g++ and the HIP headers")
    objs, procs = [], []
    for src in SOURCES:
        objs.append(str(tmp_path / (os.path.basename(src) + ".o")))
        procs.append(subprocess.Popen(["g++", *FLAGS, f"-I{SAN}", "-c", src, "-o", objs[-1]], stdout=subprocess.PIPE,
                                      stderr=subprocess.STDOUT))
    for p in procs:
        out = p.communicate()[0].decode()
        assert p.returncode == 0, out
    exe = str(tmp_path / "train_abi_check")
    r = subprocess.run(["g++", *FLAGS, *objs, f"-L{ROCM}/lib", "-lamdhip64", f"-Wl,-rpath,{ROCM}/lib", "-o", exe],
                       capture_output=True, text=True)
    assert r.returncode == 0, r.stdout + r.stderr
    env = dict(os.environ, ASAN_OPTIONS="detect_leaks=1", UBSAN_OPTIONS="halt_on_error=1:print_stacktrace=1")
    r = subprocess.run([exe], capture_output=True, text=True, env=env, timeout=300)
    out = r.stdout + r.stderr
    print(out[-4000:])
    assert r.returncode == 0, out[-4000:]
    assert "0 failed expectations" in out
    assert "runtime error" not in out and "AddressSanitizer" not in out
