"""The library holds the kernels of the gated layer and of layer normalisation that
some call takes, and no others: what the host code chooses (driven through the entry
points in a host-only build, tests/sanitize/train_plan_check.cpp, and as
tests/test_gated_kernels.py lists it) against the library's symbols."""
import os
import re
import shutil
import subprocess

import pytest

from paper_2112_00029_amd import pixelfly as pf
from tests.test_gated_kernels import DMA, KERNELS, SMALL, STAGED
from tests.test_host_sanitizers import CSRC, FLAGS, ROCM, SAN

TYPES = {"unsigned short": "bf16", "float": "fp32"}


@pytest.fixture(scope="module")
def kernels():
    if shutil.which("nm") is None:
        pytest.skip("needs nm")
    out = subprocess.run(["nm", "-C", "--defined-only", pf.LIB_PATH], capture_output=True, text=True, check=True).stdout
    return [(m[1], [a.strip() for a in m[2].split(",")])
            for m in re.finditer(r"__device_stub__(\w+)<([^<>]*)>\(", out)]


def test_gated_forward_kernels(kernels):
    held = set()
    for name, a in kernels:
        if name == "ntd_kernel" and a[8] == "4":
            held.add((DMA, "bf16", int(a[0]), int(a[3]), int(a[0]) * int(a[1]), int(a[4]), int(a[6])))
        if name == "nt_kernel" and a[6] == "4":
            held.add((STAGED, TYPES[a[0]], int(a[1]), int(a[4]), int(a[1]) * int(a[2]), 32, 4))
        if name == "small_kernel" and a[4] == "4":
            # (Blocks of 64 and 128 share one, fp32 ones all.)
            blk = 0 if a[0] == "float" else 32 if a[1] == "2" else 64
            held.add((SMALL, TYPES[a[0]], blk, 32, 64, 32 if a[0] == "float" else 64, int(a[5])))
    taken = set()
    for (family, *tile), (dtype, _, _, _, b, _, _) in KERNELS:
        if family == SMALL:
            b = 0 if dtype == "fp32" else min(b, 64)
        taken.add((family, dtype, b, *tile))
    assert held == taken, (held - taken, taken - held)


def test_normalisation_kernels(kernels, tmp_path):
    if shutil.which("g++") is None or not os.path.isdir(f"{ROCM}/include/hip"):
        pytest.skip("needs g++ and the HIP headers")
    src = [os.path.join(CSRC, f) for f in ("layout.cpp", "capi.cpp", "capi_train.cpp")] + [
        os.path.join(SAN, f) for f in ("kernel_stubs.cpp", "train_kernel_stubs.cpp", "train_plan_check.cpp")]
    exe = str(tmp_path / "plans")
    r = subprocess.run(["g++", *FLAGS, f"-I{SAN}", *src, f"-L{ROCM}/lib", "-lamdhip64", f"-Wl,-rpath,{ROCM}/lib",
                        "-o", exe], capture_output=True, text=True)
    assert r.returncode == 0, r.stdout + r.stderr
    r = subprocess.run([exe], capture_output=True, text=True, timeout=300)
    assert r.returncode == 0 and "0 failed expectations" in r.stdout, r.stdout[-4000:] + r.stderr[-4000:]
    taken = set(re.findall(r"^(?:fwd|bwd) .*$", r.stdout, re.M))
    held = {f"{name[5:8]} {TYPES[a[0]]} {a[1]} {a[2]} {a[3]} {int(a[4] == 'true')}"
            for name, a in kernels if name in ("norm_fwd_kernel", "norm_bwd_kernel")}
    assert held == taken, (sorted(held - taken), sorted(taken - held))
