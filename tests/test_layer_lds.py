"""LDS of the layer operators' launches (CPU only): what passes 64 KB is asked for,
for each kernel and device, over the widths at which the kernels change."""
import os
import shutil
import subprocess

import pytest

HERE = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(HERE)
PKG = os.path.join(ROOT, "paper_2407_01614_amd")
ROCM = os.environ.get("ROCM_PATH", "/opt/rocm")


@pytest.mark.skipif(not shutil.which("g++"), reason="g++ not found")
def test_large_lds_is_asked_for(tmp_path):
    if not os.path.exists(os.path.join(PKG, "libzpp.so")):
        from paper_2407_01614_amd import build
        build.build()
    exe = str(tmp_path / "layer_lds_check")
    r = subprocess.run(["g++", "-O1", "-std=c++17", "-Wall", "-D__HIP_PLATFORM_AMD__",
                        "-I", os.path.join(ROOT, "include"), "-isystem",
                        os.path.join(ROCM, "include"), os.path.join(HERE, "layer_lds_check.cpp"),
                        "-o", exe, os.path.join(PKG, "libzpp.so"), "-Wl,-rpath," + PKG,
                        "-Wl,-rpath-link," + os.path.join(ROCM, "lib"),
                        "-Wl,-rpath," + os.path.join(ROCM, "lib")],
                       capture_output=True, text=True)
    assert r.returncode == 0, r.stderr
    r = subprocess.run([exe], capture_output=True, text=True, timeout=120)
    assert r.returncode == 0, r.stdout + r.stderr
