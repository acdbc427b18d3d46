"""The layer operators' kernels, compiled for gfx950 (CPU only), keep everything
in registers: no vector register spilled, no scratch memory.  A norm kernel that
spilled hundreds gave wrong results in lanes whose chunk lay past the row, and
the weight gradient's spills cost it a fifth of its speed; both run close to the
registers there are."""
import os
import re
import subprocess

import pytest

from paper_2407_01614_amd import build


@pytest.mark.skipif(not os.path.exists(build.hipcc()), reason="hipcc not found")
@pytest.mark.parametrize("source", ["activations.hip", "layer_norm.hip", "weight_grad.hip"])
def test_no_kernel_spills(source, tmp_path):
    flags = [f for f in build.HIPCC_FLAGS if f != "-shared"]
    r = subprocess.run([build.hipcc(), *flags, "--cuda-device-only", "-c",
                        "-Rpass-analysis=kernel-resource-usage", "-I", build.INCLUDE,
                        "-I", build.CSRC, os.path.join(build.CSRC, source),
                        "-o", str(tmp_path / "out.o")], capture_output=True, text=True)
    assert r.returncode == 0, r.stderr
    names = re.findall(r"Function Name: (\S+)", r.stderr)
    spills = re.findall(r"VGPRs Spill: (\d+)", r.stderr)
    scratch = re.findall(r"ScratchSize \[bytes/lane\]: (\d+)", r.stderr)
    assert names and len(names) == len(spills) == len(scratch)
    bad = [n for n, a, b in zip(names, spills, scratch) if int(a) or int(b)]
    assert not bad, bad
