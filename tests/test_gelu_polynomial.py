"""GELU's tail polynomial (CPU only): its constants as the kernel has them, rounded
to fp32 and evaluated in 64 bits, keep the relative error that is stated for it."""
import os
import re

import numpy as np
import torch

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))),
                    "paper_2407_01614_amd", "csrc")


def test_stated_error_of_the_tail():
    with open(os.path.join(CSRC, "activations.hip")) as f:
        source = f.read()
    body = source[source.index("Normal normal(float u)"):]
    body = body[:body.index("exp2f")]
    slope = re.search(r"fmaf\((\S+)f, u, 1\.0f\)", body).group(1)
    first = re.search(r"float q = (\S+)f;", body).group(1)
    rest = re.findall(r"q = __builtin_fmaf\(q, t, (\S+)f\);", body)
    assert len(rest) == 7
    stated = float(re.search(r"relative error, (\S+) at most over 0 <= u <= 14", source).group(1))
    assert stated <= 1.5e-7   # what the tests of the kernels allow it
    slope, *c = (float(np.float32(x)) for x in (slope, first, *rest))
    u = torch.linspace(0, 14, 2_000_001, dtype=torch.float64)
    t = 1 / (1 + slope * u)
    q = torch.zeros_like(t)
    for k in c:
        q = q * t + k
    want = torch.special.erfcx(u * 0.5 ** 0.5) / 2
    assert float((q * t / want - 1).abs().max()) <= stated
