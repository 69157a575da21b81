"""The polynomial behind gelu's tail, with the constants as they stand in the source, against erfcx in 64 bits: as near as its comment says."""
import os
import re

import numpy as np
from scipy import special

from paper_2608_24070_amd import build

TEXT = open(os.path.join(build.CSRC, "slim_act.h")).read()


def constants():
    slope = float(re.search(r"act_rcp\(__builtin_fmaf\(([\d.]+)f, __builtin_fabsf\(x\), 1\.f\)\)", TEXT).group(1))
    c = [float(v) for v in re.findall(r"-?\d+\.\d+", re.search(r"constexpr float c\[9\] = \{(.*?)\}", TEXT, re.S).group(1))]
    assert len(c) == 9
    return slope, c


def stated():
    exact, fp32 = re.search(r"relative error \(([\de.-]+) with these constants, ([\de.-]+) in fp32\)", TEXT).groups()
    return float(exact), float(fp32)


def test_error_of_the_polynomial():
    slope, c = constants()
    exact, fp32 = stated()
    x = np.linspace(0, 9.5, 400001) * np.sqrt(2)
    ref = special.erfcx(x / np.sqrt(2)) / 2
    t = 1 / (1 + slope * x)
    worst = np.abs(t * np.polyval(c[::-1], t) / ref - 1).max()
    assert exact / 2 < worst <= exact
    # step by step in 32 bits, with the roundings of fused operations
    f = np.float32
    xs = x.astype(f)
    t = (1 / (f(slope) * xs.astype(np.float64) + 1).astype(f).astype(np.float64)).astype(f)
    p = np.full_like(t, c[8])
    for v in c[7::-1]:
        p = (p.astype(np.float64) * t + float(f(v))).astype(f)
    ref = special.erfcx(xs.astype(np.float64) / np.sqrt(2)) / 2
    worst = np.abs((p * t).astype(f) / ref - 1).max()
    assert fp32 / 2 < worst <= fp32
