"""The polynomials of the selective scan's kernels (csrc/selective_scan.cuh), read from the source and evaluated in 64 bits, against what they stand
for: within the errors that their comments state."""
import os
import re

import numpy as np

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_1810_00952_b200", "csrc")
with open(os.path.join(CSRC, "selective_scan.cuh")) as f:
    SOURCE = f.read()


def values(text):
    return [float(np.float32(v)) for v in re.findall(r"-?[0-9.]+e?[-+]?[0-9]*(?=f)", text)]


def test_softplus_polynomial():
    of = values(re.search(r"constexpr float of\[10\] = \{([^}]*)\}", SOURCE).group(1))
    assert len(of) == 10 and of[0] == 1.0
    w = np.concatenate([np.linspace(0, 1, 100001)[1:], np.geomspace(1e-38, 1e-5, 1000)])
    off = sum(c * w ** (k + 1) for k, c in enumerate(of)) / np.log1p(w) - 1
    assert np.abs(off).max() <= 5.4e-9, np.abs(off).max()
    # of either sign in nearly equal measure: steps do not drift
    assert abs(off[:100000].mean()) <= 1e-9


def test_decays_of_long_memories():
    body = re.search(r"f32x2 decay2\(f32x2 x\)\s*\{(.*?)\n\}", SOURCE, re.S).group(1)
    c = [values(m)[0] for m in re.findall(r"pair\(([-0-9.e]+f), \1\)", body)]
    assert len(c) == 4 and c[3] == 1.0
    x = np.linspace(-0.03125, 0.03125, 20001)
    off = (((c[0] * x + c[1]) * x + c[2]) * x + c[3]) / np.exp2(x) - 1
    assert np.abs(off).max() <= 1e-8 and np.abs(off[np.abs(x) <= 0.015625]).max() <= 1e-8 / 16 + 2e-9
