"""Host-side checks of the operators around a verification: what can be known of them without a device."""
import ctypes as C
import os
import re

import numpy as np

from paper_2602_16994_b200 import build
from .test_step_cpu import Rope, filled, lib  # noqa: F401


def test_the_polynomial_for_exponentials():
    """The coefficients that the attention's kernel is built with, in its own arithmetic (fused in 32 bits), against 2^f."""
    with open(os.path.join(build.HERE, "csrc", "attend.cuh")) as f:
        text = re.search(r"EXP2_FIT\[5\] = \{(.*?)\}", f.read()).group(1)
    fit = [np.float32(x.strip().rstrip("f")) for x in text.split(",")]
    f = np.linspace(-0.5, 0.5, 200001).astype(np.float32)
    p = np.full_like(f, fit[4])
    for c in (*fit[3::-1], np.float32(1.0)):
        p = (p.astype(np.float64) * f.astype(np.float64) + np.float64(c)).astype(np.float32)
    assert float(np.abs(p.astype(np.float64) / np.exp2(f.astype(np.float64)) - 1.0).max()) < 2.0e-7
    assert p[f == 0] == 1.0


def test_token_counts_up_to_the_end_of_32_bits_are_refused(lib):  # noqa: F811
    """A CTA goes from token to token in steps of the grid: the step past the last token must not wrap round."""
    for tokens in (2**31 - 1, 2**31 - 4000):
        assert lib.spec_norm_rope_cache(C.byref(filled(Rope, D=64, rot=64, T=tokens)), None) == -2
