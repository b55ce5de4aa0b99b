"""The exponential by polynomial at the lower end of binary32, with the kernels' roundings and bit operations: nothing is exactly nothing."""
import os
import re

import numpy as np
import pytest

from tests.conftest import ROOT


@pytest.mark.parametrize("name", ["mxn_prompt.cu", "mxn_weights_many.cu"])
def test_small_powers(name):
    with open(os.path.join(ROOT, "paper_2603_13180_b200", "csrc", name)) as f:
        text = f.read()
    body = text[text.index("float2 ex2_fma("):]
    body = body[:body.index("\n}\n")]
    least = np.float32(re.search(r"\w+\(u\.x, (-[\d.]+)f\)", body).group(1))
    c = [np.float32(v) for v in re.findall(r"float2 p = f2\(([\d.]+)f\)", body) + re.findall(r"__ffma2_rn\(p, f, f2\(([\d.]+)f\)\)", body)]
    u = np.concatenate([np.linspace(-130, -120, 1 << 16), [-127, -1e4, -1e30, -np.inf]]).astype(np.float32)
    magic = np.float32(12582912.0)
    v = np.maximum(u, least)
    t = v + magic
    f = v - (t - magic)
    p = np.full_like(f, c[0])
    for k in c[1:]:
        p = (p.astype(np.float64) * f + float(k)).astype(np.float32)
    y = (p.view(np.uint32) + (t.view(np.uint32) << np.uint32(23))).view(np.float32)
    assert bool((y[u <= -127] == 0).all()) and bool((y >= 0).all())
    with np.errstate(under="ignore"):
        want = np.exp2(u.astype(np.float64))
    # half of 2^-126 where the result has no exponent of its own, else the polynomial's error and rounding (2^-22)
    assert bool((np.abs(y - want) <= np.where(u < -126, 2.0 ** -127 * (1 + 2.0 ** -20), 2.0 ** -22 * want)).all())
