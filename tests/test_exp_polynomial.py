"""The polynomial that stands in for one exponential in eight in the prompt attention: its coefficients as they are written in the source,
evaluated with the kernel's roundings, against 2^f in 64 bits."""
import os
import re

import numpy as np

from tests.conftest import ROOT


def test_error_is_as_stated():
    with open(os.path.join(ROOT, "paper_2603_13180_b200", "csrc", "mxn_prompt.cu")) as f:
        text = f.read()
    body = text[text.index("float2 ex2_fma("):]
    body = body[:body.index("\n}\n")]
    c = [np.float32(v) for v in re.findall(r"float2 p = f2\(([\d.]+)f\)", body) + re.findall(r"__ffma2_rn\(p, f, f2\(([\d.]+)f\)\)", body)]
    assert len(c) == 6 and c[-1] == 1
    exact, rounded = (float(v) for v in re.search(r"as its constant: ([\d.e-]+), with the roundings ([\d.e-]+)", text).groups())
    x = np.unique(np.linspace(-0.5, 0.5, 1 << 20).astype(np.float32)).astype(np.float64)
    p, q = np.full_like(x, float(c[0])), np.full_like(x, float(c[0]))
    for v in c[1:]:
        p = p * x + float(v)
        q = (q * x + float(v)).astype(np.float32).astype(np.float64)   # a product and a sum in one rounding, but for 2^-53
    assert np.abs(p / np.exp2(x) - 1).max() <= exact
    assert np.abs(q / np.exp2(x) - 1).max() <= rounded
