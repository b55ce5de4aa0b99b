"""The keys' summed weights use the prompt attention's polynomial: the same function, whose error tests/test_exp_polynomial.py holds."""
import os

from tests.conftest import ROOT


def body(name):
    with open(os.path.join(ROOT, "paper_2603_13180_b200", "csrc", name)) as f:
        text = f.read()
    text = text[text.index("float2 ex2_fma("):]
    return text[:text.index("\n}\n")]


def test_same_polynomial():
    assert body("mxn_weights_many.cu") == body("mxn_prompt.cu")
