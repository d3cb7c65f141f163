"""The decoding example: projection, router and layer together, captured into a graph."""
import os
import sys

import pytest

pytestmark = pytest.mark.gpu
pytest.importorskip("torch")

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.mark.parametrize("extra", [[], ["--dense"], ["--tokens", "1", "--experts", "40", "--k", "6"], ["--tokens", "20"]])
def test_routed_decode(extra):
    sys.path.insert(0, os.path.join(ROOT, "examples"))
    try:
        import routed_decode
    finally:
        sys.path.pop(0)
    # y, the shares, D and the sum X + D are rounded to bf16 (2^-9 of their size on the average, errors of a norm):
    # four such roundings and what a rounded y does to the products behind it stay below 1e-2
    assert routed_decode.main(["--width", "256", "--hidden", "192"] + extra) < 1e-2
