"""examples/shared_prompt.py: the rotated append and attention over shared prefixes together, step after step, against plain attention.

The cached keys that the plain side holds are rounded from 64 bits, the kernels' from binary32: where the two fall on different sides of a rounding
border a key element differs by one step.  That happens to a share of about 2^-12 of the elements (bf16; the rotation in binary32 is off by 2^-21
or so, a step is 2^-8) and moves a score by 2^-8 |q k| of one element, which the next figures allow for: a score of D products, a share 2^-12
of them off by 2^-8 of a product of size 1 / sqrt(D), adds below 2^-14 to the error relative to the bound's 2^-8.  FP8: a step is 2^-4 at most and
the share 2^-16."""
import importlib.util
import os

import pytest

pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

PATH = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "shared_prompt.py")


@pytest.mark.parametrize("shape", [dict(hq=32, hkv=8, dim=128, batch=12), dict(hq=6, hkv=2, dim=64, layers=2, batch=9, prompt=777, turn=90),
                                   dict(hq=8, hkv=1, dim=128, layers=2, batch=20, prompt=1024, fp8=True)], ids=["d128", "d64", "fp8"])
def test_conversations_attend_to_what_they_should(shape):
    spec = importlib.util.spec_from_file_location("shared_prompt", PATH)
    example = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(example)
    lines = []
    worst = example.run(steps=4, check=True, log=lines.append, **shape)
    assert len(lines) == 4
    # in units of one rounding of every probability and of the result (bf16), and 1% for the rest
    assert worst <= 1.0
