"""examples/draft_and_evict.py: drafting, acceptance, watched decoding and eviction together, against plain attention."""
import importlib.util
import os

import pytest

pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

PATH = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "draft_and_evict.py")


@pytest.mark.parametrize("shape", [dict(hq=32, hkv=8, dim=128), dict(hq=6, hkv=2, dim=64, layers=2)], ids=["d128", "d64"])
def test_cache_holds_what_was_accepted_and_kept(shape):
    spec = importlib.util.spec_from_file_location("draft_and_evict", PATH)
    example = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(example)
    lines = []
    worst = example.run(steps=6, check=True, log=lines.append, **shape)
    assert len(lines) == 6 and any("cut down" in x for x in lines) and not all("cut down" in x for x in lines)
    # in units of one rounding of every probability and of the result (bf16), and 1% for what is rounded in 32 bits
    assert worst <= 1.0
