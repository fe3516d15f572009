"""Speculative decoding end to end (examples/verify_cycle.py): drafted trees verified through the
rotary, cache, tree-attention and accepted-row operators give the text that decoding token by
token gives, and the accepted tokens vary in number."""
import os
import sys

import pytest

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def cycle():
    sys.path.insert(0, os.path.join(ROOT, "examples"))
    import verify_cycle
    return verify_cycle


def test_drafted_text_equals_plain_text(cycle):
    """float32: the tree pass and the single-token pass agree to ~1e-6 of the logits, far below the
    gaps between a random head's largest logits."""
    text, plain, accepted = cycle.run("f32", steps=24)
    assert text == plain
    assert len({n for acc in accepted for n in acc}) > 1 and max(n for acc in accepted for n in acc) == 3


@pytest.mark.parametrize("cache", ["bf16", "e4m3"])
def test_reduced_caches_agree_at_the_start(cycle, cache):
    """16- and 8-bit caches: tree and single-token passes round alike up to the order of sums, so the
    texts may part at a near-tie but not at once; the planted tokens before that are accepted."""
    text, plain, accepted = cycle.run(cache, steps=12)
    for t, p in zip(text, plain):
        assert t[:3] == p[:3]
    assert max(n for acc in accepted for n in acc) >= 2
