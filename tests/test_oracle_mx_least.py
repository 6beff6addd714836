"""How far a quantised element may be off: the bound that the header states, down to blocks whose shared exponent is at its least."""
import numpy as np
import pytest

from oracle import mx


@pytest.mark.parametrize("fmt,own,of_largest,least", [("mxfp4", 2.0 ** -2, 2.0 ** -3, -125), ("mxfp8", 2.0 ** -4, 2.0 ** -17, -117)])
def test_the_stated_bound(fmt, own, of_largest, least):
    """At most 2^-4 (2^-2) of the element, or 2^-17 (2^-3) of its block's largest, or where the exponent is at its least half of the smallest step, 2^-127."""
    rng = np.random.default_rng(0)
    beyond = 0
    for size in list(range(-135, -100)) + [-60, 0, 100, 126]:
        x = rng.standard_normal((200, 32)) * rng.choice([1.0, 2.0 ** -6, 2.0 ** -12], (200, 32))
        x *= 2.0 ** size / np.abs(x).max(-1, keepdims=True) * (1 + rng.random((200, 1)))             # the largest between 2^size and 2^(size + 1)
        _, scale = mx.encode(x, fmt)
        off = np.abs(mx.held(x, fmt) - x)
        bound = np.maximum(own * np.abs(x), of_largest * np.abs(x).max(-1, keepdims=True))
        at_least = scale == least + 127
        assert np.all(off <= np.maximum(bound, np.where(at_least, 2.0 ** -127, 0)))
        beyond += int(np.sum((off > bound) & at_least))
    assert beyond > 0                                               # the third part is needed
