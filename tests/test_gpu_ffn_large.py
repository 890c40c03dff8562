"""Blocks of the feed-forward unit's largest tiles that go on from tile to tile, in
every form of the product: their next tile's first loads are under way while a tile's
results are stored, and the waits count those stores.  tests/test_ffn_plans.py checks
that the sizes here still take these tiles, more of them than there are CUs."""

import numpy as np
import pytest

from oracle import blocks as O  # noqa: F401  (the oracle of Unit's checks)
from tests.test_gpu_blocks import Unit

pytestmark = pytest.mark.gpu

# (rows, channels, hidden), the products that it is here for, and whether gate, up and
# act are stored and gradients taken.  Most have part of a tile last in rows and
# columns; contracted axes of 1, 2, 3, 10, 11 and 32 steps and parts of one, whole and
# in slices that end inside a segment of dx.
CASES = [
    ((12400, 2056, 2056), ("gated_saved", "down", "dhidden", "dx"), True),
    ((1827, 632, 15272), ("gated_saved", "dhidden"), True),
    ((147, 3512, 10592), ("weights",), True),
    ((678, 1448, 7072), ("weights",), True),
    ((7208, 12720, 136), ("weights_sliced",), True),
    ((22801, 136, 3512), ("dx_sliced",), True),
    ((121275, 136, 8), ("dx",), True),
    ((109253, 8, 104), ("gated_saved",), True),
    ((12400, 2056, 2056), ("gated", "down"), False),
    ((121275, 80, 80), ("gated",), False),
    ((34635, 136, 4224), ("gated", "down_sliced"), False),
]
# dX takes the largest tiles where w_gate and w_up have one stride, and others where
# they have two.
STRIDES = (8100, 2048, 2056)


def _some(rows):
    """Rows at both ends and throughout."""
    return np.unique(np.concatenate([np.arange(min(rows, 300)), np.arange(max(0, rows - 300), rows), np.arange(0, rows, 61)]))


@pytest.mark.parametrize("size,products,train", CASES)
def test_tile_after_tile(size, products, train):
    import torch
    c = Unit("bf16", *size, size[0] % 2 == 1, 8, saved=train).forward().check(_some(size[0]))
    if train:
        c.gradients().check_gradients()
    results = [c.out] + [t for t in c.saved if t is not None] + (c.grads if train else [])
    first = [t.x.clone() for t in results]
    for _ in range(3):
        for t in results:
            t.x.fill_(float("nan"))
        c.forward()
        if train:
            c.gradients()
            results[4:] = c.grads
        assert all(torch.equal(a, t.x) for a, t in zip(first, results))


def test_two_strides_where_one_would_take_the_largest_tiles():
    """The step from one weight's rows to the other's with strides that differ."""
    c = Unit("bf16", *STRIDES, False, apart=True).forward()
    c.check(_some(STRIDES[0])).gradients(want=(1, 1, 1, 1)).check_gradients()
    c.gradients(want=(1, 0, 0, 0)).check_gradients()
