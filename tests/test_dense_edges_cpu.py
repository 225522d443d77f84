"""Dense row operators: layouts that a call must refuse because its output would overwrite what it has still to read.  Nothing is
launched: the pointers are never followed."""
import ctypes

import pytest

from paper_2307_03500_b200 import build as deft_build

deft_build.build()
from paper_2307_03500_b200 import deft  # noqa: E402

A, B, C = 1 << 20, 1 << 28, 1 << 29


def _rotary(xs, ys, batch, tokens, heads, dim=20, x=A, y=A):
    s = [(ctypes.c_int64 * 3)(*v) for v in (xs, ys)]
    return deft.lib().deft_rotary(x, s[0], y, s[1], 0, batch, tokens, heads, dim, C, dim, 0, 0, 1.0, None, 0, None)


@pytest.mark.parametrize("xs,ys,counts", [
    ((200, 40, 20), (40, 200, 20), (5, 5, 2)),       # batches and tokens change places
    ((500, 100, 20), (500, 20, 100), (2, 5, 5)),     # tokens and heads
    ((500, 100, 20), (20, 100, 500), (5, 5, 5)),     # batches and heads
    ((500, 100, 20), (100, 20, 500), (5, 5, 5)),     # all three
    ((0, 100, 20), (0, 20, 100), (1, 5, 5)),
], ids=str)
def test_rotary_refuses_a_transposition_in_place(xs, ys, counts):
    """The same elements in another order are not x, element for element."""
    assert _rotary(xs, ys, *counts) == deft.ERR_INVALID_ARG
