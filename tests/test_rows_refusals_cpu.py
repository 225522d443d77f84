"""Refusals of the row operators' C ABI beyond single bad arguments: scales that do not fit fp32, and dropout whose output
overlaps its inputs.  Everything is refused on the host; the pointers are never followed."""
import numpy as np
import pytest

from paper_2307_03500_b200 import build as deft_build
from tests.test_rows_cpu import A, _dropout, _embed, _grad

deft_build.build()
from paper_2307_03500_b200 import deft  # noqa: E402

FLT_MAX = float(np.finfo(np.float32).max)


@pytest.mark.parametrize("scale", [1e39, -1e39, 1e308, 2.0 ** 128, FLT_MAX * (1 + 2.0 ** -24)])
def test_scales_that_no_fp32_number_holds(scale):
    """The products are fp32: such a scale would turn the zeros of a row outside the table into NaN."""
    assert _embed(scale=scale) == deft.ERR_INVALID_ARG
    assert _grad(scale=scale) == _grad(n=0, acc=1, dy=None, ids=None, scale=scale) == deft.ERR_INVALID_ARG


def test_scales_that_overflow_with_the_gain():
    """The gradient's factor is scale times the gain of the kept elements, rounded once."""
    nothing = dict(n=0, acc=1, dy=None, ids=None)
    for scale, p, ok in [(FLT_MAX, 0.0, True), (-FLT_MAX, 0.0, True), (FLT_MAX, 0.5, False), (FLT_MAX / 2, 0.5, True), (1e35, 0.9999, False),
                         (1e35, 0.99, True), (-3e38, 0.25, False)]:
        assert _grad(scale=scale, p=p, **nothing) == (deft.OK if ok else deft.ERR_INVALID_ARG)
    assert _embed(n=0, scale=FLT_MAX, table=None, ids=None, out=None) == deft.OK
