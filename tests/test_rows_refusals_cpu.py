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


@pytest.mark.parametrize("kw", [
    dict(ty=1), dict(tx=1), dict(tx=1, ty=2),                                   # x's place, but other elements
    dict(ld_x=9), dict(ld_y=9), dict(ld_y=16),                                  # ... or another pitch
    dict(y=A + 4), dict(x=A + 4), dict(y=A + 3 * 32 + 28), dict(x=A + 3 * 32),  # shifted by an element, or as far as the last row
    dict(y=A + 40, ld_x=16, ld_y=16), dict(y=A + 64 + 28, ld_x=16, ld_y=16),    # the same pitch: into its own row's end, a later row's start
    dict(y=A + 4, rows=1), dict(y=A, ty=1, rows=1, ld_x=100),
    dict(x=2 * A, add=A, ld_add=9), dict(x=2 * A, add=A, ld_add=8, y=A + 4), dict(x=2 * A, add=A + 64, ld_add=8),
    dict(y=A + 32, ld_x=16, ld_y=24),                                           # different pitches: y's second row is x's third
    dict(rows=2 ** 20, y=A + 4 * (2 ** 23 - 1), ld_x=8, ld_y=9),
], ids=lambda kw: ",".join("%s=%s" % i for i in kw.items()))
def test_dropout_refuses_outputs_that_overlap_its_inputs(kw):
    """y is x or add, element for element, or apart from both: anything else would be written before another thread reads it."""
    assert _dropout(**kw) == deft.ERR_INVALID_ARG
