"""Row operators without a GPU: the generator against its published known answers, the mask's rate, and the refusals
of the C ABI (every refusal happens on the host, before anything touches a device)."""
import ctypes

import numpy as np
import pytest

from paper_2307_03500_b200 import build as deft_build
from tests import rows_plain as P

deft_build.build()
from paper_2307_03500_b200 import deft  # noqa: E402

NAN, INF = float("nan"), float("inf")


@pytest.mark.parametrize("counter,key,want", [
    # the known-answer vectors published with the generator
    ([0, 0, 0, 0], [0, 0], [0x6627E8D5, 0xE169C58D, 0xBC57AC4C, 0x9B00DBD8]),
    ([0xFFFFFFFF] * 4, [0xFFFFFFFF] * 2, [0x408F276D, 0x41C83B0E, 0xA20BC7C6, 0x6D5451FD]),
    ([0x243F6A88, 0x85A308D3, 0x13198A2E, 0x03707344], [0xA4093822, 0x299F31D0], [0xD16CFE09, 0x94FDCCEB, 0x5001E420, 0x24126EA1]),
])
def test_generator_known_answers(counter, key, want):
    assert [int(x[0]) for x in P.philox([np.array([c]) for c in counter], key)] == want


@pytest.mark.parametrize("p", [0.1, 0.5, 0.9])
def test_rate_of_the_mask(p):
    k = P.keep(2000, 1000, p, 77, 5)
    n = k.size
    assert abs(k.mean() - (1 - P.threshold(p) / 65536)) < 5 * np.sqrt(p * (1 - p) / n)      # five standard deviations
    assert np.abs(k.mean(0) - k.mean()).max() < 6 * np.sqrt(p * (1 - p) / 2000)             # every column
    other = P.keep(2000, 1000, p, 77, 6)
    agree = (k == other).mean()
    assert abs(agree - (p * p + (1 - p) ** 2)) < 5e-3                                       # another offset: independent


def test_types_and_sizes_of_the_binding():
    header = open(deft_build._ROOT + "/include/deft.h").read()
    assert "#define DEFT_MAX_PARTS %d\n" % deft.MAX_PARTS in header
    assert "#define DEFT_EMBED_MAX_ROWS %dLL\n" % deft.EMBED_MAX_ROWS in header
    for args in [(-1, 5, 5), (5, 0, 5), (5, 5, 0), (2 ** 31, 5, 5), (5, deft.EMBED_MAX_ROWS + 1, 5)]:
        assert deft.deft_embed_workspace_bytes(*args) == 0
    small, large = deft.deft_embed_workspace_bytes(10, 50, 8), deft.deft_embed_workspace_bytes(1000, 50, 8)
    assert 0 < small < large


# Plausible arguments; every test replaces one of them.  The pointers are never followed: the calls refuse first.
A = 0x10000


def _embed(**kw):
    a = dict(table=A, tt=0, rows=10, width=8, ld_table=8, ids=A, id_bytes=8, n=4, scale=1.0, pos=None, pos_rows=0, ld_pos=0, p=0.0, seed=0,
             offset=0, offset_d=None, out=A, to=0, ld_out=8, stream=None)
    a.update(kw)
    return deft.lib().deft_embed(*a.values())


def _grad(**kw):
    a = dict(dy=A, t=0, ld=8, ids=A, id_bytes=8, n=4, rows=10, width=8, skip=-1, scale=1.0, p=0.0, seed=0, offset=0, offset_d=None, grad=A,
             acc=0, ws=A, ws_bytes=1 << 30, stream=None)
    a.update(kw)
    return deft.lib().deft_embed_grad(*a.values())


def _dropout(**kw):
    a = dict(x=A, tx=0, ld_x=8, add=None, ld_add=0, y=A, ty=0, ld_y=8, rows=4, cols=8, p=0.5, seed=0, offset=0, offset_d=None, stream=None)
    a.update(kw)
    return deft.lib().deft_dropout(*a.values())


@pytest.mark.parametrize("kw", [dict(table=None), dict(ids=None), dict(out=None), dict(tt=3), dict(to=-1), dict(rows=0), dict(width=0), dict(n=-1),
                                dict(ld_table=7), dict(ld_out=7), dict(id_bytes=2), dict(scale=NAN), dict(scale=INF), dict(p=1.0), dict(p=-0.1),
                                dict(p=NAN), dict(table=A + 2), dict(out=A + 1, to=1), dict(ids=A + 4), dict(pos=A, pos_rows=0, ld_pos=8),
                                dict(pos=A, pos_rows=2, ld_pos=7), dict(pos=A + 2, pos_rows=2, ld_pos=8), dict(offset_d=A + 4)])
def test_embed_refuses(kw):
    assert _embed(**kw) == deft.ERR_INVALID_ARG


@pytest.mark.parametrize("kw", [dict(dy=None), dict(ids=None), dict(grad=None), dict(ws=None), dict(t=3), dict(id_bytes=1), dict(n=-1), dict(rows=0),
                                dict(width=0), dict(ld=7), dict(scale=INF), dict(p=1.0), dict(p=NAN), dict(dy=A + 2), dict(grad=A + 2),
                                dict(ws=A + 128), dict(ids=A + 4), dict(offset_d=A + 1)])
def test_embed_grad_refuses(kw):
    assert _grad(**kw) == deft.ERR_INVALID_ARG


@pytest.mark.parametrize("kw", [dict(x=None), dict(y=None), dict(tx=7), dict(ty=-2), dict(rows=-1), dict(cols=-1), dict(ld_x=7), dict(ld_y=7),
                                dict(add=A, ld_add=7), dict(add=A + 1, ld_add=8), dict(p=1.0), dict(p=-1e-9), dict(p=NAN), dict(x=A + 3)])
def test_dropout_refuses(kw):
    assert _dropout(**kw) == deft.ERR_INVALID_ARG


def test_sizes_beyond_a_call():
    big = 2 ** 31
    assert _embed(n=big) == _embed(rows=big) == _embed(width=big, ld_table=big, ld_out=big) == deft.ERR_TOO_LARGE
    assert _grad(n=big) == _grad(rows=deft.EMBED_MAX_ROWS + 1) == _grad(width=big, ld=big) == deft.ERR_TOO_LARGE
    assert _dropout(rows=big) == _dropout(cols=big, ld_x=big, ld_y=big) == deft.ERR_TOO_LARGE
    assert _grad(ws_bytes=100) == deft.ERR_CAPACITY


def test_nothing_to_do():
    assert _embed(n=0, table=None, ids=None, out=None) == deft.OK
    assert _grad(n=0, dy=None, ids=None, acc=1) == deft.OK
    assert _dropout(rows=0, x=None, y=None) == deft.OK
    assert _dropout(cols=0, ld_x=0, ld_y=0, x=None, y=None) == deft.OK


@pytest.mark.parametrize("parts", [[(5, 3)], [(0, 101)], [(-1, 4)], [(10, 20), (15, 30)], [(10, 20), (0, 5)], [(i, i + 1) for i in range(0, 18, 2)]])
def test_parts_refuse(parts):
    pt = np.array(parts, dtype=np.int64)
    rc = deft.lib().deft_layer_norms_part(A, A, 100, pt.ctypes.data, len(pt), A, 1, A, A, 1 << 30, None)
    assert rc == deft.ERR_INVALID_ARG
    rc = deft.lib().deft_layer_norms_part(A, A, 100, None, 1, A, 1, A, A, 1 << 30, None)
    assert rc == deft.ERR_INVALID_ARG
    h = np.zeros(64, dtype=np.int64).ctypes.data
    rc = deft.lib().deft_step_part(A, A, 100, pt.ctypes.data, len(pt), h, A, 1, 1, 1, 1, 0, 0, -1, A, h, h, ctypes.byref(ctypes.c_int64(0)), h, h, h,
                                   1 << 20, A, A, A, 10, A, 1 << 30, None, None)
    assert rc == deft.ERR_INVALID_ARG


def test_matrix_shapes_of_the_binding():
    import torch
    x = torch.zeros(4, 6, 8)
    assert deft._matrix(x, "x") == (24, 8, 8)
    assert deft._matrix(x[:, :, :5], "x") == (24, 5, 8)
    assert deft._matrix(x[:2, :, 1:4], "x") == (12, 3, 8)
    assert deft._matrix(x[:, 2:3, :5], "x") == (4, 5, 48)
    assert deft._matrix(x[0, 0], "x") == (1, 8, 8)
    for bad in (x[:, ::2, :5][:, :2], x.transpose(1, 2), x[:, :3, :5], x[:, :, ::2], torch.zeros(1, 8).expand(4, 8), torch.zeros(())):
        with pytest.raises(ValueError):
            deft._matrix(bad, "x")
    with pytest.raises(ValueError):
        deft._type(torch.zeros(1, dtype=torch.float64))
    for ids in (torch.zeros(4, dtype=torch.int16), torch.zeros(4, 4, dtype=torch.int64)[:, 1]):
        with pytest.raises(ValueError):
            deft._ids(ids)
    with pytest.raises(ValueError):
        deft._offset(torch.zeros(1))
    with pytest.raises(ValueError):
        deft._device(torch.zeros(1))


def test_workspace_serves_smaller_calls():
    """deft_embed_workspace_bytes does not fall with any of its arguments (small calls are split finer than large ones)."""
    rng = np.random.default_rng(0)
    for _ in range(3000):
        n, rows, width = (int(np.exp(rng.uniform(0, hi))) for hi in (14, 14.9, 9))
        most = deft.deft_embed_workspace_bytes(n, rows, width)
        less = [int(rng.integers(1, x + 1)) for x in (n, rows, width)]
        assert 0 < deft.deft_embed_workspace_bytes(*less) <= most
        assert deft.deft_embed_workspace_bytes(0, rows, width) <= most


def test_pitches_beyond_a_call():
    big = 2 ** 30
    assert _grad(ld=big) == _grad(width=big, ld=big) == deft.ERR_TOO_LARGE
    assert deft.deft_embed_workspace_bytes(5, 5, big) == 0
    assert _embed(ld_table=2 ** 60) == _embed(ld_out=2 ** 60) == _dropout(ld_x=2 ** 60) == deft.ERR_INVALID_ARG
