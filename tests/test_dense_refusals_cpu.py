"""Refusals of the dense row operators (C ABI, then binding) and the rotary frequencies.  Everything is refused on the host; the pointers
are never followed."""
import ctypes
import math

import numpy as np
import pytest
import torch

from paper_2307_03500_b200 import build as deft_build
from tests import dense_plain as plain

deft_build.build()
from paper_2307_03500_b200 import deft  # noqa: E402

A, B, C, D = 1 << 20, 1 << 28, 1 << 29, 1 << 30          # apart from one another
BAD, LARGE, CAPACITY = deft.ERR_INVALID_ARG, deft.ERR_TOO_LARGE, deft.ERR_CAPACITY
NAN, INF = float("nan"), float("inf")


def _norm(x=A, tx=0, ld_x=8, add=None, ld_add=8, sum=None, ld_sum=8, gamma=None, beta=None, tw=0, y=B, ty=0, ld_y=8, rows=4, cols=8, eps=1e-5, mean=None, rstd=None):
    return deft.lib().deft_layer_norm(x, tx, ld_x, add, ld_add, sum, ld_sum, gamma, beta, tw, y, ty, ld_y, rows, cols, eps, mean, rstd, None)


@pytest.mark.parametrize("kw,want", [
    (dict(tx=3), BAD), (dict(ty=-1), BAD), (dict(tw=7), BAD), (dict(rows=-1), BAD), (dict(cols=0), BAD), (dict(eps=-1e-9), BAD), (dict(eps=NAN), BAD),
    (dict(eps=INF), BAD), (dict(eps=1e39), BAD), (dict(x=None), BAD), (dict(y=None), BAD), (dict(x=A + 2), BAD), (dict(y=B + 1, ty=1), BAD), (dict(ld_x=7), BAD),
    (dict(ld_y=7), BAD), (dict(sum=C), BAD), (dict(add=D, ld_add=7), BAD), (dict(add=D, sum=C, ld_sum=7), BAD), (dict(gamma=C + 2), BAD), (dict(gamma=C + 1, tw=2), BAD),
    (dict(beta=C + 3), BAD), (dict(mean=C + 2), BAD), (dict(rstd=C + 1), BAD), (dict(cols=16385, ld_x=16385, ld_y=16385), LARGE), (dict(rows=2 ** 31), LARGE),
    (dict(y=A + 4), BAD), (dict(y=A, ty=1), BAD), (dict(y=A, ld_y=9), BAD), (dict(add=D, sum=A + 4), BAD), (dict(add=D, sum=D + 32), BAD), (dict(add=D, sum=C, y=C), BAD),
    (dict(add=D, sum=C, y=C + 4), BAD), (dict(add=D, y=D + 8), BAD), (dict(x=A, ld_x=2 ** 61), BAD),
    (dict(rows=0, x=None, y=None), deft.OK),
], ids=str)
def test_layer_norm(kw, want):
    assert _norm(**kw) == want


def _grad(dy=A, td=0, ld_dy=8, x=B, tx=0, ld_x=8, mean=A - 4096, rstd=A - 2048, gamma=None, tw=0, add=None, ld_add=8, gx=C, ld_gx=8, gg=D, gb=None, rows=4, cols=8, acc=0,
          scale=1.0, ws=D + 4096, ws_bytes=1 << 20):
    return deft.lib().deft_layer_norm_grad(dy, td, ld_dy, x, tx, ld_x, mean, rstd, gamma, tw, add, ld_add, gx, ld_gx, gg, gb, rows, cols, acc, scale, ws, ws_bytes, None)


@pytest.mark.parametrize("kw,want", [
    (dict(td=3), BAD), (dict(tx=3), BAD), (dict(tw=3), BAD), (dict(rows=-1), BAD), (dict(cols=0), BAD), (dict(dy=None), BAD), (dict(x=None), BAD), (dict(mean=None), BAD),
    (dict(rstd=None), BAD), (dict(gx=None, gg=None), BAD), (dict(ws=None), BAD), (dict(ws=D + 4096 + 128), BAD), (dict(ws_bytes=4 * 64 - 1), CAPACITY), (dict(scale=1e39), BAD),
    (dict(scale=NAN), BAD), (dict(gg=D + 2), BAD), (dict(gb=D + 1), BAD), (dict(gamma=D + 2), BAD), (dict(ld_dy=7), BAD), (dict(ld_x=7), BAD), (dict(ld_gx=7), BAD),
    (dict(add=A, ld_add=7), BAD), (dict(gx=A + 4), BAD), (dict(gx=A, td=1), BAD), (dict(gx=B + 8), BAD), (dict(gx=B, ld_gx=9), BAD), (dict(add=C + 4), BAD),
    (dict(cols=16385, ld_dy=16385, ld_x=16385, ld_gx=16385), LARGE), (dict(rows=2 ** 31), LARGE),
    (dict(rows=0, acc=1, dy=None, x=None, mean=None, rstd=None), deft.OK), (dict(rows=0, gg=None, ws=None, dy=None, x=None, gx=None), deft.OK),
], ids=str)
def test_layer_norm_grad(kw, want):
    assert _grad(**kw) == want


def test_layer_norm_workspace():
    size = deft.deft_layer_norm_workspace_bytes
    assert size(0, 5) > 0 and size(100, 1000) >= 100 * 8000
    assert size(-1, 5) == size(5, 0) == size(5, 16385) == size(2 ** 31, 5) == 0
    sizes = [[size(r, c) for c in (1, 7, 8, 100, 1027, 16384)] for r in (0, 1, 7, 9, 295, 296, 10 ** 6)]
    for rows in sizes:
        assert rows == sorted(rows)
    assert all(list(col) == sorted(col) for col in zip(*sizes)), "enough for fewer rows and columns"
    with pytest.raises(deft.DeftError):
        deft.alloc_layer_norm_workspace(5, 0, "cpu")


def _rotary(x=A, xs=(800, 80, 20), y=B, ys=(800, 80, 20), ty=0, batch=2, tokens=10, heads=4, dim=20, turns=C, rot=20, inter=0, inverse=0, gain=1.0, pos=None, pos_bytes=0):
    s = [None if v is None else (ctypes.c_int64 * 3)(*v) for v in (xs, ys)]
    return deft.lib().deft_rotary(x, s[0], y, s[1], ty, batch, tokens, heads, dim, turns, rot, inter, inverse, gain, pos, pos_bytes, None)


@pytest.mark.parametrize("kw,want", [
    (dict(ty=3), BAD), (dict(batch=-1), BAD), (dict(tokens=-1), BAD), (dict(heads=-1), BAD), (dict(dim=0), BAD), (dict(rot=0), BAD), (dict(rot=5), BAD), (dict(rot=22), BAD),
    (dict(gain=1e39), BAD), (dict(gain=NAN), BAD), (dict(xs=None), BAD), (dict(ys=None), BAD), (dict(x=None), BAD), (dict(y=None), BAD), (dict(turns=None), BAD), (dict(turns=C + 4), BAD),
    (dict(x=A + 2), BAD), (dict(pos=D, pos_bytes=2), BAD), (dict(pos=D + 4, pos_bytes=8), BAD), (dict(xs=(-800, 80, 20)), BAD), (dict(ys=(800, 80, 19)), BAD), (dict(ys=(800, 0, 20)), BAD),
    (dict(ys=(800, 79, 20)), BAD), (dict(ys=(799, 80, 20)), BAD), (dict(ys=(2 ** 60, 80, 20)), BAD), (dict(y=A + 4), BAD), (dict(y=A, ys=(800, 80, 21)), BAD), (dict(y=A + 80 * 4), BAD),
    (dict(y=A + 6396), BAD), (dict(y=A - 4 * 20), BAD), (dict(y=A, xs=(800, 80, 0)), BAD), (dict(xs=(8000, 800, 40), ys=(8000, 800, 40), y=A + 4 * 30), BAD),
    (dict(xs=(8000, 800, 40), ys=(8000, 800, 40), y=A + 4 * 781), BAD), (dict(tokens=2 ** 31), LARGE), (dict(batch=2 ** 16, tokens=2 ** 16), LARGE), (dict(heads=2 ** 30), LARGE),
    (dict(dim=2 ** 31, rot=2), LARGE), (dict(dim=5000, rot=4098), LARGE),
    (dict(batch=0, x=None, y=None), deft.OK), (dict(tokens=0, x=None, y=None), deft.OK), (dict(heads=0), deft.OK),
], ids=str)
def test_rotary(kw, want):
    assert _rotary(**kw) == want


def _distill(z=A, ty=0, ld=8, rows=4, vocab=8, ids=C, id_bytes=8, ld_ids=3, teacher=D, tt=0, ld_t=3, top=3, lse=None, temp=1.0, weight=None, scale=1.0, loss=A - 4096, grad=B, ld_g=8):
    return deft.lib().deft_distill(z, ty, ld, rows, vocab, ids, id_bytes, ld_ids, teacher, tt, ld_t, top, lse, temp, weight, scale, loss, grad, ld_g, None)


@pytest.mark.parametrize("kw,want", [
    (dict(ty=3), BAD), (dict(tt=3), BAD), (dict(rows=-1), BAD), (dict(vocab=0), BAD), (dict(top=0), BAD), (dict(id_bytes=2), BAD), (dict(temp=0.0), BAD), (dict(temp=-1.0), BAD),
    (dict(temp=NAN), BAD), (dict(temp=INF), BAD), (dict(temp=1e7), BAD), (dict(temp=1e-7), BAD), (dict(scale=1e39), BAD), (dict(scale=NAN), BAD), (dict(scale=1e38, temp=100.0), BAD),
    (dict(loss=None, grad=None), BAD), (dict(z=None), BAD), (dict(ids=None), BAD), (dict(teacher=None), BAD), (dict(ids=C + 4), BAD), (dict(teacher=D + 2), BAD), (dict(z=A + 2), BAD),
    (dict(ld=7), BAD), (dict(ld_ids=2), BAD), (dict(ld_t=2), BAD), (dict(ld_g=7), BAD), (dict(lse=C + 2), BAD), (dict(weight=C + 1), BAD), (dict(loss=A - 2), BAD), (dict(grad=A + 4), BAD),
    (dict(grad=A, ld_g=9), BAD), (dict(grad=A + 96), BAD), (dict(rows=2 ** 28), LARGE), (dict(vocab=262145, ld=262145, ld_g=262145), LARGE), (dict(top=1025, ld_ids=1025, ld_t=1025), LARGE),
    (dict(rows=0, z=None, ids=None, teacher=None, loss=None, grad=None), deft.OK),
], ids=str)
def test_distill(kw, want):
    assert _distill(**kw) == want


@pytest.mark.parametrize("kw,want", [
    (dict(rot=0), BAD), (dict(rot=7), BAD), (dict(rot=-2), BAD), (dict(base=0.5), BAD), (dict(base=NAN), BAD), (dict(base=INF), BAD), (dict(scaling=4), BAD), (dict(scaling=-1), BAD),
    (dict(scaling=1, factor=0.0), BAD), (dict(scaling=2, factor=NAN), BAD), (dict(scaling=3, original=0.0), BAD), (dict(scaling=3, low=32.0), BAD), (dict(scaling=3, high=INF), BAD),
    (dict(turns=None), BAD), (dict(rot=4098), LARGE), (dict(scaling=0, factor=NAN, original=NAN, low=NAN, high=NAN), deft.OK), (dict(scaling=1, original=NAN), deft.OK),
], ids=str)
def test_frequencies_refused(kw, want):
    a = dict(rot=8, base=10000.0, scaling=0, factor=2.0, original=2048.0, low=1.0, high=32.0, turns=np.zeros(4096, dtype=np.int64))
    a.update(kw)
    turns = a.pop("turns")
    assert deft.lib().deft_rotary_frequencies(*a.values(), None if turns is None else turns.ctypes.data) == want


@pytest.mark.parametrize("rot", [2, 4, 10, 64, 128, 4096])
@pytest.mark.parametrize("kw", [dict(), dict(base=500000.0), dict(base=1.0), dict(scaling="linear", factor=4.0), dict(scaling="linear", factor=0.01), dict(scaling="base", factor=16.0),
                                dict(scaling="parts", factor=8.0, original=2048.0), dict(scaling="parts", factor=32.0, original=8192.0, low=1.0, high=4.0)], ids=str)
def test_frequencies(rot, kw):
    got = deft.deft_rotary_frequencies(rot, **kw).view(np.uint64).astype(np.float64) * 2.0 ** -64
    want = np.mod(plain.frequencies(rot, **kw) / (2.0 * math.pi), 1.0)
    # the 64-bit powers are off by a few units in the last place times their exponents (up to ln(base factor^..) = 15)
    assert np.all(np.abs(got - want) <= 64 * 2.0 ** -53 * np.maximum(want, plain.frequencies(rot, **kw) / (2.0 * math.pi)) + 2.0 ** -64)


def test_binding_refuses():
    """Shapes and types that disagree, before anything is launched (on CPU tensors at the latest by their device)."""
    x, w = torch.zeros(4, 8), torch.zeros(8)
    s = torch.zeros(4)
    ids, t = torch.zeros(4, 3, dtype=torch.int64), torch.zeros(4, 3)
    turns = torch.zeros(4, dtype=torch.int64)
    for call in [
        lambda: deft.deft_layer_norm(x, x[:3]), lambda: deft.deft_layer_norm(x, x.t()), lambda: deft.deft_layer_norm(x, x, gamma=w[:7]), lambda: deft.deft_layer_norm(x, x, gamma=w, beta=w.half()),
        lambda: deft.deft_layer_norm(x, x, add=x.half()), lambda: deft.deft_layer_norm(x, x, add=x, sum=x[:2]), lambda: deft.deft_layer_norm(x, x, mean=s[:3]),
        lambda: deft.deft_layer_norm(x, x, rstd=s.double()), lambda: deft.deft_layer_norm(x.double(), x), lambda: deft.deft_layer_norm(x, x),
        lambda: deft.deft_layer_norm_grad(x[:3], x, s, s, x), lambda: deft.deft_layer_norm_grad(x, x, s[:2], s, x), lambda: deft.deft_layer_norm_grad(x, x, s, s, x.half()),
        lambda: deft.deft_layer_norm_grad(x, x, s, s, x, add=x.half()), lambda: deft.deft_layer_norm_grad(x, x, s, s, grad_gamma=w[:7]),
        lambda: deft.deft_layer_norm_grad(x, x, s, s, grad_gamma=w.half()), lambda: deft.deft_layer_norm_grad(x, x, s, s, x, ws=x.t()), lambda: deft.deft_layer_norm_grad(x, x, s, s, x),
        lambda: deft.deft_rotary(x, x, turns), lambda: deft.deft_rotary(x.view(2, 2, 8), x.view(4, 1, 8), turns), lambda: deft.deft_rotary(x.view(2, 2, 8), x.view(2, 2, 8).half(), turns),
        lambda: deft.deft_rotary(x.view(2, 2, 8).transpose(1, 2), x.view(2, 2, 8).transpose(1, 2), turns), lambda: deft.deft_rotary(x.view(2, 2, 8), x.view(2, 2, 8), turns.float()),
        lambda: deft.deft_rotary(x.view(2, 2, 8), x.view(2, 2, 8), turns, positions=ids[:3, 0]), lambda: deft.deft_rotary(x.view(2, 2, 8), x.view(2, 2, 8), turns, positions=s[:2]),
        lambda: deft.deft_rotary(x.view(2, 2, 8), x.view(2, 2, 8), turns), lambda: deft.deft_rotary_frequencies(8, scaling="other"),
        lambda: deft.deft_distill(x, ids[:3], t, loss=s), lambda: deft.deft_distill(x, ids, t[:, :2], loss=s), lambda: deft.deft_distill(x, ids.float(), t, loss=s),
        lambda: deft.deft_distill(x, ids, t, loss=s[:3]), lambda: deft.deft_distill(x, ids, t, grad=x.half()), lambda: deft.deft_distill(x, ids, t, loss=s, teacher_lse=s[:3]),
        lambda: deft.deft_distill(x, ids, t, loss=s, weight=s.double()), lambda: deft.deft_distill(x, ids, t.double(), loss=s), lambda: deft.deft_distill(x, ids, t, loss=s),
    ]:
        with pytest.raises(ValueError):
            call()
    for rot in (0, 3, 5000):
        with pytest.raises(deft.DeftError):
            deft.deft_rotary_frequencies(rot)
