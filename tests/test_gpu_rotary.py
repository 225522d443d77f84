"""Rotary positions against the definition: layouts, parts of heads, strides, far and negative positions, in place, gradient."""
import numpy as np
import pytest
import torch

from paper_2307_03500_b200 import build as deft_build
from tests import dense_plain as plain

deft_build.build()
from paper_2307_03500_b200 import deft  # noqa: E402

pytestmark = pytest.mark.gpu
F32, BF16, F16 = torch.float32, torch.bfloat16, torch.float16


def _rand(shape, dtype, seed):
    return torch.empty(shape, device="cuda").normal_(generator=torch.Generator(device="cuda").manual_seed(seed)).to(dtype)


def _check(x, rot, y=None, positions=None, **kw):
    freq = {k: kw.pop(k) for k in ("base", "scaling", "factor", "original") if k in kw}
    turns = deft.deft_rotary_frequencies(rot, **freq)
    y = torch.full(x.shape, 9.0, dtype=x.dtype, device="cuda") if y is None else y
    before = x.clone()
    deft.deft_rotary(x, y, torch.from_numpy(turns).cuda(), positions=positions, **kw)
    pos = torch.arange(x.shape[-3], device="cuda").expand(x.shape[:-2]) if positions is None else positions.long()
    want, tol = plain.rotary(before, turns, pos, **kw)
    plain.close(y, want, tol)
    return y


@pytest.mark.parametrize("heads,dim,rot", [(1, 2, 2), (3, 8, 4), (2, 16, 16), (5, 64, 64), (4, 128, 32), (3, 80, 40), (7, 66, 66), (1, 13, 6), (2, 100, 50),
                                           (12, 160, 24), (1, 5000, 4096)])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("dtype", [BF16, F32, F16])
def test_shapes(heads, dim, rot, interleaved, dtype):
    _check(_rand((2, 5, heads, dim), dtype, 1), rot, interleaved=interleaved)


@pytest.mark.parametrize("batch,tokens", [(1, 1), (1, 700), (64, 1), (3, 333), (700, 2)])
def test_tokens(batch, tokens):
    _check(_rand((batch, tokens, 6, 64), BF16, 2), 64)
    _check(_rand((batch * tokens, 6, 64), BF16, 2), 64, inverse=True)


@pytest.mark.parametrize("pos_type", [torch.int64, torch.int32])
def test_positions(pos_type):
    """Far ones as exact as near ones; negative ones; in any order."""
    p = [0, 1, -1, 4095, 131071, 2 ** 24 + 1, 2 ** 31 - 1, -2 ** 31] + ([2 ** 53 + 1, -2 ** 63, 2 ** 63 - 1] if pos_type == torch.int64 else [])
    pos = torch.tensor(p, dtype=pos_type, device="cuda")
    x = _rand((len(p), 4, 32), F32, 3)
    _check(x, 32, positions=pos)
    _check(x, 32, positions=pos, interleaved=True, inverse=True, gain=1.25)


@pytest.mark.parametrize("scaling", ["plain", "linear", "base", "parts"])
def test_scaled(scaling):
    _check(_rand((40, 4, 48), F32, 4), 48, scaling=scaling, factor=8.0, original=2048.0, gain=0.7)


@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("offset,wide", [(0, 200), (1, 200), (4, 203), (2, 128)])
def test_strides_and_what_lies_beside(interleaved, offset, wide):
    """Heads inside a fused projection, columns at odd places; what lies beside the heads stays."""
    buf = _rand((2, 9, 5, wide + 8), BF16, 5)
    x = buf[:, :, 1:4, offset:offset + 96]
    out = torch.full((9, 2, 6, wide), 7.0, dtype=BF16, device="cuda")
    y = out.transpose(0, 1)[:, :, 2:5, :96]
    _check(x, 64, y=y, interleaved=interleaved)
    y.fill_(7.0)
    assert (out == 7.0).all()
    # [batch, heads, tokens, dim] storage
    x = _rand((2, 3, 17, 40), BF16, 6).transpose(1, 2)
    _check(x, 40, y=torch.empty((2, 3, 17, 40), dtype=BF16, device="cuda").transpose(1, 2), interleaved=interleaved)


@pytest.mark.parametrize("interleaved", [False, True])
def test_in_place_repeated_heads_and_nothing(interleaved):
    fused = _rand((2, 50, 9, 72), BF16, 7)
    want = fused.clone()
    _check(fused[:, :, :6], 48, y=fused[:, :, :6], interleaved=interleaved)
    assert torch.equal(fused[:, :, 6:], want[:, :, 6:]) and torch.equal(fused[..., 48:], want[..., 48:])
    _check(_rand((2, 50, 1, 72), BF16, 8).expand(2, 50, 4, 72), 72, interleaved=interleaved)
    empty = torch.empty((0, 3, 8), device="cuda")
    deft.deft_rotary(empty, empty.clone(), torch.from_numpy(deft.deft_rotary_frequencies(8)).cuda())


def test_gradient_is_the_inverse_rotation():
    """<R x, dy> = <x, R' dy>, and the inverse undoes the rotation."""
    x, dy = _rand((2, 70, 3, 40), F32, 9), _rand((2, 70, 3, 40), F32, 10)
    turns = torch.from_numpy(deft.deft_rotary_frequencies(24)).cuda()
    y, dx, back = torch.empty_like(x), torch.empty_like(x), torch.empty_like(x)
    deft.deft_rotary(x, y, turns, gain=1.5)
    deft.deft_rotary(dy, dx, turns, gain=1.5, inverse=True)
    a, b = (y.double() * dy.double()).sum(), (x.double() * dx.double()).sum()
    assert abs(a - b) <= 16 * plain.U * (y.double() * dy.double()).abs().sum()
    deft.deft_rotary(y, back, turns, gain=1 / 1.5, inverse=True)
    want = x.double()
    plain.close(back, want, 32 * plain.U * (want.abs() + want.abs().amax(-1, keepdim=True)))


def test_relative_positions():
    """Products of rotated queries and keys depend on distances alone, far out too."""
    q, k = _rand((1, 1, 64), F32, 11), _rand((1, 1, 64), F32, 12)
    turns = torch.from_numpy(deft.deft_rotary_frequencies(64)).cuda()
    dots = []
    for start in (0, 1000, 2 ** 40):
        a, b = torch.empty_like(q), torch.empty_like(k)
        deft.deft_rotary(q, a, turns, positions=torch.tensor([start + 37], device="cuda"))
        deft.deft_rotary(k, b, turns, positions=torch.tensor([start], device="cuda"))
        dots.append((a.double() * b.double()).sum().item())
    size = (q.double().abs().sum() * k.double().abs().max()).item()
    assert np.ptp(dots) <= 32 * plain.U * size
