"""Layer norm and its gradient against the definition in 64 bits: sizes, types, strides, rows far from zero, in place."""
import pytest
import torch

from paper_2307_03500_b200 import build as deft_build
from tests import dense_plain as plain

deft_build.build()
from paper_2307_03500_b200 import deft  # noqa: E402

pytestmark = pytest.mark.gpu
F32, BF16, F16 = torch.float32, torch.bfloat16, torch.float16


def _rand(shape, dtype, seed, std=1.0, mean=0.0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return torch.empty(shape, device="cuda").normal_(mean, std, generator=g).to(dtype)


def _strided(t, pad, offset):
    """The same values in rows of a wider buffer, `offset` elements in, and the buffer."""
    buf = torch.full((t.shape[0] * (t.shape[1] + pad) + offset + 8,), 7.0, dtype=t.dtype, device=t.device)
    view = buf[offset:offset + t.shape[0] * (t.shape[1] + pad)].view(t.shape[0], t.shape[1] + pad)[:, :t.shape[1]]
    view.copy_(t)
    return view, buf


def _forward(x, y_dtype, add=None, gamma=None, beta=None, eps=1e-5, keep_sum=True):
    rows = x.shape[0]
    y = torch.full(x.shape, 9.0, dtype=y_dtype, device="cuda")
    s = torch.full(x.shape, 9.0, dtype=x.dtype, device="cuda") if add is not None and keep_sum else None
    mean, rstd = torch.full((rows,), 9.0, device="cuda"), torch.full((rows,), 9.0, device="cuda")
    deft.deft_layer_norm(x, y, gamma, beta, eps=eps, add=add, sum=s, mean=mean, rstd=rstd)
    want, want_s, m, r, tol, tol_m, tol_r = plain.layer_norm(x, add, gamma, beta, eps)
    plain.close(y, want, tol)
    plain.close(mean, m, tol_m)
    plain.close(rstd, r, tol_r)
    if s is not None:
        plain.close(s, want_s, plain.U * want_s.abs())
    return y, s, mean, rstd


@pytest.mark.parametrize("rows,cols", [(1, 1), (3, 2), (1, 7), (5, 8), (2, 31), (9, 64), (17, 100), (33, 250), (64, 256), (700, 257), (5, 1000), (300, 1024),
                                       (37, 1027), (20, 1500), (3000, 48), (11, 2049), (4, 4099), (3, 8184), (3, 8192), (2, 16381), (2, 16384), (3, 16384), (600, 8192), (1300, 72)])
@pytest.mark.parametrize("xt,yt", [(BF16, BF16), (F32, BF16), (F16, F32)])
def test_sizes(rows, cols, xt, yt):
    x, add = _rand((rows, cols), xt, 1, 2.0, 0.5), _rand((rows, cols), xt, 2)
    gamma, beta = _rand((cols,), F32, 3, 0.3, 1.0), _rand((cols,), F32, 4)
    _forward(x, yt, add if rows % 2 else None, gamma, beta)


@pytest.mark.parametrize("xt", [F32, BF16, F16])
@pytest.mark.parametrize("yt", [F32, BF16, F16])
@pytest.mark.parametrize("wt", [F32, BF16, F16, None])
def test_types(xt, yt, wt):
    x, add = _rand((40, 515), xt, 1), _rand((40, 515), xt, 2)
    gamma = None if wt is None else _rand((515,), wt, 3, 0.3, 1.0)
    beta = None if wt in (None, F16) else _rand((515,), wt, 4)
    _forward(x, yt, add, gamma, beta, keep_sum=yt != F16)


@pytest.mark.parametrize("mean,std", [(1e4, 1.0), (-300.0, 1e-2), (0.0, 1e-6), (5.0, 0.0)])
def test_rows_far_from_zero(mean, std):
    """The mean's own rounding is taken out: nothing is lost however far the row lies from zero."""
    _forward(_rand((50, 700), F32, 5, std, mean), F32, eps=1e-12)


def test_constant_and_non_finite_rows():
    x = torch.ones((6, 300), device="cuda")
    x[1, 7], x[2, 0], x[3, 299] = float("nan"), float("inf"), float("-inf")
    x[4] = 0.0
    y = torch.empty_like(x)
    deft.deft_layer_norm(x, y)
    assert torch.equal(y[0], torch.zeros(300, device="cuda")) and torch.equal(y[4], y[0]) and torch.equal(y[5], y[0])
    assert torch.isnan(y[1:4]).all()


@pytest.mark.parametrize("pad,offset", [(0, 0), (8, 0), (3, 0), (0, 1), (5, 3), (4, 4)])
@pytest.mark.parametrize("same", [True, False])
def test_strides(pad, offset, same):
    """Rows of wider buffers, all matrices alike (one shift serves them) or each on its own; what lies beside the rows stays."""
    x, add = _rand((29, 333), BF16, 6), _rand((29, 333), BF16, 7)
    (xs, _), (adds, _) = _strided(x, pad, offset), _strided(add, pad, offset if same else 0)
    y, y_buf = _strided(torch.zeros_like(x), pad if same else 16, offset)
    s, s_buf = _strided(torch.zeros_like(x), pad, offset if same else 2)
    deft.deft_layer_norm(xs, y, add=adds, sum=s)
    want, want_s, _, _, tol, _, _ = plain.layer_norm(x, add)
    plain.close(y, want, tol)
    plain.close(s, want_s, plain.U * want_s.abs())
    for view, buf in ((y, y_buf), (s, s_buf)):
        view.fill_(7.0)
        assert (buf == 7.0).all(), "written beside the rows"


def test_in_place_and_none():
    x, add = _rand((130, 771), BF16, 8), _rand((130, 771), BF16, 9)
    want, want_s, _, _, tol, _, _ = plain.layer_norm(x, add)
    stream, branch = x.clone(), add.clone()
    deft.deft_layer_norm(stream, branch, add=branch, sum=stream)         # the sum in the stream's place, y in the branch's
    plain.close(branch, want, tol)
    plain.close(stream, want_s, plain.U * want_s.abs())
    y = x.clone()
    deft.deft_layer_norm(y, y)
    plain.close(y, plain.layer_norm(x)[0], plain.layer_norm(x)[4])
    empty = torch.empty((0, 5), device="cuda")
    deft.deft_layer_norm(empty, empty.clone())
    # three dimensions are a list of rows
    x3, y3 = x[:128].view(4, 32, 771), torch.empty((4, 32, 771), dtype=F32, device="cuda")
    deft.deft_layer_norm(x3, y3)
    plain.close(y3.view(-1, 771), plain.layer_norm(x[:128])[0], plain.layer_norm(x[:128])[4])


def _backward(dy, x, gamma=None, add=None, scale=1.0, accumulate=False, want_x=True, want_w=True, ws_rows=None):
    rows, cols = x.shape
    _, _, mean, rstd, *_ = plain.layer_norm(x)
    mean, rstd = mean.float(), rstd.float()
    gx = torch.full(x.shape, 9.0, dtype=x.dtype, device="cuda") if want_x else None
    flat = _rand((2 * cols,), F32, 11)
    before = flat.clone()
    ws = deft.alloc_layer_norm_workspace(ws_rows or rows, cols) if want_w else None
    if ws is not None:
        ws.fill_(255)
    deft.deft_layer_norm_grad(dy, x, mean, rstd, gx, gamma, add=add, grad_gamma=flat[:cols] if want_w else None,
                              grad_beta=flat[cols:] if want_w else None, ws=ws, accumulate=accumulate, scale=scale)
    dx, dg, db, tol, tol_g, tol_b = plain.layer_norm_grad(dy, x, mean, rstd, gamma, add, scale)
    if want_x:
        plain.close(gx, dx, tol)
    if want_w:
        old = before.double() if accumulate else torch.zeros(2 * cols, dtype=torch.float64, device="cuda")
        plain.close(flat[:cols], dg + old[:cols], tol_g + plain.U * old[:cols].abs())
        plain.close(flat[cols:], db + old[cols:], tol_b + plain.U * old[cols:].abs())
    else:
        assert torch.equal(flat, before)
    return gx, flat


@pytest.mark.parametrize("rows,cols", [(1, 1), (3, 2), (1, 7), (5, 8), (2, 31), (9, 64), (17, 100), (700, 257), (5, 1000), (600, 1024), (37, 1027),
                                       (700, 1500), (9000, 48), (3000, 16), (11, 2049), (30, 4099), (3, 8184), (3, 8192), (2, 16381), (20, 16384), (3, 16384), (600, 8192), (33, 520), (90, 1030)])
@pytest.mark.parametrize("dt,xt", [(BF16, BF16), (F32, F32), (F16, F32), (BF16, F16)])
def test_gradient_sizes(rows, cols, dt, xt):
    x, add = _rand((rows, cols), xt, 1, 2.0, 0.5), _rand((rows, cols), xt, 2)
    _backward(_rand((rows, cols), dt, 3), x, _rand((cols,), F32, 4, 0.3, 1.0), add if rows % 2 else None, accumulate=cols % 2 == 0)


@pytest.mark.parametrize("kw", [dict(want_x=False), dict(want_w=False), dict(scale=-0.37, accumulate=True), dict(ws_rows=100000)],
                         ids=lambda kw: ",".join(kw))
def test_gradient_parts(kw):
    x = _rand((77, 650), BF16, 1)
    _backward(_rand((77, 650), BF16, 3), x, _rand((650,), BF16, 4, 0.3, 1.0), None, **kw)


def test_gradient_only_gamma_or_beta_and_no_rows():
    x, dy = _rand((40, 90), F32, 1), _rand((40, 90), F32, 2)
    _, _, mean, rstd, *_ = plain.layer_norm(x)
    mean, rstd = mean.float(), rstd.float()
    ws = deft.alloc_layer_norm_workspace(40, 90)
    both, one = torch.empty(180, device="cuda"), torch.full((180,), 3.0, device="cuda")
    deft.deft_layer_norm_grad(dy, x, mean, rstd, grad_gamma=both[:90], grad_beta=both[90:], ws=ws)
    deft.deft_layer_norm_grad(dy, x, mean, rstd, grad_gamma=one[:90], ws=ws)
    assert torch.equal(one[:90], both[:90]) and (one[90:] == 3.0).all()
    deft.deft_layer_norm_grad(dy, x, mean, rstd, grad_beta=one[90:], ws=ws)
    assert torch.equal(one, both)
    none = torch.empty((0, 90), device="cuda")
    deft.deft_layer_norm_grad(none, none, none[:, 0], none[:, 0], grad_gamma=one[:90], grad_beta=one[90:], ws=ws, accumulate=True)
    assert torch.equal(one, both)
    deft.deft_layer_norm_grad(none, none, none[:, 0], none[:, 0], grad_gamma=one[:90], grad_beta=one[90:], ws=ws)
    assert not one.any()


def test_gradient_in_place_same_bits_and_unequal_strides():
    x, dy, add = (_rand((501, 1030), BF16, s) for s in (1, 2, 3))
    gamma = _rand((1030,), F32, 4, 0.3, 1.0)
    gx, flat = _backward(dy, x, gamma, add)
    _, _, mean, rstd, *_ = plain.layer_norm(x)
    mean, rstd = mean.float(), rstd.float()
    ws = deft.alloc_layer_norm_workspace(501, 1030)
    for place in range(3):
        t = [dy.clone(), x.clone(), add.clone()]
        w = torch.empty(2060, device="cuda")
        deft.deft_layer_norm_grad(t[0], t[1], mean, rstd, t[place], gamma, add=t[2], grad_gamma=w[:1030], grad_beta=w[1030:], ws=ws)
        assert torch.equal(t[place], gx) and torch.equal(w, flat), "other bits"
    out, buf = _strided(torch.zeros_like(x), 11, 5)
    w = torch.empty(2060, device="cuda")
    deft.deft_layer_norm_grad(_strided(dy, 2, 1)[0], x, mean, rstd, out, gamma, add=_strided(add, 8, 0)[0], grad_gamma=w[:1030], grad_beta=w[1030:], ws=ws)
    dx, dg, db, tol, tol_g, tol_b = plain.layer_norm_grad(dy, x, mean, rstd, gamma, add)
    plain.close(out, dx, tol)
    plain.close(w, torch.cat([dg, db]), torch.cat([tol_g, tol_b]))
    out.fill_(7.0)
    assert (buf == 7.0).all()


def test_gradient_against_differences():
    """The formula itself: central differences of the definition in 64 bits."""
    x, dy, gamma, beta = _rand((3, 20), F32, 1), _rand((3, 20), F32, 2), _rand((20,), F32, 3, 0.3, 1.0), _rand((20,), F32, 4)
    _, _, mean, rstd, *_ = plain.layer_norm(x)
    gx, gw = torch.empty_like(x), torch.empty(40, device="cuda")
    deft.deft_layer_norm_grad(dy, x, mean.float(), rstd.float(), gx, gamma, grad_gamma=gw[:20], grad_beta=gw[20:], ws=deft.alloc_layer_norm_workspace(3, 20))

    def value(x, g, b):
        return (plain.layer_norm(x, None, g, b)[0] * dy.double()).sum().item()
    step = 1e-5
    args = [x.double(), gamma.double(), beta.double()]
    for which, got in ((0, gx), (1, gw[:20]), (2, gw[20:])):
        for i in range(0, got.numel(), 7):
            moved = []
            for sign in (1, -1):
                a = [t.clone() for t in args]
                a[which].view(-1)[i] += sign * step
                moved.append(value(*a))
            # the third derivative times step^2 / 6 and 64-bit roundings over the step: below 1e-6; the fp32 result 1e-5
            assert abs((moved[0] - moved[1]) / (2 * step) - got.reshape(-1)[i].item()) < 2e-5
