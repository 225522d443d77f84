"""Dense row operators at the edges of rows and calls: what lies beside a row, lanes without work, rows that share a warp."""
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


def _placed(t, pad, offset, fill):
    """The same values in rows of a wider buffer, `offset` elements in; everything beside them is `fill`."""
    rows, cols = t.shape
    buf = torch.full((rows * (cols + pad) + offset + 8,), fill, dtype=t.dtype, device=t.device)
    return buf[offset:offset + rows * (cols + pad)].view(rows, cols + pad)[:, :cols].copy_(t)


def _norm(x, add=None, gamma=None):
    rows, cols = x.shape
    y, s = _placed(torch.zeros_like(x), x.stride(0) - cols, x.storage_offset(), 7.0), None
    if add is not None:
        s = _placed(torch.zeros_like(x), x.stride(0) - cols, x.storage_offset(), 7.0)
    mean, rstd = torch.empty(rows, device="cuda"), torch.empty(rows, device="cuda")
    deft.deft_layer_norm(x, y, gamma, add=add, sum=s, mean=mean, rstd=rstd)
    return y, s, mean, rstd


def _grad(dy, x, mean, rstd, gamma=None, add=None, grad_x=None, **kw):
    rows, cols = x.shape
    if grad_x is None:
        grad_x = _placed(torch.zeros_like(x), x.stride(0) - cols, x.storage_offset(), 7.0)
    w = torch.empty(2 * cols, device="cuda")
    deft.deft_layer_norm_grad(dy, x, mean, rstd, grad_x, gamma, add=add, grad_gamma=w[:cols], grad_beta=w[cols:], ws=deft.alloc_layer_norm_workspace(rows, cols), **kw)
    return grad_x, w


@pytest.mark.parametrize("offset", range(1, 8))
@pytest.mark.parametrize("rows,cols", [(29, 333), (3, 20), (700, 9)])
@pytest.mark.parametrize("dtype", [BF16, F32])
def test_lanes_without_columns(rows, cols, offset, dtype):
    """Teams with more threads than a row has groups, in matrices that begin at any place of a granule."""
    x, add, dy = (_placed(_rand((rows, cols), dtype, s), 0, offset, 7.0) for s in (1, 2, 3))
    y, s, mean, rstd = _norm(x, add)
    want, want_s, m, r, tol, tol_m, tol_r = plain.layer_norm(x, add)
    plain.close(y, want, tol)
    plain.close(s, want_s, plain.U * want_s.abs())
    plain.close(mean, m, tol_m)
    plain.close(rstd, r, tol_r)
    _, _, m, r, *_ = plain.layer_norm(x)
    dx, w = _grad(dy, x, m.float(), r.float(), add=add)
    want, dg, db, tol, tol_g, tol_b = plain.layer_norm_grad(dy, x, m.float(), r.float(), None, add)
    plain.close(dx, want, tol)
    plain.close(w, torch.cat([dg, db]), torch.cat([tol_g, tol_b]))


BAD = [float("nan"), float("inf"), -float("inf")]


@pytest.mark.parametrize("bad", BAD)
@pytest.mark.parametrize("rows", [9, 700])             # one cluster, partial sums
@pytest.mark.parametrize("cols", [1027, 99, 1500])
@pytest.mark.parametrize("dt,xt", [(BF16, BF16), (F32, F32), (F16, F32)])
def test_a_bad_row_spoils_no_other_gradient(bad, rows, cols, dt, xt):
    """The last elements of a row share a granule with the next row's first ones: every other row keeps its bits."""
    dy, x, add = _rand((rows, cols), dt, 1), _rand((rows, cols), xt, 2, 2.0, 0.5), _rand((rows, cols), xt, 3)
    gamma = _rand((cols,), F32, 4, 0.3, 1.0)
    _, _, mean, rstd, *_ = plain.layer_norm(x)
    mean, rstd = mean.float(), rstd.float()
    clean, w = _grad(dy, x, mean, rstd, gamma, add)
    others = torch.arange(rows, device="cuda") != 4
    for t in (dy, x, add):
        kept = t[4].clone()
        t[4, -3:] = bad
        got, w_got = _grad(dy, x, mean, rstd, gamma, add)
        t[4] = kept
        assert torch.equal(got[others], clean[others])
        assert torch.equal(w_got[:cols - 3], w[:cols - 3]) and torch.equal(w_got[cols:-3], w[cols:-3])


@pytest.mark.parametrize("bad", BAD)
@pytest.mark.parametrize("rows", [9, 700])
@pytest.mark.parametrize("pad,offset", [(0, 1), (8, 2), (16, 3), (8, 4), (3, 5), (8, 6), (9, 7), (5, 0)])
@pytest.mark.parametrize("dtype", [BF16, F32])
def test_what_lies_beside_the_rows(bad, rows, pad, offset, dtype):
    """Norm and gradient of columns of a wider buffer: the bits do not depend on what the buffer holds beside them."""
    cols = 331
    x, add, dy = (_rand((rows, cols), dtype, s) for s in (1, 2, 3))
    gamma = _rand((cols,), F32, 4, 0.3, 1.0)

    def both(fill):
        xs, adds, dys = (_placed(t, pad, offset, fill) for t in (x, add, dy))
        y, s, mean, rstd = _norm(xs, adds, gamma)
        return [y, s, mean, rstd] + list(_grad(dys, xs, mean, rstd, gamma, adds))
    clean, got = both(0.0), both(bad)
    assert all(torch.isfinite(t).all() for t in clean) and all(torch.equal(a, b) for a, b in zip(got, clean))


@pytest.mark.parametrize("bad", BAD)
@pytest.mark.parametrize("dtype", [BF16, F32])
def test_gradient_beside_its_input(bad, dtype):
    """x and grad_x as columns of one buffer, which nobody has written yet."""
    rows, cols = 70, 328
    x, dy = _rand((rows, cols), dtype, 1), _rand((rows, cols), dtype, 2)
    _, _, mean, rstd, *_ = plain.layer_norm(x)
    mean, rstd = mean.float(), rstd.float()
    buf = torch.full((rows, 2 * cols + 8), bad, dtype=dtype, device="cuda")
    gx, xs = buf[:, 3:3 + cols], buf[:, 3 + cols:3 + 2 * cols]
    xs.copy_(x)
    dys = _placed(dy, cols + 8, 3, bad)
    got, w = _grad(dys, xs, mean, rstd, grad_x=gx)
    want, dg, db, tol, tol_g, tol_b = plain.layer_norm_grad(dy, x, mean, rstd)
    plain.close(got, want, tol)
    plain.close(w, torch.cat([dg, db]), torch.cat([tol_g, tol_b]))
    assert torch.equal(xs, x)


@pytest.mark.parametrize("bad", BAD)
@pytest.mark.parametrize("pad,offset", [(0, 1), (3, 3), (8, 7)])
def test_distillation_and_rotary_beside_bad_numbers(bad, pad, offset):
    rows, vocab = 5, 2003
    z = _rand((rows, vocab), BF16, 1)
    t, ids = _rand((rows, vocab), F32, 2).topk(6, dim=1)
    lse = t.logsumexp(1) + 0.5
    turns = torch.from_numpy(deft.deft_rotary_frequencies(60)).cuda()

    def both(fill):
        zs, gs = _placed(z, pad, offset, fill), _placed(torch.zeros_like(z), pad, offset, fill)
        loss = torch.empty(rows, device="cuda")
        deft.deft_distill(zs, ids, t, loss=loss, grad=gs, teacher_lse=lse)
        heads = zs[:, :1998].unflatten(1, (3, 666))
        turned = torch.empty((rows, 3, 666), dtype=BF16, device="cuda")
        deft.deft_rotary(heads, turned, turns)
        return loss, gs, turned
    assert all(torch.isfinite(a).all() and torch.equal(a, b) for a, b in zip(both(0.0), both(bad)))


def test_rotary_in_place_of_transposed_heads():
    """[batch, heads, tokens, dim] storage with equal numbers of all three, turned where it lies."""
    x = _rand((6, 6, 6, 40), BF16, 1)
    turns = torch.from_numpy(deft.deft_rotary_frequencies(40)).cuda()
    want, tol = plain.rotary(x.transpose(1, 2), turns.cpu().numpy(), torch.arange(6).expand(6, 6))
    view = x.transpose(1, 2)
    deft.deft_rotary(view, view, turns)
    plain.close(view, want, tol)
    with pytest.raises(deft.DeftError):
        deft.deft_rotary(view, x, turns)


@pytest.mark.parametrize("cols", [16, 40, 48, 100, 128])
@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("rows", [50, 40000])
def test_short_rows_that_share_a_warp(cols, dtype, rows):
    """A row's bits do not depend on whether its neighbours take the second pass for their variance."""
    x = _rand((rows, cols), dtype, 1, 1.0, 0.3)
    y, _, mean, rstd = _norm(x)
    for row, change in ((3, 100.0), (7, float("nan")), (30, float("inf"))):
        other = x.clone()
        other[row] += change
        got = _norm(other)
        kept = torch.arange(rows, device="cuda") != row
        for a, b in ((got[0], y), (got[2], mean), (got[3], rstd)):
            assert torch.equal(a[kept], b[kept]), "other bits"


@pytest.mark.parametrize("rows,cols", [(3, 48), (1, 16), (5, 100), (9, 24)])
@pytest.mark.parametrize("odd", [False, True])
def test_few_short_rows_after_other_calls(rows, cols, odd):
    """Teams without a row have no say: the same bits whatever the shared memory and the registers hold."""
    x = _rand((rows, cols), F32, 1, 1.0, 0.4)
    first = None
    for seed in range(12):
        far = _rand((20000, cols), F32, seed, 1.0, 1000.0 if seed % 2 else 0.0)
        _norm(_placed(far, 1, 0, 0.0) if odd else far)
        y = torch.empty(rows * cols + 1, device="cuda")[1:].view(rows, cols) if odd else torch.empty((rows, cols), device="cuda")   # (odd: no shift serves both)
        mean, rstd = torch.empty(rows, device="cuda"), torch.empty(rows, device="cuda")
        deft.deft_layer_norm(x, y, mean=mean, rstd=rstd)
        got = [y.clone(), mean, rstd]
        first = first or got
        assert all(torch.equal(a, b) for a, b in zip(got, first)), "other bits"


@pytest.mark.parametrize("rows,cols", [(9, 1024), (700, 1024), (30, 331), (3000, 64), (700, 1500)])
@pytest.mark.parametrize("scale", [-0.37, 1.0 / 3.0, 1.0])
def test_accumulation_is_one_rounded_addition(rows, cols, scale):
    """What is added is what would be written: before + written, rounded once."""
    x, dy = _rand((rows, cols), F32, 1), _rand((rows, cols), F32, 2)
    _, _, mean, rstd, *_ = plain.layer_norm(x)
    mean, rstd = mean.float(), rstd.float()
    _, written = _grad(dy, x, mean, rstd, scale=scale)
    before = _rand((2 * cols,), F32, 3)
    added = before.clone()
    deft.deft_layer_norm_grad(dy, x, mean, rstd, grad_gamma=added[:cols], grad_beta=added[cols:], ws=deft.alloc_layer_norm_workspace(rows, cols), accumulate=True, scale=scale)
    assert torch.equal(added, before + written)


@pytest.mark.parametrize("vocab", [1001, 2003, 30011, 60013])
@pytest.mark.parametrize("dtype", [BF16, F16, F32])
@pytest.mark.parametrize("offset", range(8))
def test_entries_at_both_ends_of_the_row(vocab, dtype, offset):
    """The row's first and last elements share words and granules with what does not belong to it."""
    rows, top = 6, 24
    z = _placed(_rand((rows, vocab), dtype, 1, 2.0), 0, offset, 5.0)
    ids = torch.cat([torch.arange(vocab - 16, vocab), torch.arange(8)]).flip(0).expand(rows, top).contiguous().cuda()
    t = _rand((rows, top), F32, 2, 2.0)
    loss, grad = torch.empty(rows, device="cuda"), _placed(torch.zeros_like(z), 0, offset, 7.0)
    for lse in (None, t.logsumexp(1) + 1.0):
        deft.deft_distill(z, ids, t, loss=loss, grad=grad, teacher_lse=lse)
        want, want_g, tol, tol_g = plain.distill(z, ids, t, lse)
        plain.close(loss, want, tol)
        plain.close(grad, want_g, tol_g)


@pytest.mark.parametrize("vocab", [1024, 40000])
@pytest.mark.parametrize("first", [0, 700])
def test_normaliser_of_one_large_and_many_small_entries(vocab, first):
    """A student that agrees with the teacher: 1 and 1023 times e^-17, each below half a step of 1.  The loss is 0; what an entry's power,
    its logarithm or a probability is off by (at most 2^-21 and 17 times 2^-24 relative) counts by the small entries' share of
    4.3e-5 alone, which makes 1e-10.  Terms lost from the sum of the powers would make up to 1.3e-6."""
    t = torch.full((3, 1024), -17.0, device="cuda")
    t[:, first] = 0.0
    z = torch.full((3, vocab), -float("inf"), device="cuda")
    z[:, :1024] = t
    ids = torch.arange(1024, device="cuda").expand(3, 1024).contiguous()
    loss = torch.empty(3, device="cuda")
    deft.deft_distill(z, ids, t, loss=loss)
    assert loss.abs().max().item() <= 1e-9


def test_probabilities_of_arguments_between_two_numbers():
    """The teacher's log q = t - lse lies 4.5e-7 beside an fp32 number, almost half a step (4.8e-7) off: the probabilities hold it all the same.
    An error of d relative in all of them is one of 4.7 d in the loss of 4.41 (0.249 of the mass, 18.6 between the logarithms, 0.29
    of the rest's).  Allowed: expf's unit in the last place, 2^-24 relative as e^-8.3228 lies just below a power of two, and half a
    unit of the product's, 4.7 times 9e-8; the student's exponents of 20 times 1.4e-8 (log2(e) in fp32) on 0.249, 7e-8; the
    result's own rounding, 2.4e-7: 8e-7.  Without the smaller piece the loss is 4.7 times 4.5e-7 = 2.1e-6 off."""
    t = torch.full((2, 1024), 4.5e-7, device="cuda")
    lse = torch.full((2,), 8.32278, device="cuda")
    z = torch.zeros((2, 2024), device="cuda")
    z[:, :1024] = -20.0
    ids = torch.arange(1024, device="cuda").expand(2, 1024).contiguous()
    loss = torch.empty(2, device="cuda")
    deft.deft_distill(z, ids, t, loss=loss, teacher_lse=lse)
    want = plain.distill(z, ids, t, lse)[0]
    assert (loss.double().cpu() - want).abs().max().item() <= 8e-7


@pytest.mark.parametrize("bad", BAD)
@pytest.mark.parametrize("cols", [4099, 8201, 16381])
@pytest.mark.parametrize("dtype", [BF16, F32])
def test_long_rows_beside_bad_numbers(bad, cols, dtype):
    """Rows of one CTA, with the ring and (fp32, three matrices) without: a bad row and a gap of bad numbers reach no other row."""
    rows = 40
    x, add, dy = (_rand((rows, cols), dtype, s) for s in (1, 2, 3))
    gamma = _rand((cols,), F32, 4, 0.3, 1.0)

    def both(fill, row):
        xs, adds, dys = (_placed(t, 3, 5, fill) for t in (x, add, dy))
        y, s, mean, rstd = _norm(xs, adds, gamma)
        xs[row] = fill
        return [y, s, mean, rstd] + list(_grad(dys, xs, mean, rstd, gamma, adds))
    clean, got = both(0.0, 7), both(bad, 7)
    others = torch.arange(rows, device="cuda") != 7
    assert all(torch.equal(a, b) for a, b in zip(clean[:4], got[:4]))
    assert torch.isfinite(clean[4]).all() and torch.equal(clean[4][others], got[4][others])


def test_every_kernel_twice_at_once():
    """Two streams, each with its own workspace and outputs: the same bits as one after the other."""
    rows, cols, vocab = 3000, 520, 5003

    def calls(seed, stream):
        with torch.cuda.stream(stream):
            x, add, dy = (_rand((rows, cols), BF16, seed + s) for s in (1, 2, 3))
            y, s, mean, rstd = _norm(x, add)
            dx, w = _grad(dy, s, mean, rstd, add=add)
            z = _rand((rows, vocab), BF16, seed)
            t, ids = z.float().topk(9, dim=1)
            loss, grad = torch.empty(rows, device="cuda"), torch.empty_like(z)
            deft.deft_distill(z, ids, t, loss=loss, grad=grad, teacher_lse=z.float().logsumexp(1))
            turned = torch.empty((rows, 8, 65), dtype=BF16, device="cuda")
            deft.deft_rotary(y.view(rows, 8, 65), turned, torch.from_numpy(deft.deft_rotary_frequencies(64)).cuda())
        return [y, s, mean, rstd, dx, w, loss, grad, turned]
    streams = [torch.cuda.Stream() for _ in range(2)]
    want = []
    for seed in (10, 20):
        want.append(calls(seed, streams[0]))
        torch.cuda.synchronize()
    for _ in range(5):
        got = [calls(seed, s) for seed, s in zip((10, 20), streams)]
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for g, v in zip(got, want) for a, b in zip(g, v))


@pytest.mark.parametrize("gap", [0.3, 0.7, 1.1, 2.3, -0.9])
@pytest.mark.parametrize("temperature", [1.0, 4.0])
def test_loss_that_is_left_of_logarithms_that_cancel(gap, temperature):
    """Student and teacher agree on eight entries and the rest of 2000 columns: what is left of the logarithms is T^2 times what the entries'
    probabilities are off by, at most 2^-23 and 2^-24 relative on their share (below 0.05), 1.8e-7 times 0.05, and what the rest's
    sum is off by, 2^-22, times the difference of the rest's probabilities, which is of the same size: 1e-8 T^2.  A logarithm or a
    power in fp32 would be off by up to 6e-8 T^2 itself."""
    z = torch.zeros((3, 2000), device="cuda")
    z[:, 5:13] = gap
    ids = torch.arange(5, 13, device="cuda").expand(3, 8).contiguous()
    t = z[:, 5:13].contiguous()
    lse = torch.logsumexp(z.double() / temperature, 1).float()
    loss = torch.empty(3, device="cuda")
    deft.deft_distill(z, ids, t, loss=loss, teacher_lse=lse, temperature=temperature)
    want = plain.distill(z, ids, t, lse, temperature=temperature)[0]
    assert (loss.double().cpu() - want).abs().max().item() <= 1e-8 * temperature ** 2


@pytest.mark.parametrize("gap", [0.3, 0.7, 1.1, -0.9])
def test_gradient_of_a_rest_that_nearly_agrees(gap):
    """Teacher's probabilities twice the student's on eight of 2000 columns: the rest's factor 1 - q0 / p0 is some 0.004, of which a difference of
    fp32 quotients would lose 1e-7 / 0.004.  Allowed, relative: in the numerator q p0 - q0 p_e, whose terms are at most 2 and 1 times
    it, 3 and 2.5 times 2^-23 (a power each, sums, products), 1e-6; quotients, factors and the element's power (2^-22) 7e-7: 2e-6."""
    z = torch.zeros((3, 2000), device="cuda")
    z[:, 5:13] = gap
    ids = torch.arange(5, 13, device="cuda").expand(3, 8).contiguous()
    t = z[:, 5:13] + 4.0 * 0.6931472
    lse = torch.logsumexp(z.double() / 4.0, 1).float()
    grad = torch.empty_like(z)
    deft.deft_distill(z, ids, t, grad=grad, teacher_lse=lse, temperature=4.0)
    want = plain.distill(z, ids, t, lse, temperature=4.0)[1]
    rest = torch.ones(2000, dtype=torch.bool)
    rest[5:13] = False
    err = (grad.double().cpu() - want)[:, rest] / want[:, rest]
    assert err.abs().max().item() <= 2e-6
