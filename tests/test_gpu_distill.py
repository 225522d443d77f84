"""Distillation loss and gradient against the definition in 64 bits: sizes, types, strides, masks, repeated and missing entries."""
import math

import pytest
import torch

from paper_2307_03500_b200 import build as deft_build
from tests import dense_plain as plain

deft_build.build()
from paper_2307_03500_b200 import deft  # noqa: E402

pytestmark = pytest.mark.gpu
F32, BF16, F16 = torch.float32, torch.bfloat16, torch.float16
INF = math.inf


def _inputs(rows, vocab, top, dtype, seed=1, tail=True, temperature=1.0, id_type=torch.int64, teacher_type=F32, std=3.0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    z = torch.empty((rows, vocab), device="cuda").normal_(0.0, std, generator=g).to(dtype)
    t = z.float() + torch.empty((rows, vocab), device="cuda").normal_(generator=g)
    teacher, ids = t.topk(top, dim=1)
    teacher = teacher.to(teacher_type)
    lse = torch.logsumexp(t / temperature, 1) if tail else None
    return z, ids.to(id_type), teacher, lse


def _check(z, ids, teacher, lse=None, grad=None, want_grad=True, want_loss=True, **kw):
    rows = z.shape[0]
    loss = torch.full((rows,), 9.0, device="cuda") if want_loss else None
    before = z.clone()
    if want_grad and grad is None:
        grad = torch.full(z.shape, 9.0, dtype=z.dtype, device="cuda")
    deft.deft_distill(z, ids, teacher, loss=loss, grad=grad, teacher_lse=lse, **kw)
    want_l, want_g, tol_l, tol_g = plain.distill(before, ids, teacher, lse, **kw)
    if want_loss:
        plain.close(loss, want_l, tol_l)
    if want_grad:
        plain.close(grad, want_g, tol_g)
    return loss, grad


@pytest.mark.parametrize("rows,vocab,top", [(1, 1, 1), (2, 5, 3), (1, 7, 7), (3, 8, 1), (5, 33, 4), (4, 257, 16), (3, 1000, 1000), (9, 4099, 64), (300, 2003, 9),
                                            (2, 33278, 1024), (1, 50257, 300), (3, 131072, 20), (1, 262144, 5), (2, 262141, 64)])
@pytest.mark.parametrize("dtype", [BF16, F32, F16])
@pytest.mark.parametrize("tail", [False, True])
def test_sizes(rows, vocab, top, dtype, tail):
    _check(*_inputs(rows, vocab, top, dtype, tail=tail), scale=0.3)


@pytest.mark.parametrize("temperature", [0.05, 0.7, 2.0, 50.0])
@pytest.mark.parametrize("tail", [False, True])
def test_temperatures(temperature, tail):
    _check(*_inputs(20, 3001, 12, F32, tail=tail, temperature=temperature), temperature=temperature)


@pytest.mark.parametrize("id_type,teacher_type", [(torch.int32, BF16), (torch.int64, F16), (torch.int32, F32)])
def test_entry_types(id_type, teacher_type):
    _check(*_inputs(30, 1111, 10, BF16, id_type=id_type, teacher_type=teacher_type, tail=False))


@pytest.mark.parametrize("pad,offset,g_pad,g_offset", [(0, 1, 0, 1), (3, 0, 3, 0), (5, 2, 16, 7), (7, 0, 0, 0)])
def test_strides(pad, offset, g_pad, g_offset):
    rows, vocab = 7, 20011
    z, ids, teacher, lse = _inputs(rows, vocab, 8, BF16)

    def place(t, pad, offset):
        buf = torch.full((rows * (vocab + pad) + offset + 8,), 7.0, dtype=BF16, device="cuda")
        view = buf[offset:offset + rows * (vocab + pad)].view(rows, -1)[:, :vocab]
        return view.copy_(t), buf
    zs, _ = place(z, pad, offset)
    g, buf = place(torch.zeros_like(z), g_pad, g_offset)
    wide_ids, wide_t = torch.zeros((rows, 20), dtype=torch.int64, device="cuda"), torch.zeros((rows, 17), device="cuda")
    wide_ids[:, 3:11], wide_t[:, 9:17] = ids, teacher
    _check(zs, wide_ids[:, 3:11], wide_t[:, 9:17], lse, grad=g)
    g.fill_(7.0)
    assert (buf == 7.0).all(), "written beside the rows"


@pytest.mark.parametrize("tail", [False, True])
def test_rows_that_do_not_count(tail):
    """Nothing is read of a row of weight 0: infinities and NaN there do not spread."""
    z, ids, teacher, lse = _inputs(12, 5003, 6, F32, tail=tail)
    weight = torch.tensor([1.0, 0.0, 2.5, -1.0, 0.0, 1e-3] * 2, device="cuda")
    z[1], teacher[4], ids[1] = float("nan"), INF, 10 ** 12
    if tail:
        lse[4] = float("nan")
    loss, grad = _check(z, ids, teacher, lse, weight=weight, scale=2.0)
    assert not loss[[1, 4, 7, 10]].any() and not grad[[1, 4, 7, 10]].any()
    _check(z, ids, teacher, lse, weight=torch.zeros(12, device="cuda"))


@pytest.mark.parametrize("tail", [False, True])
@pytest.mark.parametrize("dtype", [BF16, F32])
def test_missing_and_repeated_entries(tail, dtype):
    z, ids, teacher, lse = _inputs(8, 999, 40, dtype, tail=tail)
    ids[0] = -1                              # no entry at all
    ids[1, 5:] = -100                        # ragged lists: padding behind the entries
    ids[2, ::2] = 999                        # outside the vocabulary
    ids[3] = ids[3, :1]                      # one column forty times
    ids[4, 20:] = ids[4, :20]                # every column twice
    ids[5] = 2 ** 40                         # (as 32 bits this is column 0)
    teacher[6, 3:] = -INF                    # entries of no probability
    teacher[7] = -INF
    if tail:
        lse[3] += 4.0                        # the sum of the probabilities stays below 1
        lse[4] += 2.0
    _check(z, ids, teacher, lse)
    again = [_check(z, ids, teacher, lse) for _ in range(2)]
    assert torch.equal(again[0][1], again[1][1]) and torch.equal(again[0][0], again[1][0]), "other bits"


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_repeated_entries_of_many_threads(dtype):
    """Which of a column's entries counts is no matter of chance: the same bits on every call, in one CTA and in a cluster."""
    for vocab in (5000, 60000):
        z, ids, teacher, lse = _inputs(40, vocab, 400, dtype)
        ids = ids[:, torch.randint(0, 150, (400,), generator=torch.Generator(device="cuda").manual_seed(3), device="cuda")].contiguous()
        first = _check(z, ids, teacher, lse + 3.0)
        for _ in range(10):
            loss, grad = torch.empty_like(first[0]), torch.empty_like(z)
            deft.deft_distill(z, ids, teacher, loss=loss, grad=grad, teacher_lse=lse + 3.0)
            assert torch.equal(loss, first[0]) and torch.equal(grad, first[1]), "other bits"


@pytest.mark.parametrize("dtype", [BF16, F32, F16])
@pytest.mark.parametrize("tail", [False, True])
def test_masked_vocabulary(dtype, tail):
    """Logits of -inf or the type's lowest value: no share, no NaN; an entry there costs an infinite loss."""
    z, ids, teacher, lse = _inputs(6, 20000, 5, dtype, tail=tail)
    low = torch.finfo(dtype).min
    keep = torch.zeros_like(z, dtype=torch.bool).scatter_(1, ids, True)
    z[0, 100:19000] = -INF
    z[1] = torch.where(keep[1], z[1], torch.full_like(z[1], -INF))      # nothing but the entries is left
    z[2] = torch.where(keep[2], z[2], torch.full_like(z[2], low))
    z[3, ids[3, 0]] = -INF                                              # an entry masked away
    z[0].scatter_(0, ids[0], 2.0)
    z[4, :] = 0.0                                                       # equal logits
    z[5, ids[5, 2]] = low
    _check(z, ids, teacher, lse)


def test_rest_far_below_the_entries():
    """The rest's share is far below what fp32 holds; its logarithm counts all the same."""
    z, ids, teacher, lse = _inputs(3, 3000, 4, F32)
    z.scatter_(1, ids, 300.0 + torch.arange(4.0, device="cuda").expand(3, 4))
    _check(z, ids, teacher, lse)
    _check(-z, ids, teacher, lse)


@pytest.mark.parametrize("bad", [float("nan"), INF])
def test_non_finite_logits(bad):
    z, ids, teacher, lse = _inputs(4, 1000, 5, F32)
    z[0, ids[0, 1]] = bad                    # an entry
    z[1, (ids[1, 0] + 1) % 1000] = bad       # beside them, or another entry
    loss, grad = torch.empty(4, device="cuda"), torch.empty_like(z)
    deft.deft_distill(z, ids, teacher, loss=loss, grad=grad, teacher_lse=lse)
    assert torch.isnan(loss[:2]).all() and torch.isnan(grad[:2]).all()
    want = plain.distill(z[2:], ids[2:], teacher[2:], lse[2:])
    plain.close(loss[2:], want[0], want[2])
    plain.close(grad[2:], want[1], want[3])


def test_in_place_one_output_and_other_lengths():
    z, ids, teacher, lse = _inputs(130, 7001, 16, BF16)
    loss, grad = _check(z, ids, teacher, lse, scale=0.5)
    same = z.clone()
    _check(same, ids, teacher, lse, grad=same, scale=0.5)
    assert torch.equal(same, grad)
    assert torch.equal(_check(z, ids, teacher, lse, want_grad=False)[0], loss)
    assert torch.equal(_check(z, ids, teacher, lse, want_loss=False, scale=0.5)[1], grad)
    one = torch.empty_like(z)                # a row's bits do not depend on the rows beside it ... as long as it is split alike
    deft.deft_distill(z[:129], ids[:129], teacher[:129], grad=one[:129], teacher_lse=lse[:129], scale=0.5)
    assert torch.equal(one[:129], grad[:129])
    none = torch.empty((0, 7001), device="cuda")
    deft.deft_distill(none, ids[:0], teacher[:0], grad=none.clone())
    z3 = z[:120].view(4, 30, 7001)
    g3 = torch.empty_like(z3)
    deft.deft_distill(z3, ids[:120].view(4, 30, 16), teacher[:120].view(4, 30, 16), grad=g3, teacher_lse=lse[:120].view(4, 30), scale=0.5)
    assert torch.equal(g3.view(120, 7001), grad[:120])


@pytest.mark.parametrize("tail", [False, True])
def test_gradient_against_differences(tail):
    z, ids, teacher, lse = _inputs(2, 40, 6, F32, tail=tail, temperature=1.7, std=1.0)
    _, grad = _check(z, ids, teacher, lse, temperature=1.7)
    step = 1e-4
    for r in range(2):
        for v in [ids[r, 0].item(), ids[r, 5].item(), 0, 17, 39]:
            up, down = z.double(), z.double()
            up[r, v] += step
            down[r, v] -= step
            value = [plain.distill(t, ids, teacher, lse, temperature=1.7)[0].sum().item() for t in (up, down)]
            # step^2 / 6 times the third derivative (below 1), 64-bit roundings over the step, fp32 result
            assert abs((value[0] - value[1]) / (2 * step) - grad[r, v].item()) < 1e-5


def test_student_that_knows_the_teacher():
    """Loss and gradient vanish where student and teacher agree."""
    z, _, _, _ = _inputs(5, 600, 10, F32)
    teacher, ids = z.topk(10, dim=1)
    loss, grad = _check(z, ids, teacher, torch.logsumexp(z, 1))
    assert loss.abs().max() < 1e-5 and grad.abs().max() < 1e-5
