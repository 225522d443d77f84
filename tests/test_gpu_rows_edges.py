"""Row operators at the sizes where another path takes over (tolerances: tests/test_gpu_rows.py)."""
import numpy as np
import pytest
import torch

from tests import rows_plain as P
from tests.test_gpu_rows import HALF, TINY, TYPES, U, check_grad, deft, host, ids_of, laid_out, randn  # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("n", [16383, 16384, 16385, 17408, 17409])
@pytest.mark.parametrize("how", ["outside", "zipf", "one"])
def test_embed_grad_around_the_split_pass(deft, n, how):  # noqa: F811
    """Up to 16384 tokens one pass groups them, above it a pass over tiles of 1024 goes first (the 17th tile has one token);
    the workspace is exactly as large as asked for, and nothing is written behind it."""
    rng = np.random.default_rng(n)
    for rows, width, kind, kw in [(1000, 8, "f32", dict(skip_id=500 if how != "one" else 3)),
                                  (129, 20, "bf16", dict(wide=False, accumulate=True, p=0.5)),
                                  (40000, 36, "f16", dict(layout="pitch_odd", shift=1))]:
        size = deft.deft_embed_workspace_bytes(n, rows, width)
        room = torch.full((size + 4096,), 171, dtype=torch.uint8, device="cuda")
        check_grad(deft, rng, n, rows, width, kind, ids_of(rng, n, rows, how), ws=room[:size], **kw)
        assert torch.all(room[size:] == 171)


@pytest.mark.parametrize("n", [8191, 9217, 12345, 16384])
def test_embed_grad_large_calls_of_one_pass(deft, n):  # noqa: F811
    rng = np.random.default_rng(n)
    for accumulate in (False, True):
        check_grad(deft, rng, n, 5000, 12, "bf16", ids_of(rng, n, 5000, "zipf"), accumulate=accumulate, p=0.1)
        check_grad(deft, rng, n, 300, 9, "f32", ids_of(rng, n, 300, "uniform"), accumulate=accumulate, wide=False)


@pytest.mark.parametrize("width", [1020, 1021])
@pytest.mark.parametrize("pos_rows", [0, 100])
@pytest.mark.parametrize("kind,out,layout", [("bf16", "bf16", "plain"), ("f16", "f32", "shifted"), ("f32", "bf16", "pitch_odd"), ("f32", "f32", "plain")])
def test_embed_rows_off_16_byte_boundaries_where_threads_take_several(deft, width, pos_rows, kind, out, layout):  # noqa: F811
    """Rows on 8-byte boundaries and on those of single elements, with several tokens a thread."""
    rng = np.random.default_rng(width + pos_rows)
    n, rows = 16384 + 37, 300
    w, pos = laid_out(randn(rng, (rows, width), kind), layout), randn(rng, (pos_rows, width), kind) if pos_rows else None
    ids = ids_of(rng, n, rows, "outside")
    ids[-1] = rows - 1
    y = torch.full((n + 1, width), 9.0, dtype=TYPES[out], device="cuda")
    kw = dict(scale=-0.5, p=0.25, seed=11)
    deft.deft_embed(w, torch.from_numpy(ids).cuda(), y[:n], pos=pos, **kw)
    want = P.embed(host(w), ids, pos=None if pos is None else host(pos), **kw)
    size = P.embed(np.abs(host(w)), ids, pos=None if pos is None else np.abs(host(pos)), **dict(kw, scale=0.5))
    assert np.all(np.abs(host(y[:n]) - want) <= 5 * U * size + HALF[out] * np.abs(want) + TINY[out])
    assert torch.all(y[n] == 9.0)


@pytest.mark.parametrize("kind,with_add", [("f32", True), ("f16", False)])
def test_dropout_rows_on_8_byte_boundaries_where_threads_take_several(deft, kind, with_add):  # noqa: F811
    rng = np.random.default_rng(3)
    rows, cols = 20003, 1022 if kind == "f32" else 1020
    x = randn(rng, (rows, cols), kind)
    add = randn(rng, (rows, cols), kind) if with_add else None
    y = torch.full((rows + 1, cols), 9.0, dtype=TYPES[kind], device="cuda")
    deft.deft_dropout(x, y[:rows], add=add, p=0.5, seed=7, offset=1)
    want = P.dropout(host(x), None if add is None else host(add), p=0.5, seed=7, offset=1)
    size = P.dropout(np.abs(host(x)), None if add is None else np.abs(host(add)), p=0.5, seed=7, offset=1)
    assert np.all(np.abs(host(y[:rows]) - want) <= 5 * U * size + HALF[kind] * np.abs(want) + TINY[kind])
    assert torch.all(y[rows] == 9.0)


@pytest.mark.parametrize("kind", ["f32", "f16", "bf16"])
def test_gradient_of_position_rows(deft, kind):  # noqa: F811
    """Every position row has n / S tokens: the ids a caller makes with arange."""
    rng = np.random.default_rng(9)
    batch, seq, width = 24, 640, 264
    check_grad(deft, rng, batch * seq, seq, width, kind, np.arange(batch * seq) % seq, accumulate=True, p=0.1)
    check_grad(deft, rng, batch * seq, seq, width, kind, np.arange(batch * seq) % seq)
