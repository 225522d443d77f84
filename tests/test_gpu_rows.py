"""Row operators on the GPU against their definitions in 64 bits (tests/rows_plain.py).

Tolerances.  u = 2^-24 is the fp32 unit roundoff (half an eps), h = eps / 2 that of the output's type, tiny the half spacing
of its subnormals.  Lookup and dropout: at most four fp32 roundings (scale, position, gain, and the gain's own) of terms
whose absolute values sum to S, then one to the output's type: 4 u S + h |y| + tiny (h |y| of the computed value: another 4 u S
of it is covered by 5 u S).  Gradient: m terms added in fp32 in some order, one product with a factor rounded once, one
addition to what is there: (m + 3) u times the sum of the absolute values of everything that is added.
"""
import numpy as np
import pytest
import torch

from paper_2307_03500_b200 import build as deft_build
from tests import rows_plain as P

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
HALF = {"f32": 2.0 ** -24, "bf16": 2.0 ** -8, "f16": 2.0 ** -11}
TINY = {"f32": 2.0 ** -150, "bf16": 2.0 ** -134, "f16": 2.0 ** -25}


@pytest.fixture(scope="module")
def deft():
    if not torch.cuda.is_available():
        pytest.fail("GPU tests need a CUDA device")
    deft_build.build()
    from paper_2307_03500_b200 import deft as d
    d.lib()
    return d


def host(t):
    return t.detach().double().cpu().numpy()


def randn(rng, shape, kind, std=1.0):
    return torch.from_numpy((rng.standard_normal(shape) * std).astype(np.float32)).to(TYPES[kind]).cuda()


def laid_out(t, how):
    """The same values as a contiguous matrix, in rows with a pitch, or behind an odd number of elements."""
    if how == "plain":
        return t.clone()
    rows, cols = t.shape
    if how == "pitch16":                                  # a pitch that keeps 16-byte groups
        buf = torch.full((rows, cols + (-cols) % 8 + 8), 7.0, dtype=t.dtype, device="cuda")
        view = buf[:, :cols]
    elif how == "pitch_odd":
        buf = torch.full((rows, cols + 3), 7.0, dtype=t.dtype, device="cuda")
        view = buf[:, :cols]
    else:                                                 # "shifted": contiguous, one element past an aligned address
        buf = torch.full((rows * cols + 9,), 7.0, dtype=t.dtype, device="cuda")
        view = buf[1:1 + rows * cols].view(rows, cols)
    view.copy_(t)
    return view


def ids_of(rng, n, rows, how):
    if how == "zipf":
        ids = np.floor(np.exp(rng.random(n) * np.log(rows + 1.0)) - 1).astype(np.int64).clip(0, rows - 1)
    elif how == "uniform":
        ids = rng.integers(0, rows, n)
    elif how == "one":
        ids = np.full(n, rows // 2, dtype=np.int64)
    elif how == "ascending":
        ids = np.arange(n) % rows
    else:                                                 # "outside": some beyond the table on both sides
        ids = rng.integers(-rows // 2 - 1, rows + rows // 2 + 2, n)
    return ids


SHAPES = [(1, 1, 1), (1, 1, 8), (3, 5, 7), (33, 40, 9), (64, 100, 64), (257, 301, 255), (300, 33, 1027), (700, 500, 1500), (129, 4000, 256), (40, 9, 4104)]


@pytest.mark.parametrize("n,rows,width", SHAPES)
@pytest.mark.parametrize("table,out", [("f32", "f32"), ("bf16", "bf16"), ("f32", "bf16"), ("f16", "f32"), ("f16", "f16"), ("bf16", "f16")])
def test_embed_matches_definition(deft, n, rows, width, table, out):
    rng = np.random.default_rng(n * 1000003 + rows * 1009 + width)
    for k, (how, p, scale, pos, wide) in enumerate([("uniform", 0.0, 1.0, False, True), ("zipf", 0.1, 3.5, True, True), ("outside", 0.5, -0.25, True, False),
                                                    ("one", 0.999, 1.0, False, False)]):
        w = laid_out(randn(rng, (rows, width), table), ["plain", "pitch16", "pitch_odd", "shifted"][k])
        pw = laid_out(randn(rng, (max(1, n // 3), width), table), ["plain", "plain", "pitch16", "plain"][k]) if pos else None
        ids = ids_of(rng, n, rows, how)
        ids_d = torch.from_numpy(ids).to(torch.int64 if wide else torch.int32).cuda()
        y = laid_out(torch.full((n, width), -99.0, dtype=TYPES[out], device="cuda"), ["plain", "pitch16", "shifted", "pitch_odd"][k])
        kw = dict(scale=scale, p=p, seed=0x1234567890ABCDEF + k, offset=k * (2 ** 33 + 1))
        deft.deft_embed(w, ids_d, y, pos=pw, **kw)
        got = host(y)
        want = P.embed(host(w), ids, pos=None if pw is None else host(pw), **kw)
        size = P.embed(np.abs(host(w)), ids, pos=None if pw is None else np.abs(host(pw)), **dict(kw, scale=abs(scale)))
        assert np.all(np.abs(got - want) <= 5 * U * size + HALF[out] * np.abs(want) + TINY[out])
        if y._base is not None:                           # what lies between and behind the rows is untouched
            total = host(y._base).size
            assert (host(y._base) == 7.0).sum() >= total - n * width


@pytest.mark.parametrize("rows,cols", [(1, 1), (1, 100003), (7, 9), (64, 64), (33, 1027), (700, 1500), (5000, 8), (3, 4100)])
@pytest.mark.parametrize("x_kind,y_kind", [("f32", "f32"), ("bf16", "bf16"), ("f16", "f16"), ("bf16", "f32"), ("f32", "f16")])
def test_dropout_matches_definition(deft, rows, cols, x_kind, y_kind):
    rng = np.random.default_rng(rows * 7919 + cols)
    for k, (p, with_add) in enumerate([(0.1, False), (0.5, True), (0.0, True), (0.9999, False), (2.0 ** -16, True), (1e-9, False)]):
        x = laid_out(randn(rng, (rows, cols), x_kind), ["plain", "pitch16", "shifted", "pitch_odd", "plain", "plain"][k])
        add = laid_out(randn(rng, (rows, cols), y_kind), ["plain", "plain", "pitch16", "plain", "shifted", "plain"][k]) if with_add else None
        y = laid_out(torch.full((rows, cols), -99.0, dtype=TYPES[y_kind], device="cuda"), ["plain", "pitch_odd", "pitch16", "plain", "plain", "shifted"][k])
        kw = dict(p=p, seed=-5 + k, offset=2 ** 64 - 1 - k)
        deft.deft_dropout(x, y, add=add, **kw)
        want = P.dropout(host(x), None if add is None else host(add), **kw)
        size = P.dropout(np.abs(host(x)), None if add is None else np.abs(host(add)), **kw)
        assert np.all(np.abs(host(y) - want) <= 5 * U * size + HALF[y_kind] * np.abs(want) + TINY[y_kind])
        if p and with_add is False:                       # the mask itself, bit by bit
            assert np.array_equal(host(y) != 0, P.keep(rows, cols, p, kw["seed"], kw["offset"]) & (host(x) != 0)) or y_kind == "f16"


def check_grad(deft, rng, n, rows, width, kind, ids, wide=True, accumulate=False, layout="plain", skip_id=-1, scale=1.0, p=0.0, ws=None, dy=None, shift=0):
    dy = laid_out(randn(rng, (n, width), kind), layout) if dy is None else dy
    ids_d = torch.from_numpy(np.asarray(ids)).to(torch.int64 if wide else torch.int32).cuda()
    flat = torch.full((shift + rows * width + 5,), 3.0, device="cuda")
    g = flat[shift:shift + rows * width].view(rows, width)
    before = randn(rng, (rows, width), "f32")
    g.copy_(before)
    kw = dict(skip_id=skip_id, scale=scale, p=p, seed=99, offset=2 ** 40 + 7)
    want, size, tokens = P.embed_grad(host(dy), np.asarray(ids), rows, **kw)
    if accumulate:                                        # rows without tokens must not even be read as numbers
        g[torch.from_numpy(tokens == 0).cuda()] = float("nan")
    ws = deft.alloc_embed_workspace(n, rows, width) if ws is None else ws
    deft.deft_embed_grad(dy, ids_d, g, ws, accumulate=accumulate, **kw)
    got = host(g)
    assert torch.all(flat[:shift] == 3.0) and torch.all(flat[shift + rows * width:] == 3.0)
    if accumulate:
        assert np.all(np.isnan(got[tokens == 0]))
        want, size = want + host(before), size + np.abs(host(before))
        got, want, size, tokens = got[tokens > 0], want[tokens > 0], size[tokens > 0], tokens[tokens > 0]
    else:
        assert np.all(got[tokens == 0] == 0.0) and not np.any(np.signbit(got[tokens == 0]))
    assert np.all(np.abs(got - want) <= (tokens[:, None] + 3) * U * size + 2.0 ** -149)
    return g


@pytest.mark.parametrize("n,rows,width", SHAPES)
@pytest.mark.parametrize("kind", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("accumulate", [False, True])
def test_embed_grad_matches_definition(deft, n, rows, width, kind, accumulate):
    rng = np.random.default_rng(n * 31 + rows * 17 + width)
    check_grad(deft, rng, n, rows, width, kind, ids_of(rng, n, rows, "uniform"), accumulate=accumulate)
    check_grad(deft, rng, n, rows, width, kind, ids_of(rng, n, rows, "zipf"), accumulate=accumulate, wide=False, layout="pitch16", p=0.1, skip_id=0, shift=4)
    check_grad(deft, rng, n, rows, width, kind, ids_of(rng, n, rows, "outside"), accumulate=accumulate, layout="pitch_odd", p=0.5, scale=-7.25, shift=1)
    check_grad(deft, rng, n, rows, width, kind, ids_of(rng, n, rows, "one"), accumulate=accumulate, wide=False, layout="shifted", shift=2)


@pytest.mark.parametrize("n,rows,width,how", [
    (20000, 50, 72, "zipf"),            # every row has hundreds of tokens
    (20011, 3, 40, "uniform"),          # rows with thousands
    (70000, 7, 16, "one"),              # one row has them all
    (66000, 40000, 24, "zipf"),
    (9000, 300000, 16, "uniform"),      # more rows than the counters of 32 warps hold
    (5000, 1000000, 8, "zipf"),
    (4096, 4096, 32, "ascending"),
])
@pytest.mark.parametrize("accumulate", [False, True])
def test_embed_grad_long_rows_and_large_tables(deft, n, rows, width, how, accumulate):
    rng = np.random.default_rng(n + rows)
    check_grad(deft, rng, n, rows, width, "bf16", ids_of(rng, n, rows, how), accumulate=accumulate, p=0.1)


@pytest.mark.parametrize("n", [32767, 32768, 32769, 33792, 40000])
@pytest.mark.parametrize("how", ["outside", "zipf", "one"])
def test_embed_grad_where_tokens_are_split_first(deft, n, how):
    """Both sides of the size from which tokens are ordered by CTA first, whole and broken tiles of them."""
    rng = np.random.default_rng(n)
    check_grad(deft, rng, n, 1000, 8, "f32", ids_of(rng, n, 1000, how), skip_id=500 if how != "one" else 3)
    check_grad(deft, rng, n, 129, 20, "bf16", ids_of(rng, n, 129, how), wide=False, accumulate=True, p=0.5)


@pytest.mark.parametrize("n,rows", [(3000, 400000), (70000, 400000), (5000, 1500000), (40000, 3000000)])
def test_embed_grad_lists_longer_than_their_room(deft, n, rows):
    """Tables whose counters leave little room for a warp's list of tokens, and one token in all places: the ids (or the
    split tiles) are read again."""
    rng = np.random.default_rng(rows)
    check_rows(deft, rng, n, rows, np.where(rng.random(n) < 0.9, rows - 1, rng.integers(0, rows, n)))
    check_rows(deft, rng, n, rows, np.full(n, rows - 2))


def check_rows(deft, rng, n, rows, ids):
    """check_grad for tables too large for a dense reference: the rows with tokens, and that no others were written."""
    width = 8
    dy = randn(rng, (n, width), "f32")
    g = torch.full((rows, width), float("nan"), device="cuda")
    uniq, inv = np.unique(ids, return_inverse=True)
    at = torch.from_numpy(uniq).cuda()
    g[at] = 0.0
    deft.deft_embed_grad(dy, torch.from_numpy(ids).cuda(), g, deft.alloc_embed_workspace(n, rows, width), accumulate=True)
    want, size, tokens = P.embed_grad(host(dy), inv, uniq.size)
    assert np.all(np.abs(host(g[at]) - want) <= (tokens[:, None] + 3) * U * size)
    assert int(torch.isnan(g).any(1).sum()) == rows - uniq.size


@pytest.mark.parametrize("n", [0, 5])
def test_embed_grad_without_contributing_tokens(deft, n):
    rng = np.random.default_rng(1)
    for accumulate in (False, True):
        check_grad(deft, rng, n, 6, 16, "bf16", np.full(n, 4, dtype=np.int64), accumulate=accumulate, skip_id=4)
        check_grad(deft, rng, n, 6, 16, "f32", np.full(n, 600, dtype=np.int64), accumulate=accumulate)


@pytest.mark.parametrize("pos_rows", [0, 64, 100, 16384, 20000])
@pytest.mark.parametrize("kind,out", [("bf16", "bf16"), ("f32", "f16")])
def test_embed_where_threads_take_several_rows(deft, pos_rows, kind, out):
    """Enough tokens for several rows a thread, with position rows that repeat inside them, do not divide them, or never repeat."""
    rng = np.random.default_rng(pos_rows)
    n, rows, width = 16384 + 37, 300, 1032
    w, pos = randn(rng, (rows, width), kind), randn(rng, (pos_rows, width), kind) if pos_rows else None
    ids = ids_of(rng, n, rows, "outside")
    ids[-1] = rows - 1
    y = torch.full((n + 1, width), 9.0, dtype=TYPES[out], device="cuda")
    deft.deft_embed(w, torch.from_numpy(ids).cuda(), y[:n], scale=0.5, pos=pos, p=0.25, seed=11)
    kw = dict(scale=0.5, p=0.25, seed=11)
    want = P.embed(host(w), ids, pos=None if pos is None else host(pos), **kw)
    size = P.embed(np.abs(host(w)), ids, pos=None if pos is None else np.abs(host(pos)), **kw)
    assert np.all(np.abs(host(y[:n]) - want) <= 5 * U * size + HALF[out] * np.abs(want) + TINY[out])
    assert torch.all(y[n] == 9.0)


@pytest.mark.parametrize("x_kind,y_kind", [("bf16", "bf16"), ("f32", "f32"), ("f16", "f32")])
@pytest.mark.parametrize("with_add", [False, True])
@pytest.mark.parametrize("cols", [1024, 1500, 1021])
def test_dropout_where_threads_take_several_rows(deft, x_kind, y_kind, with_add, cols):
    rng = np.random.default_rng(cols)
    rows = 40003
    x = torch.empty((rows, cols), dtype=TYPES[x_kind], device="cuda").normal_()
    add = torch.empty((rows, cols), dtype=TYPES[y_kind], device="cuda").normal_() if with_add else None
    y = torch.full((rows + 1, cols), 9.0, dtype=TYPES[y_kind], device="cuda")
    deft.deft_dropout(x, y[:rows], add=add, p=0.1, seed=2, offset=8)
    assert torch.all(y[rows] == 9.0)
    pick = np.concatenate([np.arange(0, rows, 997), [rows - 1]])
    sel = torch.from_numpy(pick).cuda()
    c0, c1 = np.meshgrid(np.arange(-(-cols // 8), dtype=np.uint64), pick.astype(np.uint64))
    words = np.stack(P.philox([c0, c1, np.full_like(c0, 8), 0 * c0], (2, 0)), -1)
    k = np.stack([words & np.uint64(0xFFFF), words >> np.uint64(16)], -1).reshape(pick.size, -1)[:, :cols] >= P.threshold(0.1)
    xs = host(x[sel])
    want = np.where(k, xs * P.gain(0.1), 0.0) + (host(add[sel]) if with_add else 0.0)
    size = np.abs(xs) * P.gain(0.1) + (np.abs(host(add[sel])) if with_add else 0.0)
    assert np.all(np.abs(host(y[sel]) - want) <= 5 * U * size + HALF[y_kind] * np.abs(want) + TINY[y_kind])
    again = torch.empty_like(y[:rows])                      # every row, against the same call on single rows' worth of work
    half = rows // 2
    deft.deft_dropout(x, again, add=add, p=0.1, seed=2, offset=8)
    assert torch.equal(again, y[:rows])
    small = torch.empty_like(x[:half], dtype=TYPES[y_kind])
    deft.deft_dropout(x[:half], small, add=None if add is None else add[:half], p=0.1, seed=2, offset=8)
    assert torch.equal(small, y[:half])                     # a row's mask does not depend on how many rows there are


def test_largest_table_and_offsets_beyond_32_bits(deft):
    """rows * width and n * width beyond 2^31: the last rows of a table of the largest size."""
    rows, width, n = deft.EMBED_MAX_ROWS, 760, 1000
    assert rows * width > 2 ** 31
    rng = np.random.default_rng(5)
    ids = np.concatenate([np.arange(rows - n // 2, rows), rng.integers(0, rows, n - n // 2)])
    ids_d = torch.from_numpy(ids).cuda()
    dy = randn(rng, (n, width), "bf16")
    g = torch.full((rows, width), 5.0, device="cuda")
    deft.deft_embed_grad(dy, ids_d, g, deft.alloc_embed_workspace(n, rows, width))
    uniq, inv = np.unique(ids, return_inverse=True)
    want, size, tokens = P.embed_grad(host(dy), inv, uniq.size)
    got = host(g[torch.from_numpy(uniq).cuda()])
    assert np.all(np.abs(got - want) <= (tokens[:, None] + 3) * U * size)
    assert int(torch.count_nonzero(g.any(1))) == uniq.size
    y = torch.empty((n, width), device="cuda")
    deft.deft_embed(g, ids_d, y, scale=2.0)
    assert torch.equal(y, 2.0 * g[ids_d])
    del g, y
    rows, cols = 2 ** 20 + 1, 2056
    x = torch.ones((rows, cols), dtype=torch.bfloat16, device="cuda")
    deft.deft_dropout(x, x, p=0.5, seed=3)                # in place
    last = P.keep(8, cols, 0.5, 3, 0)                     # the first rows ...
    assert np.array_equal(host(x[:8]) != 0, last)
    c0, c1 = np.meshgrid(np.arange(cols // 8, dtype=np.uint64), np.arange(rows - 4, rows, dtype=np.uint64))
    w = np.stack(P.philox([c0, c1, 0 * c0, 0 * c0], (3, 0)), -1)
    want = np.stack([w & np.uint64(0xFFFF), w >> np.uint64(16)], -1).reshape(4, cols) >= 32768
    assert np.array_equal(host(x[-4:]) != 0, want)        # ... and the last


def test_one_mask_for_lookup_dropout_and_gradients(deft):
    """Dropout applied by the lookup is dropout of the lookup, bit for bit in fp32, and both gradients use its mask."""
    rng = np.random.default_rng(8)
    n, rows, width = 300, 90, 260
    w, ids = randn(rng, (rows, width), "f32"), torch.from_numpy(ids_of(rng, n, rows, "zipf")).cuda()
    pos = randn(rng, (50, width), "f32")
    kw = dict(p=0.3, seed=2 ** 63 + 11, offset=9)
    y, plain, other = (torch.empty((n, width), device="cuda") for _ in range(3))
    deft.deft_embed(w, ids, y, scale=1.7, pos=pos, **kw)
    deft.deft_embed(w, ids, plain, scale=1.7, pos=pos)
    deft.deft_dropout(plain, other, **kw)
    assert torch.equal(y, other)
    ones = torch.ones((n, width), device="cuda")
    mask = torch.empty_like(ones)
    deft.deft_dropout(ones, mask, **kw)
    assert torch.equal(mask != 0, y != 0)
    # the gradient of distinct rows is the masked incoming gradient
    g = torch.empty((n, width), device="cuda")
    deft.deft_embed_grad(ones, torch.arange(n, device="cuda"), g, deft.alloc_embed_workspace(n, n, width), **kw)
    assert torch.equal(g, mask)


@pytest.mark.parametrize("p", [0.0, 0.25])
def test_gradients_against_differences(deft, p):
    """<dL/dW, V> = (L(W + V) - L(W - V)) / 2 for the linear loss L = <y, c>, and the same for positions and for dropout's
    input.  Both sides are exact up to rounding: the operators are linear."""
    rng = np.random.default_rng(13)
    n, rows, width, seq = 120, 40, 72, 24
    w, v, c = (randn(rng, s, "f32") for s in ((rows, width), (rows, width), (n, width)))
    pos, dpos = randn(rng, (seq, width), "f32"), randn(rng, (seq, width), "f32")
    ids = torch.from_numpy(ids_of(rng, n, rows, "zipf")).cuda()
    kw = dict(p=p, seed=4, offset=4)

    def loss(table, positions):
        y = torch.empty((n, width), device="cuda")
        deft.deft_embed(table, ids, y, scale=1.5, pos=positions, **kw)
        return (y.double() * c.double()).sum().item()

    ws = deft.alloc_embed_workspace(n, rows, width)
    gw, gp, gx = torch.empty_like(w), torch.empty_like(pos), torch.empty_like(c)
    deft.deft_embed_grad(c, ids, gw, ws, scale=1.5, **kw)
    deft.deft_embed_grad(c, torch.arange(n, device="cuda") % seq, gp, ws, **kw)
    size = (1.5 * (w.abs().max() + v.abs().max()) + pos.abs().max() + dpos.abs().max()).item() / (1 - p) * c.abs().sum().item()
    tol = 8 * U * size
    assert abs((loss(w + v, pos) - loss(w - v, pos)) / 2 - (gw.double() * v.double()).sum().item()) <= tol
    assert abs((loss(w, pos + dpos) - loss(w, pos - dpos)) / 2 - (gp.double() * dpos.double()).sum().item()) <= tol
    x = randn(rng, (n, width), "f32")
    if p:
        y = torch.empty_like(x)
        deft.deft_dropout(x, y, **kw)
        deft.deft_dropout(c, gx, **kw)
        assert abs((y.double() * c.double()).sum().item() - (x.double() * gx.double()).sum().item()) <= tol


def test_infinities_and_nan(deft):
    """A dropped element contributes zero whatever it is; a kept one keeps its infinity or NaN; so do padding tokens."""
    n, rows, width, p, seed = 64, 8, 40, 0.5, 21
    k = torch.from_numpy(P.keep(n, width, p, seed, 0)).cuda()
    for bad in (float("inf"), float("-inf"), float("nan")):
        for kind in ("f32", "bf16", "f16"):
            x = torch.where(k, 1.0, bad).to(TYPES[kind])
            y = torch.empty_like(x)
            deft.deft_dropout(x, y, p=p, seed=seed)
            assert torch.equal(y, torch.where(k, 2.0, 0.0).to(y.dtype)) and not torch.signbit(y).any()
            ids = torch.arange(n, device="cuda") % rows
            g = torch.empty((rows, width), device="cuda")
            ws = deft.alloc_embed_workspace(n, rows, width)
            deft.deft_embed_grad(x, ids, g, ws, p=p, seed=seed)
            want = torch.zeros(rows, width, device="cuda").index_add_(0, ids, torch.where(k, 2.0, 0.0))
            assert torch.equal(g, want)
            deft.deft_dropout(torch.full_like(x, bad), y, p=p, seed=seed)
            assert torch.equal(y[~k], torch.zeros_like(y[~k])) and not torch.isfinite(y[k]).any()
            x = torch.ones((n, width), device="cuda").to(TYPES[kind])
            x[ids == 3] = bad                              # padding rows
            deft.deft_embed_grad(x, ids, g, ws, skip_id=3)
            assert torch.all(g[3] == 0) and torch.all(g[:3] == n // rows) and torch.all(g[4:] == n // rows)
            deft.deft_embed_grad(x, ids, g, ws)
            assert not torch.isfinite(g[3]).any() and torch.isfinite(g[4:]).all()
    w = torch.full((4, 16), float("nan"), device="cuda")
    y = torch.empty((3, 16), device="cuda")
    deft.deft_embed(w, torch.tensor([-1, 4, 2], device="cuda"), y)      # rows outside the table are zeros, not NaN
    assert torch.all(y[:2] == 0) and torch.isnan(y[2]).all()


def test_same_bits_every_time_and_reused_workspace(deft):
    rng = np.random.default_rng(2)
    big = deft.alloc_embed_workspace(30000, 5000, 136)
    big.fill_(255)                                        # it holds nothing between calls
    for n, rows, width in [(30000, 700, 136), (900, 5000, 64), (30000, 5000, 136), (1, 1, 8)]:
        ids = torch.from_numpy(ids_of(rng, n, rows, "zipf")).cuda()
        dy = randn(rng, (n, width), "bf16")
        first = None
        for ws in (big, deft.alloc_embed_workspace(n, rows, width), big):
            for accumulate in (False, True):
                g = torch.zeros((rows, width), device="cuda")
                deft.deft_embed_grad(dy, ids, g, ws, accumulate=accumulate, p=0.1, seed=1)
                first = g if first is None else first
                assert torch.equal(g, first)


def test_in_place_and_added_to_itself(deft):
    rng = np.random.default_rng(3)
    x = randn(rng, (100, 1028), "bf16")
    want, add = torch.empty_like(x), randn(rng, (100, 1028), "bf16")
    deft.deft_dropout(x, want, add=add, p=0.2, seed=6)
    a = add.clone()
    deft.deft_dropout(x, a, add=a, p=0.2, seed=6)
    assert torch.equal(a, want)
    deft.deft_dropout(x, want, p=0.2, seed=6)
    deft.deft_dropout(x, x, p=0.2, seed=6)
    assert torch.equal(x, want)


def test_other_streams_and_two_calls_at_once(deft):
    rng = np.random.default_rng(4)
    n, rows, width = 20000, 300, 520
    ids = torch.from_numpy(ids_of(rng, n, rows, "zipf")).cuda()
    dy = randn(rng, (n, width), "bf16")
    want = torch.empty((rows, width), device="cuda")
    deft.deft_embed_grad(dy, ids, want, deft.alloc_embed_workspace(n, rows, width), p=0.1)
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(3)]
    out = [(torch.empty((rows, width), device="cuda"), deft.alloc_embed_workspace(n, rows, width)) for _ in streams]
    torch.cuda.synchronize()
    for _ in range(3):
        for s, (g, ws) in zip(streams, out):
            deft.deft_embed_grad(dy, ids, g, ws, p=0.1, stream=s)
    torch.cuda.synchronize()
    assert all(torch.equal(g, want) for g, _ in out)


def test_captured_and_replayed(deft):
    """Two graphs with workspaces of their own; the mask of a replay follows the counter on the device."""
    rng = np.random.default_rng(6)
    n, rows, width = 700, 200, 152
    w = randn(rng, (rows, width), "f32")
    graphs = []
    for k in range(2):
        ids = torch.from_numpy(ids_of(rng, n, rows, "zipf")).cuda()
        count = torch.zeros(1, dtype=torch.int64, device="cuda")
        y, g = torch.empty((n, width), device="cuda"), torch.empty((rows, width), device="cuda")
        ws = deft.alloc_embed_workspace(n, rows, width)
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            graph = torch.cuda.CUDAGraph()
            with torch.cuda.graph(graph, stream=side):
                deft.deft_embed(w, ids, y, p=0.5, seed=k, offset=100, offset_d=count)
                deft.deft_embed_grad(y, ids, g, ws, p=0.5, seed=k, offset=100, offset_d=count)
                count.add_(1)
        graphs.append((graph, ids, count, y, g))
    for t in range(3):
        for k, (graph, ids, count, y, g) in enumerate(graphs):
            if t == 2:
                ids.copy_(torch.from_numpy(ids_of(rng, n, rows, "one")))     # new inputs in the captured buffers
            graph.replay()
        torch.cuda.synchronize()
        for k, (graph, ids, count, y, g) in enumerate(graphs):
            assert int(count) == t + 1
            y2, g2 = torch.empty_like(y), torch.empty_like(g)
            deft.deft_embed(w, ids, y2, p=0.5, seed=k, offset=100 + t)
            deft.deft_embed_grad(y2, ids, g2, deft.alloc_embed_workspace(n, rows, width), p=0.5, seed=k, offset=100 + t)
            assert torch.equal(y, y2) and torch.equal(g, g2)


def test_refusals_of_the_binding(deft):
    f = lambda *s, **kw: torch.zeros(*s, device="cuda", **kw)  # noqa: E731
    ids = f(4, dtype=torch.int64)
    ws = deft.alloc_embed_workspace(4, 6, 8)
    for call in (lambda: deft.deft_embed(f(6, 8), ids, f(4, 9)), lambda: deft.deft_embed(f(6, 8), ids, f(5, 8)),
                 lambda: deft.deft_embed(f(6, 8), ids.cpu(), f(4, 8)), lambda: deft.deft_embed(f(6, 8), ids, f(4, 8), pos=f(4, 8).half()),
                 lambda: deft.deft_embed(f(6, 8).double(), ids, f(4, 8)), lambda: deft.deft_embed(f(6, 8), ids.short(), f(4, 8)),
                 lambda: deft.deft_embed_grad(f(4, 8), ids, f(6, 8).half(), ws), lambda: deft.deft_embed_grad(f(4, 9), ids, f(6, 8), ws),
                 lambda: deft.deft_embed_grad(f(4, 8), ids, f(6, 16)[:, :8], ws), lambda: deft.deft_embed_grad(f(1, 8).expand(4, 8), ids, f(6, 8), ws),
                 lambda: deft.deft_dropout(f(4, 8), f(4, 9)), lambda: deft.deft_dropout(f(4, 8), f(4, 8), add=f(4, 8).half()),
                 lambda: deft.deft_dropout(f(8, 4).t(), f(4, 8)), lambda: deft.deft_embed_grad(f(4, 8), ids, f(6, 8), ws[::2]),
                 lambda: deft.deft_dropout(f(4, 8), f(4, 8), offset_d=f(1, dtype=torch.complex64))):
        with pytest.raises(ValueError):
            call()
    for call in (lambda: deft.deft_dropout(f(4, 8), f(4, 8), p=1.0), lambda: deft.deft_embed(f(6, 8), ids, f(4, 8), scale=float("inf")),
                 lambda: deft.deft_embed_grad(f(4, 8), ids, f(6, 8), ws[:256]), lambda: deft.alloc_embed_workspace(1, deft.EMBED_MAX_ROWS + 1, 8)):
        with pytest.raises(deft.DeftError):
            call()


# ---- the framework's own path: a step whose embedding gradient comes by rows ----
def _parts_reference(deft, e, grad, parts, start, ws):
    """What deft_layer_norms gives for the gradient with zeros in the parts."""
    g = grad.clone()
    for a, b in parts:
        g[a:b] = 0.0
    norms = torch.empty(start.numel() - 1, dtype=torch.float64, device="cuda")
    deft.deft_layer_norms(e, g, start, norms, ws)
    return norms


@pytest.mark.parametrize("sizes,parts", [
    ([100003], [(0, 100003)]),
    ([40000, 8192, 30000], [(0, 40000)]),
    ([40000, 8192, 30000], [(40000, 48192)]),
    ([50000, 50000, 7], [(1, 2), (9000, 30001), (49999, 50001), (100003, 100007)]),
    ([65536, 65536], [(0, 8192), (8192, 16384), (100000, 100000), (131071, 131072)]),
    ([5, 3, 9], [(0, 5), (8, 17)]),
])
def test_norms_with_parts_added(deft, sizes, parts):
    rng = np.random.default_rng(len(sizes))
    n_g = sum(sizes)
    start = torch.from_numpy(np.concatenate([[0], np.cumsum(sizes)]).astype(np.int64)).cuda()
    ws = deft.alloc_workspace(n_g, len(sizes))
    e, grad = randn(rng, (n_g,), "f32"), randn(rng, (n_g,), "f32")
    want_e = e.clone()
    want = _parts_reference(deft, want_e, grad, parts, start, ws)
    for a, b in parts:
        grad[a:b] = float("nan")                           # not read
    norms = torch.empty_like(want)
    deft.deft_layer_norms_part(e, grad, parts, start, norms, ws)
    assert torch.equal(e, want_e)
    ref = np.array([np.linalg.norm(host(want_e)[a:b]) for a, b in zip(host(start)[:-1].astype(int), host(start)[1:].astype(int))])
    assert np.all(np.abs(host(norms) - ref) <= 1e-5 * ref)
    before = e.clone()
    deft.deft_layer_norms_part(e, None, parts, start, norms, ws)       # without a gradient nothing is written
    assert torch.equal(e, before) and np.all(np.abs(host(norms) - ref) <= 1e-5 * ref)


def _rows_case(deft, rng, vocab, width, n, rest, N, density):
    from paper_2307_03500_b200.pipeline import DeftStep, RowGradient
    sizes = [77, vocab * width] + rest
    ds = DeftStep(sizes, N, density)
    ids = torch.from_numpy(ids_of(rng, n, vocab, "zipf")).cuda()
    row = RowGradient(1, ids, randn(rng, (n, width), "bf16"), scale=0.5, skip_id=1, p=0.1, seed=3, offset=4)
    grad = randn(rng, (ds.n_g,), "f32")
    dense = grad.clone()
    deft.deft_embed_grad(row.grad_out, ids, dense[77:77 + vocab * width].view(vocab, width), deft.alloc_embed_workspace(n, vocab, width),
                         scale=0.5, skip_id=1, p=0.1, seed=3, offset=4)
    grad[77:77 + vocab * width] = float("nan")             # not read
    return ds, row, grad, dense


@pytest.mark.parametrize("fused", [False, True])
def test_step_with_rows_is_the_step_with_the_dense_gradient(deft, fused):
    from paper_2307_03500_b200.pipeline import DeftStep
    rng = np.random.default_rng(17)
    ds, row, grad, dense = _rows_case(deft, rng, 900, 76, 500, [20000, 300, 9000], 4, 0.01)
    other = DeftStep([77, 900 * 76, 20000, 300, 9000], 4, 0.01)
    e = randn(rng, (ds.n_g,), "f32", 0.1)
    want = e.clone()
    for it in range(3):
        if fused:
            a, b = ds.step_fused(e, grad, it, rows=[row]), other.step_fused(want, dense, it)
        else:
            a, _ = ds.step(e, grad, it, rows=[row])
            b, _ = other.step(want, dense, it)
        torch.cuda.synchronize()
        assert torch.equal(e, want)
        assert a.k_l.tolist() == b.k_l.tolist() and a.bin_of_layer.tolist() == b.bin_of_layer.tolist()
        k = a.sum_k
        assert torch.equal(ds.idx_d[:k], other.idx_d[:k]) and torch.equal(ds.val_d[:k], other.val_d[:k])


def test_staged_step_with_rows(deft):
    """A vector large enough for the accumulate pass to stage for the selection: the same entries either way."""
    from paper_2307_03500_b200.pipeline import DeftStep
    rng = np.random.default_rng(19)
    rest = [20_000_000, 9_000_001, 1500]
    ds, row, grad, dense = _rows_case(deft, rng, 20000, 1024, 900, rest, 4, 0.001)
    other = DeftStep([77, 20000 * 1024] + rest, 4, 0.001)
    assert ds.n_g >= 48_000_000
    e = randn(rng, (ds.n_g,), "f32", 0.1)
    want = e.clone()
    for it in range(3):
        a, b = ds.step_fused(e, grad, it, rows=[row]), other.step_fused(want, dense, it)
        torch.cuda.synchronize()
        assert a.sum_k == b.sum_k and torch.equal(e, want)
        assert torch.equal(ds.idx_d[:a.sum_k], other.idx_d[:a.sum_k])


def test_staged_step_with_rows_and_steady_magnitudes(deft):
    """The same with a residual that starts at zero in every step (the magnitudes repeat, so that the remembered cuts hold):
    the layers are finished from what the accumulate pass staged."""
    from paper_2307_03500_b200.pipeline import DeftStep
    rng = np.random.default_rng(20)
    rest = [20_000_000, 9_000_001, 1500]
    ds, row, grad, dense = _rows_case(deft, rng, 20000, 1024, 20000, rest, 4, 0.001)
    other = DeftStep([77, 20000 * 1024] + rest, 4, 0.001)
    for it in range(3):
        e, want = torch.zeros(ds.n_g, device="cuda"), torch.zeros(ds.n_g, device="cuda")
        a, b = ds.step_fused(e, grad, it, rows=[row]), other.step_fused(want, dense, it)
        torch.cuda.synchronize()
        assert a.sum_k == b.sum_k and torch.equal(e, want)
        assert torch.equal(ds.idx_d[:a.sum_k], other.idx_d[:a.sum_k])
    assert deft.deft_select_stats(ds.ws, ds.L)["one_read"] > 0


def test_step_rows_refusals(deft):
    from dataclasses import replace
    rng = np.random.default_rng(23)
    ds, row, grad, _ = _rows_case(deft, rng, 90, 8, 50, [200, 100], 2, 0.05)
    e = randn(rng, (ds.n_g,), "f32")
    before = e.clone()
    for bad in (replace(row, tensor=-1), replace(row, tensor=9), replace(row, tensor=0), replace(row, grad_out=row.grad_out[:, :7]),
                replace(row, ids=row.ids[:-1]), replace(row, ids=row.ids.short()), replace(row, ids=row.ids.cpu()), replace(row, p=1.0),
                replace(row, scale=float("nan")), replace(row, grad_out=row.grad_out.double()), replace(row, offset_d=torch.zeros(1, device="cuda"))):
        for call in (ds.step, ds.step_fused):
            with pytest.raises(ValueError):
                call(e, grad, 0, rows=[row, bad])
    assert torch.equal(e, before)                          # refused before anything was added


def test_two_row_gradients_of_one_table(deft):
    """A table that is looked up twice (encoder and decoder): its part takes both, in order."""
    from paper_2307_03500_b200.pipeline import DeftStep, RowGradient
    rng = np.random.default_rng(37)
    vocab, width = 200, 24
    ds = DeftStep([vocab * width, 1000], 2, 0.05)
    rows = [RowGradient(0, torch.from_numpy(ids_of(rng, n, vocab, "zipf")).cuda(), randn(rng, (n, width), "f32")) for n in (300, 41)]
    e, grad = randn(rng, (ds.n_g,), "f32"), randn(rng, (ds.n_g,), "f32")
    want = e.clone()
    table = want[:vocab * width].view(vocab, width)
    for r in rows:
        deft.deft_embed_grad(r.grad_out, r.ids, table, deft.alloc_embed_workspace(300, vocab, width), accumulate=True)
    want[vocab * width:] += grad[vocab * width:]
    norms = ds.layer_norms(e, grad, rows)
    assert torch.equal(e, want)
    ref = np.array([np.linalg.norm(host(want)[a:b]) for a, b in zip(ds.layer_start[:-1], ds.layer_start[1:])])
    assert np.all(np.abs(norms - ref) <= 1e-5 * ref)


def test_multi_worker_simulation_with_rows(deft):
    """Two simulated workers with token batches of their own: the same as with their dense gradients."""
    from paper_2307_03500_b200.pipeline import RowGradient
    from paper_2307_03500_b200.simulate import MultiWorkerSim
    rng = np.random.default_rng(29)
    vocab, width, rest, n = 300, 40, [9000, 500], 64
    a = MultiWorkerSim([vocab * width] + rest, 2, 0.02)
    b = MultiWorkerSim([vocab * width] + rest, 2, 0.02)
    ws = deft.alloc_embed_workspace(n, vocab, width)
    for _ in range(3):
        rows, grads, dense = [], [], []
        for r in range(2):
            row = RowGradient(0, torch.from_numpy(ids_of(rng, n, vocab, "zipf")).cuda(), randn(rng, (n, width), "bf16"), p=0.25, seed=r)
            g = randn(rng, (a.n_g,), "f32")
            g[:vocab * width] = 0.0
            d = g.clone()
            deft.deft_embed_grad(row.grad_out, row.ids, d[:vocab * width].view(vocab, width), ws, p=0.25, seed=r)
            rows.append([row])
            grads.append(g)
            dense.append(d)
        assert a.step(grads, rows) == b.step(dense)
        assert torch.equal(a.last_union, b.last_union) and torch.equal(a.last_mean, b.last_mean)
        assert all(torch.equal(x, y) for x, y in zip(a.e, b.e))


def test_language_model_front_end_step(deft):
    """A run of them together: lookup with positions and dropout, a block's dropout into the residual stream, the backward
    calls in reverse, and the sparsification step on the vector whose embedding gradient came by rows."""
    from paper_2307_03500_b200.pipeline import DeftStep, RowGradient
    rng = np.random.default_rng(31)
    vocab, width, batch, seq = 500, 96, 6, 20
    n = batch * seq
    sizes = [vocab * width, seq * width, width * width]
    ds = DeftStep(sizes, 4, 0.02)
    flat = randn(rng, (ds.n_g,), "f32", 0.1)
    table, pos = flat[:vocab * width].view(vocab, width), flat[vocab * width:(vocab + seq) * width].view(seq, width)
    lin = flat[(vocab + seq) * width:].view(width, width)
    ids = torch.from_numpy(ids_of(rng, n, vocab, "zipf")).cuda()
    place = torch.arange(n, device="cuda") % seq
    c = randn(rng, (n, width), "f32")                      # dL/d(output)
    e = torch.zeros(ds.n_g, device="cuda")
    for it in range(2):
        kw0, kw1 = dict(p=0.1, seed=5, offset=2 * it), dict(p=0.1, seed=5, offset=2 * it + 1)
        x, y, dz = (torch.empty((n, width), device="cuda") for _ in range(3))
        deft.deft_embed(table, ids, x, scale=2.0, pos=pos, **kw0)
        z = x @ lin
        deft.deft_dropout(z, y, add=x, **kw1)              # y = x + D(x L)
        deft.deft_dropout(c, dz, **kw1)
        dx = c + dz @ lin.t()
        grad = torch.zeros(ds.n_g, device="cuda")
        grad[(vocab + seq) * width:] = (x.t() @ dz).view(-1)
        rows = [RowGradient(0, ids, dx, scale=2.0, **kw0), RowGradient(1, place, dx, **kw0)]
        before = e.clone()
        plan, outs = ds.step(e, grad, it, rows=rows)
        # the same by definition, in 64 bits
        k0, k1 = (torch.from_numpy(P.keep(n, width, 0.1, 5, 2 * it + i)).cuda().double() * P.gain(0.1) for i in range(2))
        w64, p64, l64 = (t.double().clone().requires_grad_(True) for t in (table, pos, lin))
        x64 = (2.0 * w64[ids] + p64[place]) * k0
        y64 = x64 + (x64 @ l64) * k1
        gw, gp, gl = torch.autograd.grad(y64, (w64, p64, l64), c.double())
        full = before.double() + torch.cat([gw.view(-1), gp.view(-1), gl.view(-1)])
        acc = e.double().clone()
        for val, idx in outs:                              # the step cleared what it selected
            acc[idx] = val.double()
        assert torch.allclose(y.double(), y64, rtol=1e-4, atol=1e-4)
        assert (acc - full).norm() <= 2e-3 * full.norm()   # the two products in torch run in TF32 at worst (2^-11 per term)
        sel = torch.cat([i for _, i in outs])
        assert sel.numel() == ds.k and torch.all(e[sel] == 0)


def test_subnormals_are_kept(deft):
    """Neither the mixed-precision additions nor the products flush: single tokens come back exactly."""
    for kind, tiny in (("bf16", 2.0 ** -133), ("f16", 2.0 ** -24), ("f32", 2.0 ** -149)):
        for width in (8, 41):
            x = (torch.arange(1, 4 * width + 1, device="cuda", dtype=torch.float64).view(4, width) * tiny).to(TYPES[kind])
            x[1] = -x[1]
            ids = torch.tensor([2, 0, 3, 1], device="cuda")
            g = torch.empty((4, width), device="cuda")
            ws = deft.alloc_embed_workspace(4, 4, width)
            deft.deft_embed_grad(x, ids, g, ws)
            assert torch.equal(g[ids].double(), x.double())
            y, z = torch.empty_like(x), torch.empty((4, width), device="cuda")
            deft.deft_embed(x, ids, y)
            assert torch.equal(y, x[ids])
            deft.deft_dropout(x, z, add=torch.zeros_like(z), p=0.0)
            assert torch.equal(z.double(), x.double())


def test_captured_large_calls(deft):
    """The split pass and a launch with most of the shared memory, captured and replayed with other ids."""
    rng = np.random.default_rng(41)
    n, rows, width = 20000, 150000, 40
    dy = randn(rng, (n, width), "bf16")
    ids = torch.from_numpy(ids_of(rng, n, rows, "zipf")).cuda()
    g, ws = torch.zeros((rows, width), device="cuda"), deft.alloc_embed_workspace(n, rows, width)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.stream(side), torch.cuda.graph(graph, stream=side):
        deft.deft_embed_grad(dy, ids, g, ws, p=0.1, seed=2)
    for how in ("zipf", "uniform", "one"):
        ids.copy_(torch.from_numpy(ids_of(rng, n, rows, how)))
        graph.replay()
        want = torch.empty_like(g)
        torch.cuda.synchronize()
        deft.deft_embed_grad(dy, ids, want, deft.alloc_embed_workspace(n, rows, width), p=0.1, seed=2)
        assert torch.equal(g, want)


def test_one_process_per_worker_with_rows(deft):
    """DistributedWorker as the only rank of an NCCL group: rows are the dense gradient there too."""
    import os
    import torch.distributed as dist
    from paper_2307_03500_b200.distributed import DistributedWorker
    from paper_2307_03500_b200.pipeline import RowGradient
    os.environ["MASTER_ADDR"], os.environ["MASTER_PORT"] = "127.0.0.1", "29541"
    rng = np.random.default_rng(43)
    vocab, width, n = 250, 36, 70
    dist.init_process_group("nccl", rank=0, world_size=1)
    try:
        a, b = (DistributedWorker([vocab * width, 5000], 0.02, "deft", device="cuda:0") for _ in range(2))
        ws = deft.alloc_embed_workspace(n, vocab, width)
        for t in range(2):
            row = RowGradient(0, torch.from_numpy(ids_of(rng, n, vocab, "zipf")).cuda(), randn(rng, (n, width), "f16"), p=0.5, seed=t)
            grad = randn(rng, (vocab * width + 5000,), "f32")
            dense = grad.clone()
            deft.deft_embed_grad(row.grad_out, row.ids, dense[:vocab * width].view(vocab, width), ws, p=0.5, seed=t)
            x, y = a.step(grad, [row]), b.step(dense)
            assert torch.equal(x.union, y.union) and torch.equal(x.mean, y.mean) and x.error == y.error
            assert torch.equal(a.e, b.e)
    finally:
        dist.destroy_process_group()
