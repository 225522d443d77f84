"""Steps with row gradients on the GPU: refused calls leave the residual alone."""
import numpy as np
import pytest
import torch

from paper_2307_03500_b200 import build as deft_build

pytestmark = pytest.mark.gpu

VOCAB, WIDTH, N_TOKENS, REST = 300, 40, 64, [9000, 500]
SIZES = [VOCAB * WIDTH] + REST


@pytest.fixture(scope="module")
def deft():
    if not torch.cuda.is_available():
        pytest.fail("GPU tests need a CUDA device")
    deft_build.build()
    from paper_2307_03500_b200 import deft as d
    d.lib()
    return d


def _inputs(rng, n_g):
    from paper_2307_03500_b200.pipeline import RowGradient
    row = RowGradient(0, torch.from_numpy(rng.integers(0, VOCAB, N_TOKENS)).cuda(),
                      torch.from_numpy(rng.standard_normal((N_TOKENS, WIDTH)).astype(np.float32)).cuda(), scale=0.5, p=0.1, seed=3)
    vec = lambda: torch.from_numpy(rng.standard_normal(n_g).astype(np.float32)).cuda()  # noqa: E731
    return row, vec(), vec()


def _shifted(t):
    """The same values 4 bytes past an aligned address."""
    buf = torch.empty(t.numel() + 8, device="cuda")
    buf[1:1 + t.numel()] = t
    return buf[1:1 + t.numel()]


def _bad_gradients(grad):
    return [grad.half(), grad.double(), grad.cpu(), torch.stack([grad, grad], 1)[:, 0], grad[:-1], _shifted(grad)]


@pytest.mark.parametrize("how", ["layer_norms", "step", "step_fused"])
def test_refused_step_leaves_the_residual(deft, how):
    """A gradient or a residual that the accumulate call would refuse, or a rank that is none, is refused before the rows are
    added: a caller who mends it and calls again adds them once."""
    from paper_2307_03500_b200.pipeline import DeftStep
    ds, other = DeftStep(SIZES, 4, 0.01), DeftStep(SIZES, 4, 0.01)
    row, grad, e = _inputs(np.random.default_rng(51), ds.n_g)
    before = e.clone()
    call = getattr(ds, how)
    kinds = (ValueError, deft.DeftError)
    for bad in _bad_gradients(grad):
        with pytest.raises(kinds):
            call(e, bad, rows=[row])
        assert torch.equal(e, before)
    shifted = _shifted(e)
    with pytest.raises(kinds):
        call(shifted, grad, rows=[row])
    assert torch.equal(shifted, before)
    if how != "layer_norms":
        with pytest.raises(kinds):
            call(e, grad, -1, rows=[row])
        assert torch.equal(e, before)
    if how == "step_fused":
        for rank in (-2, 4, 2 ** 31 - 1):
            with pytest.raises(kinds):
                call(e, grad, 0, rank, rows=[row])
            assert torch.equal(e, before)
        for events in ([], [torch.cuda.Event(enable_timing=True)] * 3):
            with pytest.raises(kinds):
                call(e, grad, 0, events=events, rows=[row])
            assert torch.equal(e, before)
    want = before.clone()
    call(e, grad, rows=[row])
    getattr(other, how)(want, grad, rows=[row])
    torch.cuda.synchronize()
    assert torch.equal(e, want)


def test_refused_simulation_leaves_every_residual(deft):
    """A worker whose arguments are refused leaves the residuals of the workers before it as they were, too."""
    from paper_2307_03500_b200.simulate import MultiWorkerSim
    rng = np.random.default_rng(53)
    sim, other = MultiWorkerSim(SIZES, 2, 0.02), MultiWorkerSim(SIZES, 2, 0.02)
    row, g0, g1 = _inputs(rng, sim.n_g)
    kinds = (ValueError, deft.DeftError)
    for grads, rows in [([g0, bad], [[row], [row]]) for bad in _bad_gradients(g1)] + [([g0, g1], [[row]]), ([g0], [[row], [row]])]:
        with pytest.raises(kinds):
            sim.step(grads, rows)
        assert all(not e.any() for e in sim.e)
    assert sim.step([g0, g1], [[row], [row]]) == other.step([g0, g1], [[row], [row]])
    assert all(torch.equal(a, b) for a, b in zip(sim.e, other.e))


def _row_batch(rng, n, vocab, width):
    from paper_2307_03500_b200.pipeline import RowGradient
    return RowGradient(0, torch.from_numpy(rng.integers(0, vocab, n)).cuda(),
                       torch.from_numpy(rng.standard_normal((n, width)).astype(np.float32)).cuda(), p=0.1, seed=n)


def _added(deft, ds, row, vocab, width):
    """What add_rows leaves in a residual of zeros."""
    want = torch.zeros(ds.n_g, device="cuda")
    deft.deft_embed_grad(row.grad_out, row.ids, want[:vocab * width].view(vocab, width),
                         deft.alloc_embed_workspace(row.ids.numel(), vocab, width), accumulate=True, p=row.p, seed=row.seed)
    return want


def test_rows_added_on_several_streams_at_once(deft):
    """Calls of different sizes on three streams without a wait between them, each on a residual of its own."""
    from paper_2307_03500_b200.pipeline import DeftStep
    rng = np.random.default_rng(57)
    vocab, width = 4000, 256
    ds = DeftStep([vocab * width, 1000], 2, 0.01)
    batches = [[_row_batch(rng, n, vocab, width) for n in sizes] for sizes in ((700, 20000, 64), (30000, 5, 3000), (64, 9000, 30000))]
    want = [[_added(deft, ds, row, vocab, width) for row in rows] for rows in batches]
    got = [[torch.zeros_like(w) for w in ws] for ws in want]
    streams = [torch.cuda.Stream() for _ in batches]
    torch.cuda.synchronize()
    for i in range(3):
        for s, rows, out in zip(streams, batches, got):
            ds.add_rows(out[i], [rows[i]], stream=s)
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for ws, gs in zip(want, got) for a, b in zip(ws, gs))


def test_captured_rows_and_larger_calls_after(deft):
    """A captured call keeps its workspace when later, larger calls on the same object need more."""
    from paper_2307_03500_b200.pipeline import DeftStep
    rng = np.random.default_rng(59)
    vocab, width = 2000, 136
    ds = DeftStep([vocab * width, 1000], 2, 0.01)
    small, large = _row_batch(rng, 900, vocab, width), _row_batch(rng, 40000, vocab, width)
    want_small, want_large = _added(deft, ds, small, vocab, width), _added(deft, ds, large, vocab, width)
    a, b = torch.zeros(ds.n_g, device="cuda"), torch.zeros(ds.n_g, device="cuda")
    graphs = []
    for out in (a, b):
        graph = torch.cuda.CUDAGraph()
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side), torch.cuda.graph(graph, stream=side):
            out.zero_()
            ds.add_rows(out, [small])
        graphs.append(graph)
        torch.cuda.synchronize()
    for _ in range(2):
        e = torch.zeros(ds.n_g, device="cuda")
        ds.add_rows(e, [large])
        junk = [torch.full((1 << 22,), 255, dtype=torch.uint8, device="cuda") for _ in range(8)]   # over anything that was let go
        for graph in graphs:
            graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(e, want_large) and torch.equal(a, want_small) and torch.equal(b, want_small)
        del junk


def test_dropout_beside_its_inputs_in_one_buffer(deft):
    """Outputs that are x or add element for element, or lie between or right behind their rows, give what separate ones give."""
    rows, cols, p = 50, 24, 0.3
    g = torch.Generator(device="cuda").manual_seed(5)
    fresh = lambda *shape: torch.randn(*shape, device="cuda", generator=g)  # noqa: E731

    def check(x, y, add=None):
        want = torch.empty((rows, cols), dtype=y.dtype, device="cuda")
        deft.deft_dropout(x.clone(), want, add=None if add is None else add.clone(), p=p, seed=9)
        deft.deft_dropout(x, y, add=add, p=p, seed=9)
        assert torch.equal(y, want)

    buf = fresh(2 * rows + 1, 3 * cols)
    left, middle, right = (buf[:rows, i * cols:(i + 1) * cols] for i in range(3))
    check(left, middle, right)                                       # columns side by side
    check(right, left)
    half = buf.view(torch.bfloat16)[:rows, 3 * cols:4 * cols]        # the same pitch in bytes, other elements
    check(left, half)
    check(left, buf[1:2 * rows + 1:2, cols:2 * cols])                # twice the pitch, between the rows
    check(buf[:2 * rows:2, :cols], buf[1:2 * rows + 1:2, :cols], buf[1:2 * rows + 1:2, 2 * cols:])
    check(left, left)
    check(left, right, right)
    check(left, left, left)
    flat = fresh(2 * rows * cols)
    x, y = flat[:rows * cols].view(rows, cols), flat[rows * cols:].view(rows, cols)
    check(x, y)                                                      # right behind, and right before
    check(y, x)
    one = fresh(1, 3 * cols)
    out = torch.empty((1, cols), device="cuda")
    deft.deft_dropout(one[:, :cols], out, p=p, seed=9)
    deft.deft_dropout(one[:, :cols], one[:, :cols], p=p, seed=9)     # a single row has no pitch
    assert torch.equal(one[:, :cols], out)
    with pytest.raises(deft.DeftError):
        deft.deft_dropout(buf[:rows, :cols], buf[:rows, cols // 2:cols // 2 + cols], p=p)
    with pytest.raises(deft.DeftError):
        deft.deft_dropout(left, buf.view(torch.bfloat16)[:rows, :cols], p=p)
