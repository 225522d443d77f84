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
