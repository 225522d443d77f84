"""The checks of a step with row gradients, without a GPU: the device calls are replaced by a recorder, and a refused call
must not have issued any."""
from dataclasses import replace

import numpy as np
import pytest
import torch

from paper_2307_03500_b200 import build as deft_build

deft_build.build()
from paper_2307_03500_b200 import deft  # noqa: E402
from paper_2307_03500_b200.pipeline import DeftStep, RowGradient  # noqa: E402

VOCAB, WIDTH, N_TOKENS = 30, 8, 6


@pytest.fixture
def step(monkeypatch):
    """A DeftStep over [12, VOCAB * WIDTH, 100] elements on the host; step.calls: what would have gone to the library."""
    sizes = [12, VOCAB * WIDTH, 100]
    ds = object.__new__(DeftStep)
    ds.device, ds.N, ds.n_g = torch.device("cpu"), 2, sum(sizes)
    ds.tensor_start = np.concatenate([[0], np.cumsum(sizes)])
    ds.layer_start_d = torch.from_numpy(ds.tensor_start)
    ds.calls = []
    monkeypatch.setattr(deft, "_device", lambda *tensors: 0)
    monkeypatch.setattr(deft, "_call", lambda name, device, stream, *args: ds.calls.append((name, stream, args)))
    return ds


def _row(**kw):
    row = RowGradient(1, torch.arange(N_TOKENS), torch.ones(N_TOKENS, WIDTH), scale=0.5, p=0.25, seed=3)
    return replace(row, **kw)


def test_good_rows_reach_the_call(step):
    e = torch.zeros(step.n_g)
    parts = step.add_rows(e, [_row(), _row(seed=-1, offset=2 ** 64 + 5)])
    assert parts.tolist() == [[12, 12 + VOCAB * WIDTH]] and len(step.calls) == 2
    for (name, stream, args), (seed, offset) in zip(step.calls, ((3, 0), (2 ** 64 - 1, 5))):
        assert (name, stream) == ("deft_embed_grad", None)
        assert args[1:3] == (deft.F32, WIDTH) and args[4:14] == (8, N_TOKENS, VOCAB, WIDTH, -1, 0.5, 0.25, seed, offset, None)
        assert args[14:16] == (e[12:].data_ptr(), 1) and args[17] >= deft.deft_embed_workspace_bytes(N_TOKENS, VOCAB, WIDTH)


@pytest.mark.parametrize("bad", [
    dict(seed="x"), dict(offset=None), dict(skip_id="x"), dict(scale=None), dict(scale=float("inf")), dict(p=1.0), dict(p=float("nan")),
    dict(tensor=3), dict(tensor=0), dict(ids=torch.arange(5)), dict(grad_out=torch.ones(N_TOKENS, WIDTH).double()),
    dict(grad_out=torch.empty(2 ** 30 + 8, dtype=torch.bfloat16).as_strided((2, WIDTH), (2 ** 30, 1)), ids=torch.arange(2)),
], ids=lambda kw: "-".join(kw))
def test_a_refused_row_leaves_the_rows_before_it_out(step, bad):
    """What the second gradient's own call would refuse is refused before the first one is added."""
    with pytest.raises((ValueError, TypeError, deft.DeftError)):
        step.add_rows(torch.zeros(step.n_g), [_row(), _row(**bad)])
    assert step.calls == []


def test_no_call_uses_the_workspace_of_another_stream(step, monkeypatch):
    """add_rows does not wait for the GPU: a workspace that two streams share, or one that is let go on another stream than it is
    used on, would be written by two calls at once."""
    current, made, empty = ["default"], {}, torch.empty

    class On:
        def __init__(self, stream):
            self.stream = stream

        def __enter__(self):
            current.append(self.stream)

        def __exit__(self, *exc):
            current.pop()

    def recorded(*args, **kw):
        t = empty(*args, **kw)
        made[t.data_ptr()] = (current[-1], t)        # (kept: its memory is not given out again)
        return t

    monkeypatch.setattr(torch.cuda, "stream", On)
    monkeypatch.setattr(torch, "empty", recorded)
    e, more = torch.zeros(step.n_g), _row(ids=torch.arange(200) % VOCAB, grad_out=torch.ones(200, WIDTH))
    used = {}
    for stream, row in (("A", _row()), (None, _row()), ("B", more), ("A", _row()), (None, more), ("A", more)):
        step.calls.clear()
        step.add_rows(e, [row, row], stream=stream)
        for _, on, args in step.calls:
            ws = args[16]
            assert made[ws][0] == (stream or "default") and on == stream
            used.setdefault(ws, set()).add(stream)
    assert all(len(streams) == 1 for streams in used.values())


@pytest.mark.parametrize("scale,p,ok", [(1e39, 0.0, False), (-1e308, 0.0, False), (2.0 ** 128 - 2.0 ** 103, 0.0, False), (2.0 ** 128 - 2.0 ** 104, 0.0, True),
                                        (3e38, 0.25, False), (-2.5e38, 0.25, True), (1e35, 0.9999, False), (1e33, 1 - 1e-9, True), (1e34, 1 - 1e-9, False)])
def test_scales_that_overflow_fp32_are_refused_before_the_first_row(step, scale, p, ok):
    """The same answer as the call's own, whose checks do not need a device when there are no tokens."""
    status = deft.lib().deft_embed_grad(None, deft.F32, 0, None, 8, 0, VOCAB, WIDTH, -1, scale, p, 0, 0, None, 0x10000, 1, 0x10000, 1 << 30, None)
    assert status == (deft.OK if ok else deft.ERR_INVALID_ARG)
    rows = [_row(), _row(scale=scale, p=p)]
    if ok:
        step.add_rows(torch.zeros(step.n_g), rows)
    else:
        with pytest.raises(ValueError):
            step.add_rows(torch.zeros(step.n_g), rows)
    assert len(step.calls) == (2 if ok else 0)


def test_rows_made_on_the_way_live_until_their_calls(step, monkeypatch):
    """Rows may come from a generator, which keeps none of them."""
    import weakref
    made = []

    def rows():
        for _ in range(3):
            row = _row(grad_out=torch.ones(N_TOKENS, WIDTH))
            made.append((weakref.ref(row.grad_out), row.grad_out.data_ptr()))
            yield row
            del row

    def call(name, device, stream, *args):
        ref, ptr = made[len(step.calls)]
        assert ref() is not None and args[0] == ptr
        step.calls.append(args)

    monkeypatch.setattr(deft, "_call", call)
    step.add_rows(torch.zeros(step.n_g), rows())
    assert len(step.calls) == 3


class _OnDevice:
    """What the binding asks of a CUDA tensor."""
    is_cuda = True

    def __init__(self, device, dtype, n=8):
        self.device, self.dtype, self.n = device, dtype, n

    def get_device(self):
        return self.device

    def is_contiguous(self):
        return True

    def numel(self):
        return self.n

    def element_size(self):
        return 8 if self.dtype in (torch.int64, torch.float64) else 4

    def data_ptr(self):
        return 0x10000


def test_norms_with_parts_on_the_device_of_the_tensors(monkeypatch):
    """The call runs on the tensors' one device, which need not be the current one, and on that device's stream."""
    issued = []
    monkeypatch.setattr(deft, "_call", lambda name, device, stream, *args: issued.append((name, device, stream, args)), raising=False)
    make = lambda devices: [_OnDevice(d, t) for d, t in  # noqa: E731
                            zip(devices, (torch.float32, torch.float32, torch.int64, torch.float64, torch.uint8))]
    for wrong in range(5):
        e, g, start, norms, ws = make([2 if i == wrong else 1 for i in range(5)])
        with pytest.raises(ValueError):
            deft.deft_layer_norms_part(e, g, [(0, 4)], start, norms, ws)
    assert not issued
    e, g, start, norms, ws = make([1] * 5)
    deft.deft_layer_norms_part(e, g, [(0, 4)], start, norms, ws, stream="s")
    deft.deft_layer_norms_part(e, None, [], start, norms, ws)
    assert [i[:3] for i in issued] == [("deft_layer_norms_part", 1, "s"), ("deft_layer_norms_part", 1, None)]
