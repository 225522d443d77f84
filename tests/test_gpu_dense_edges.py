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
