"""The dense row operators from their definitions, in 64 bits.  Used by the tests; shares no code with the library."""
import math

import numpy as np
import torch

STEP = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}   # half a step, relative
TINY = {torch.float32: 2.0 ** -149, torch.bfloat16: 2.0 ** -133, torch.float16: 2.0 ** -24}   # a subnormal step
U = 2.0 ** -24                                                                             # a rounding in fp32


def close(got, want, tol):
    """got (any type) within tol (of the fp32 arithmetic) and one rounding to its type of want (64 bits); infinities and NaN equal."""
    g, w = got.double().cpu(), want.double().cpu()
    t = torch.as_tensor(tol).double().cpu() + STEP[got.dtype] * (w.abs() + torch.as_tensor(tol).double().cpu()) + TINY[got.dtype]
    most = torch.finfo(got.dtype).max * (1 + STEP[got.dtype])     # rounds to an infinity
    w = torch.where(w.abs() >= most, torch.copysign(torch.full_like(w, math.inf), w), w)
    finite = torch.isfinite(w)
    assert torch.equal(torch.isnan(g), torch.isnan(w)), "NaN in other places"
    assert torch.equal(g[torch.isinf(w)], w[torch.isinf(w)]), "infinities differ"
    err = ((g - w).abs() / t.expand_as(w))[finite]
    assert err.numel() == 0 or err.max().item() <= 1.0, "off by %.3g of the tolerance" % err.max().item()


def layer_norm(x, add=None, gamma=None, beta=None, eps=1e-5):
    """y, s, mean, rstd and the fp32 tolerance of y, mean and rstd."""
    s = x.double() if add is None else x.double() + add.double()
    n = s.shape[-1]
    mean = s.sum(-1, keepdim=True) / n
    d = s - mean
    var = (d * d).sum(-1, keepdim=True) / n
    r = 1.0 / torch.sqrt(var + eps)
    g = torch.ones(n, dtype=torch.float64, device=x.device) if gamma is None else gamma.double()
    b = torch.zeros(n, dtype=torch.float64, device=x.device) if beta is None else beta.double()
    y = d * r * g + b
    # sums of a row: at most 32 terms one after the other in a thread, nine halvings, sixteen warps: below 64 roundings; what
    # the first mean is off by is taken out again.  The addition's rounding counts by the size of the sum.
    h = (d * r).abs()
    tol = U * (64 * (1 + h) * g.abs() + 4 * (h * g.abs() + b.abs()))
    if add is not None:
        tol = tol + 2 * U * (s.abs() * r + s.abs().mean(-1, keepdim=True) * r) * g.abs()
    tol_mean = U * (2 * mean.abs() + 64 * d.abs().mean(-1, keepdim=True) + (2 * s.abs().mean(-1, keepdim=True) if add is not None else 0))
    tol_r = U * 64 * r + (U * 4 * (s.abs() * r).amax(-1, keepdim=True) * r if add is not None else 0)
    return y, s, mean.squeeze(-1), r.squeeze(-1), tol, tol_mean.squeeze(-1), tol_r.squeeze(-1)


def layer_norm_grad(dy, x, mean, rstd, gamma=None, add=None, scale=1.0):
    """dx, dgamma, dbeta and their fp32 tolerances."""
    n = x.shape[-1]
    dy, x = dy.double().reshape(-1, n), x.double().reshape(-1, n)
    r = rstd.double().view(-1, 1)
    h = (x - mean.double().view(-1, 1)) * r
    d = dy * (gamma.double() if gamma is not None else 1.0)
    c1, c2 = d.mean(1, keepdim=True), (d * h).mean(1, keepdim=True)
    dx = r * (d - c1 - h * c2)
    tol = U * r * (64 * (d.abs().mean(1, keepdim=True) + h.abs() * (d * h).abs().mean(1, keepdim=True)) + 8 * (d.abs() + c1.abs() + (h * c2).abs()))
    if add is not None:
        dx = dx + add.double().reshape(-1, n)
        tol = tol + U * 2 * dx.abs()
    # rows one after the other in a thread, teams of a CTA, up to 37 CTAs in a warp's lane and sixteen warps
    rows = x.shape[0]
    depth = 3 + rows // 148 + 1 + 64 + 37 + 16
    return (dx, (dy * h).sum(0) * scale, dy.sum(0) * scale, tol, U * depth * abs(scale) * (dy * h).abs().sum(0),
            U * depth * abs(scale) * dy.abs().sum(0))


def frequencies(rot, base=10000.0, scaling="plain", factor=1.0, original=0.0, low=1.0, high=32.0):
    """Radians per position."""
    out = []
    for i in range(rot // 2):
        b = base * factor ** (rot / (rot - 2.0)) if scaling == "base" and rot > 2 else base
        f = b ** (-2.0 * i / rot)
        if scaling == "linear":
            f /= factor
        if scaling == "parts":
            c = min(1.0, max(0.0, (original * f / (2.0 * math.pi) - low) / (high - low)))
            f *= c + (1.0 - c) / factor
        out.append(f)
    return np.array(out)


def rotary(x, turns, positions, interleaved=False, inverse=False, gain=1.0):
    """x: [..., tokens, heads, dim]; positions: int64 [..., tokens]; turns: numpy int64 bits.  The result and its fp32 tolerance."""
    rot = 2 * turns.size
    with np.errstate(over="ignore"):
        units = positions.cpu().numpy().astype(np.int64).view(np.uint64)[..., None] * turns.view(np.uint64)
    # the nearest whole turn away: 64 bits of a turn do not fit a double
    angle = torch.from_numpy(units.view(np.int64).astype(np.float64) * 2.0 ** -64 * (2.0 * math.pi)).unsqueeze(-2)
    c, s = angle.cos() * gain, angle.sin() * (-gain if inverse else gain)
    y = x.double().cpu().clone()
    v = y.clone()
    first, second = (slice(0, rot, 2), slice(1, rot, 2)) if interleaved else (slice(0, rot // 2), slice(rot // 2, rot))
    a, b = v[..., first], v[..., second]
    y[..., first], y[..., second] = a * c - b * s, a * s + b * c
    # cosine and sine: two units in the last place of up to 1 and what is left of the angle; two products, a sum, the gain
    tol = torch.zeros_like(y)
    tol[..., first] = tol[..., second] = 8 * U * abs(gain) * (a.abs() + b.abs())
    return y, tol


def distill(logits, ids, teacher, teacher_lse=None, temperature=1.0, weight=None, scale=1.0):
    """Row by row in numpy: loss, grad and their fp32 tolerances."""
    z_all, ids, t_all = logits.double().cpu().numpy(), ids.cpu().numpy(), teacher.double().cpu().numpy()
    rows, vocab = z_all.shape
    loss, grad, loss_tol, grad_tol = np.zeros(rows), np.zeros((rows, vocab)), np.zeros(rows), np.zeros((rows, vocab))
    with np.errstate(all="ignore"):
        for r in range(rows):
            w = 1.0 if weight is None else float(weight[r])
            if w == 0.0:
                continue
            z = z_all[r] / temperature
            top = z.max()
            e = np.exp(z - top)
            lse = np.log(e.sum()) + top
            p = np.exp(z - lse)
            valid = (ids[r] >= 0) & (ids[r] < vocab)
            t = t_all[r][valid] / temperature
            if teacher_lse is not None:
                log_q = t - float(teacher_lse[r])
            elif t.size and t.max() > -np.inf:
                log_q = t - (np.log(np.exp(t - t.max()).sum()) + t.max())
            else:
                log_q = np.full(t.size, -np.inf)
            q = np.exp(log_q)
            some = q != 0
            cols = ids[r][valid]
            value = float((q[some] * (log_q[some] - (z[cols[some]] - lse))).sum())
            target, beyond = np.zeros(vocab), np.ones(vocab, dtype=bool)
            np.add.at(target, cols, q)
            beyond[cols] = False
            left = rest = 0.0
            if teacher_lse is not None and e[beyond].size and z[beyond].max() > -np.inf:
                left = max(0.0, 1.0 - q.sum())
                m = z[beyond].max()
                log_rest = np.log(np.exp(z[beyond] - m).sum()) + m - lse
                if left > 0.0:
                    value += left * (np.log(left) - log_rest)
                rest = np.where(beyond, np.exp(z - lse - log_rest), 0.0)
            g = p * (q.sum() + left) - target - left * rest
            # exponents are rounded once and their factor once: relative to the sizes of the logits; sums below 128 roundings
            size = np.abs(z[np.isfinite(z)]).max() if np.isfinite(z).any() else 0.0
            size_t = np.abs(t[np.isfinite(t)]).max() if np.isfinite(t).any() else 0.0
            rel = U * (128 + 4 * size + 2 * size_t)
            logs = np.abs(log_q[some] - (z[cols[some]] - lse))
            logs = logs[np.isfinite(logs)]
            far = abs(np.log(left) - log_rest) if left > 0 else 0.0
            loss[r] = w * temperature ** 2 * value
            loss_tol[r] = abs(w) * temperature ** 2 * rel * (1 + (logs.max() if logs.size else 0.0) + far)
            grad[r] = scale * w * temperature * g
            # powers and their factors below 2^-126 are 0; they are relative to sums between 2^-20 and 2^30: at most 2^-96 is lost,
            # in each of an element's two terms
            grad_tol[r] = abs(scale * w * temperature) * (rel * (p * (q.sum() + left) + target + (left + 1.0) * rest) + 2.0 ** -95)
            if np.isnan(grad[r]).any():
                grad_tol[r] = 0.0
    return torch.from_numpy(loss), torch.from_numpy(grad), torch.from_numpy(loss_tol), torch.from_numpy(grad_tol)
