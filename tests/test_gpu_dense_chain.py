"""The dense row operators as a model uses them together: lookup, norms, rotary attention and a distillation loss through to the
sparsification step; captured graphs, other streams, matrices beyond 2^31 elements."""
import concurrent.futures
import math

import pytest
import torch

from paper_2307_03500_b200 import build as deft_build
from tests import dense_plain as plain

deft_build.build()
from paper_2307_03500_b200 import deft  # noqa: E402
from paper_2307_03500_b200.pipeline import DeftStep, RowGradient  # noqa: E402

pytestmark = pytest.mark.gpu
F32 = torch.float32


def _rand(shape, seed, std=1.0, mean=0.0):
    return torch.empty(shape, device="cuda").normal_(mean, std, generator=torch.Generator(device="cuda").manual_seed(seed))


# One block of a small language model: vocabulary, width, heads, dim, batch, tokens
V, W, H, D, N, T, TOP = 501, 48, 3, 16, 2, 21, 7
SIZES = [V * W, W, W, W * 3 * W, W, W]            # table, first norm, projection, last norm


def _model64(params, ids, top, teacher, lse, angles):
    """The same model by automatic differentiation in 64 bits."""
    table, g1, b1, w, g2, b2 = params
    x = table[ids]
    h = torch.nn.functional.layer_norm(x, (W,), g1, b1, 1e-5)
    q, k, v = (h @ w).view(N, T, 3 * H, D).split(H, dim=2)

    def turn(t):
        a, b = t[..., :D // 2], t[..., D // 2:]
        c, s = angles.cos().unsqueeze(-2), angles.sin().unsqueeze(-2)
        return torch.cat([a * c - b * s, a * s + b * c], -1)
    q, k = turn(q), turn(k)
    a = torch.einsum("bqhd,bkhd->bhqk", q, k) / math.sqrt(D)
    a = a.masked_fill(torch.ones(T, T, dtype=torch.bool, device="cuda").triu(1), -math.inf).softmax(-1)
    x = x + torch.einsum("bhqk,bkhd->bqhd", a, v).reshape(N, T, W)
    y = torch.nn.functional.layer_norm(x, (W,), g2, b2, 1e-5)
    z = y @ table.t()
    log_p = torch.log_softmax(z, -1)
    log_q = teacher.double() - lse.double().unsqueeze(-1)
    rest = 1 - log_q.exp().sum(-1)
    inside = torch.zeros_like(z, dtype=torch.bool).scatter_(-1, top, True)
    log_rest = torch.logsumexp(log_p.masked_fill(inside, -math.inf), -1)
    kl = (log_q.exp() * (log_q - log_p.gather(-1, top))).sum(-1) + rest * (rest.log() - log_rest)
    return kl.mean()


class Block:
    """The same with the library's calls; every gradient goes to its part of the flat vector, the table's rows to the step."""

    def __init__(self):
        start = torch.tensor([0] + SIZES).cumsum(0).tolist()
        self.flat = torch.cat([_rand((V * W,), 1, 0.5), _rand((W,), 2, 0.1, 1.0), _rand((W,), 3, 0.1), _rand((3 * W * W,), 4, 0.15), _rand((W,), 5, 0.1, 1.0), _rand((W,), 6, 0.1)])
        self.grad = torch.zeros_like(self.flat)
        parts = lambda v: [v[a:b] for a, b in zip(start, start[1:])]  # noqa: E731
        self.p, self.g = parts(self.flat), parts(self.grad)
        self.ids = torch.randint(0, V, (N, T), generator=torch.Generator(device="cuda").manual_seed(7), device="cuda")
        t = _rand((N, T, V), 8, 2.0)
        self.teacher, self.top = t.topk(TOP, dim=-1)
        self.teacher, self.top, self.lse = self.teacher.contiguous(), self.top.contiguous(), torch.logsumexp(t, -1)
        self.turns = torch.from_numpy(deft.deft_rotary_frequencies(D)).cuda()
        self.ws = deft.alloc_layer_norm_workspace(N * T, W)
        new = lambda *shape: torch.empty(shape, device="cuda")  # noqa: E731
        self.x, self.h, self.s, self.y, self.dx, self.dy, self.dh = (new(N, T, W) for _ in range(7))
        self.m1, self.r1, self.m2, self.r2, self.loss = (new(N, T) for _ in range(5))
        self.z = new(N, T, V)

    def run(self):
        table, g1, b1, w, g2, b2 = self.p
        table, w = table.view(V, W), w.view(W, 3 * W)
        deft.deft_embed(table, self.ids, self.x)
        deft.deft_layer_norm(self.x, self.h, g1, b1, mean=self.m1, rstd=self.r1)
        qkv = (self.h @ w).view(N, T, 3 * H, D)
        deft.deft_rotary(qkv[:, :, :2 * H], qkv[:, :, :2 * H], self.turns)
        q, k, v = qkv.split(H, dim=2)
        a = torch.einsum("bqhd,bkhd->bhqk", q, k) / math.sqrt(D)
        a = a.masked_fill(torch.ones(T, T, dtype=torch.bool, device="cuda").triu(1), -math.inf).softmax(-1)
        o = torch.einsum("bhqk,bkhd->bqhd", a, v).reshape(N, T, W)
        deft.deft_layer_norm(self.x, self.y, g2, b2, add=o, sum=self.s, mean=self.m2, rstd=self.r2)
        torch.matmul(self.y, table.t(), out=self.z)
        deft.deft_distill(self.z, self.top, self.teacher, loss=self.loss, grad=self.z, teacher_lse=self.lse, scale=1.0 / (N * T))
        # backward: z now holds the logits' gradient
        torch.matmul(self.z.view(-1, V).t(), self.y.view(-1, W), out=self.g[0].view(V, W))     # the tied table's share by the loss
        torch.matmul(self.z, table, out=self.dy)
        deft.deft_layer_norm_grad(self.dy, self.s, self.m2, self.r2, self.dx, g2, grad_gamma=self.g[4], grad_beta=self.g[5], ws=self.ws)
        do = self.dx.view(N, T, H, D)
        da = torch.einsum("bqhd,bkhd->bhqk", do, v)
        ds = a * (da - (da * a).sum(-1, keepdim=True)) / math.sqrt(D)
        dqkv = torch.cat([torch.einsum("bhqk,bkhd->bqhd", ds, k), torch.einsum("bhqk,bqhd->bkhd", ds, q), torch.einsum("bhqk,bqhd->bkhd", a, do)], 2)
        deft.deft_rotary(dqkv[:, :, :2 * H], dqkv[:, :, :2 * H], self.turns, inverse=True)
        dqkv = dqkv.view(N * T, 3 * W)
        torch.matmul(self.h.view(-1, W).t(), dqkv, out=self.g[3].view(W, 3 * W))
        torch.matmul(dqkv.view(N, T, -1), w.t(), out=self.dh)
        deft.deft_layer_norm_grad(self.dh, self.x, self.m1, self.r1, self.dx, g1, add=self.dx, grad_gamma=self.g[1], grad_beta=self.g[2], ws=self.ws)
        return self.loss


def _want(b):
    params = [p.double().view(shape).requires_grad_() for p, shape in zip(b.p, [(V, W), (W,), (W,), (W, 3 * W), (W,), (W,)])]
    f = torch.from_numpy(plain.frequencies(D)).cuda()
    loss = _model64(params, b.ids, b.top, b.teacher, b.lse, torch.arange(T, device="cuda").double().unsqueeze(-1) * f)
    loss.backward()
    return loss.item(), [p.grad.reshape(-1) for p in params]


def test_a_block_from_lookup_to_the_step():
    torch.backends.cuda.matmul.allow_tf32 = False
    b = Block()
    loss = b.run().mean().item()
    want, grads = _want(b)
    # about thirty fp32 operations in a row, sums of up to 501 terms: 2^-24 times 2000 of a tensor's largest gradient
    tol = 2000 * plain.U
    assert abs(loss - want) <= tol * abs(want)
    for i in range(1, 6):
        assert (b.g[i].double() - grads[i]).abs().max() <= tol * grads[i].abs().max(), "gradient of tensor %d" % i
    # the lookup's share by rows on top of the tied output's: with the step's accumulation they give the whole gradient
    total = b.g[0].clone()
    deft.deft_embed_grad(b.dx, b.ids, total.view(V, W), deft.alloc_embed_workspace(N * T, V, W), accumulate=True)
    assert (total.double() - grads[0]).abs().max() <= tol * grads[0].abs().max()
    residual = torch.zeros_like(b.flat)
    whole = residual.clone()
    ds = DeftStep(SIZES, 2, 0.1, device="cuda")
    residual[:V * W] = b.g[0]                      # what the loss gave the table; the step adds the lookup's rows
    plan, outs = ds.step(residual, b.grad, 0, rows=[RowGradient(tensor=0, ids=b.ids.view(-1), grad_out=b.dx.view(-1, W))])
    got = torch.cat([residual, torch.zeros(0, device="cuda")])
    for val, idx in outs:
        got[idx] += val
    whole[:V * W], whole[V * W:] = total, b.grad[V * W:]
    assert torch.equal(got, whole) and sum(len(i) for _, i in outs) == plan.sum_k


def test_captured_and_replayed():
    """The block in a graph: replayed on new parameters it gives what an eager run gives, bit for bit; two graphs share a workspace in turn."""
    torch.backends.cuda.matmul.allow_tf32 = False
    b = Block()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        b.run()
    torch.cuda.synchronize()
    graphs = [torch.cuda.CUDAGraph() for _ in range(2)]
    for g in graphs:
        with torch.cuda.graph(g, stream=side):
            b.run()
    b.flat.mul_(0.9)
    b.ids.add_(1).remainder_(V)
    torch.cuda.synchronize()
    for g in graphs + graphs[:1]:
        b.grad.zero_()
        b.dx.zero_()
        g.replay()
        torch.cuda.synchronize()
        got = [t.clone() for t in (b.grad, b.dx, b.loss, b.z)]
        with torch.cuda.stream(side):
            b.run()
        torch.cuda.synchronize()
        assert all(torch.equal(x, y) for x, y in zip(got, (b.grad, b.dx, b.loss, b.z)))


def test_streams():
    """Calls take the current stream, or the one they are given."""
    x = _rand((4000, 512), 1)
    y, z = torch.empty_like(x), torch.empty_like(x)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        deft.deft_layer_norm(x, y)
    deft.deft_layer_norm(y, z, stream=s)
    ids, t = torch.zeros((4000, 1), dtype=torch.int64, device="cuda"), torch.zeros((4000, 1), device="cuda")
    s.wait_stream(torch.cuda.current_stream())
    deft.deft_distill(z, ids, t, grad=z, stream=s)
    turns = torch.from_numpy(deft.deft_rotary_frequencies(8)).cuda()
    s.wait_stream(torch.cuda.current_stream())
    deft.deft_rotary(z.view(4000, 64, 8), z.view(4000, 64, 8), turns, stream=s)
    torch.cuda.current_stream().wait_stream(s)
    want = [torch.empty_like(x) for _ in range(2)]
    deft.deft_layer_norm(x, want[0])
    deft.deft_layer_norm(want[0], want[1])
    deft.deft_distill(want[1], ids, t, grad=want[1])
    deft.deft_rotary(want[1].view(4000, 64, 8), want[1].view(4000, 64, 8), turns)
    assert torch.equal(z, want[1])


def test_calls_from_two_threads():
    """Host threads that call the same kernels with different needs of shared memory, each on a stream of its own."""
    def calls(cols, vocab, seed):
        stream = torch.cuda.Stream()
        with torch.cuda.stream(stream):
            x, z = _rand((9, cols), seed), _rand((9, vocab), seed + 1)
            y, dx, w, g = torch.empty_like(x), torch.empty_like(x), torch.empty((2, cols), device="cuda"), torch.empty_like(z)
            mean, rstd, loss = torch.empty(9, device="cuda"), torch.empty(9, device="cuda"), torch.empty(9, device="cuda")
            ids, t = torch.zeros((9, 1), dtype=torch.int64, device="cuda"), torch.zeros((9, 1), device="cuda")
            ws = deft.alloc_layer_norm_workspace(9, cols)
            for _ in range(300):
                deft.deft_layer_norm(x, y, mean=mean, rstd=rstd)
                deft.deft_layer_norm_grad(x, x, mean, rstd, dx, grad_gamma=w[0], grad_beta=w[1], ws=ws)
                deft.deft_distill(z, ids, t, loss, g)
            stream.synchronize()
        return y, dx, w, g, loss
    sizes = [(16384, 262144, 1), (8192, 120000, 3), (12288, 180000, 5)]
    want = [calls(*s) for s in sizes]
    with concurrent.futures.ThreadPoolExecutor(len(sizes)) as pool:
        got = list(pool.map(lambda s: calls(*s), sizes))
    for a, b in zip(want, got):
        assert all(torch.equal(u, v) for u, v in zip(a, b))


def test_matrices_beyond_31_bits():
    """Offsets beyond 2^31 elements: the last rows of large matrices."""
    rows, cols = 2 ** 18 + 37, 8200
    x = torch.zeros((rows, cols), dtype=torch.bfloat16, device="cuda")
    tail = slice(rows - 5, rows)
    x[tail] = _rand((5, cols), 1).bfloat16()
    last = x[tail].clone()
    mean, rstd = torch.empty(rows, device="cuda"), torch.empty(rows, device="cuda")
    deft.deft_layer_norm(x, x, mean=mean, rstd=rstd)
    want, _, m, r, tol, tol_m, tol_r = plain.layer_norm(last)
    plain.close(x[tail], want, tol)
    plain.close(mean[tail], m, tol_m)
    assert not x[:rows - 5].any()
    x[tail] = last
    dy = torch.zeros((rows, cols), dtype=torch.bfloat16, device="cuda")
    dy[tail] = _rand((5, cols), 2).bfloat16()
    dlast = dy[tail].clone()
    w = torch.empty(2 * cols, device="cuda")
    deft.deft_layer_norm_grad(dy, x, mean, rstd, dy, grad_gamma=w[:cols], grad_beta=w[cols:], ws=deft.alloc_layer_norm_workspace(rows, cols))
    dx, dg, db, tol, tol_g, tol_b = plain.layer_norm_grad(dlast, last, mean[tail], rstd[tail])
    plain.close(dy[tail], dx, tol)
    plain.close(w, torch.cat([dg, db]), torch.cat([tol_g, tol_b]))
    turns = torch.from_numpy(deft.deft_rotary_frequencies(200)).cuda()
    x[tail] = last
    heads = x.view(rows, 41, 200)
    deft.deft_rotary(heads, heads, turns)
    want, tol = plain.rotary(last.view(5, 41, 200), turns.cpu().numpy(), torch.arange(rows - 5, rows))
    plain.close(heads[tail], want, tol)
    assert not heads[:rows - 5].any()
    x[tail] = last
    ids, t = torch.randint(0, cols, (rows, 2), device="cuda"), torch.zeros((rows, 2), device="cuda")
    loss = torch.empty(rows, device="cuda")
    deft.deft_distill(x, ids, t, loss=loss, grad=x)
    want, grad, tol_l, tol_g = plain.distill(last, ids[tail], t[tail])
    plain.close(loss[tail], want, tol_l)
    plain.close(x[tail], grad, tol_g)
