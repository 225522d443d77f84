"""The dense row operators of a language model between its lookup and its loss, as measured cases.

Their gradients are what the flat gradient vector holds beside the embedding's rows.

``norm``     layer norm of every row, of a residual stream with a branch added to it (the sum is kept) or of x alone
``normgrad`` its backward pass: the input's gradient, with the residual stream's added, and the gradients of weight and
             bias summed over the rows into their parts of the flat gradient vector (written) or of the residual (added)
``rotary``   rotary positions of the heads of a [batch, tokens, heads, dim] tensor: pairs in halves or interleaved, of a
             part of the head, with frequencies for long contexts; ``inverse`` is the backward pass
``distill``  distillation from a teacher's top logits: T^2 KL(teacher || student) per row and its gradient in one pass,
             the teacher renormalised over its entries, or with one class for the rest of the vocabulary (``tail``)

With ``own = False`` the operators are computed in their plain form; with ``own = True`` by this repository's
library.
"""
import math

import torch

own = False

TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
SIZE = {"f32": 4, "bf16": 2, "f16": 2}
EPS = 1e-5


def listed():
    return [
        # one sequence's last tokens, pre-norm: latency counts
        _norm("norm_64x1024", 64, 1024, "bf16", "bf16", True),
        # a BERT-large batch, 32 sequences of 512 tokens: the norm behind a block, branch added
        _norm("norm_bert_16k", 16384, 1024, "bf16", "bf16", True),
        # odd rows that start on no vector boundary, fp32 activations handed on in bf16
        _norm("norm_odd_5003", 5003, 1027, "f32", "bf16", False),
        # the BERT batch's backward pass, gradients written to the flat vector
        _normgrad("normgrad_bert_16k", 16384, 1024, "bf16", "bf16", True, False),
        # a large GPT-2-medium batch, 128 sequences of 1024 tokens, accumulated into the residual
        _normgrad("normgrad_gpt2_128k", 131072, 1024, "bf16", "bf16", False, True),
        # the LSTM model's width in fp32, one step of 20 sequences of 35 tokens
        _normgrad("normgrad_700x1500", 700, 1500, "f32", "f32", True, True),
        # one new token of each of 48 running sequences, far positions, frequencies for a context eight times as long
        _rotary("rotary_48_tokens", 48, 1, 24, 128, 128, "bf16", "half", "parts", False, True),
        # queries and keys of a GPT-2-medium batch out of the fused projection, 16 sequences of 1024 tokens
        _rotary("rotary_gpt2_16k", 16, 1024, 32, 64, 64, "bf16", "half", "plain", False, False),
        # the backward pass of an interleaved rotation of a quarter of wide fp32 heads, packed sequences
        _rotary("rotary_back_odd", 1, 5003, 12, 160, 40, "f32", "interleaved", "linear", True, True),
        # one evaluation batch of the LSTM model's vocabulary, no gradient, renormalised
        _distill("distill_eval_700", 700, 33278, "f32", 8, False, False, 1.0, 0.0, 8),
        # a fine-tuning batch over a BERT vocabulary with padding rows, teacher's own normaliser kept
        _distill("distill_bert_2k", 2048, 30522, "bf16", 32, True, True, 2.0, 0.25, 8),
        # eight sequences of 1024 tokens over GPT-2's vocabulary, whose rows start on no vector boundary
        _distill("distill_gpt2_8k", 8192, 50257, "bf16", 64, True, True, 2.0, 0.0, 4),
    ]


def _norm(name, rows, width, x, y, add):
    return {"name": name, "op": "norm", "n": rows, "width": width, "x": x, "y": y, "add": add}


def _normgrad(name, rows, width, dy, x, add, accumulate):
    return {"name": name, "op": "normgrad", "n": rows, "width": width, "dy": dy, "x": x, "add": add, "accumulate": accumulate}


def _rotary(name, batch, tokens, heads, dim, rot, kind, layout, scaling, inverse, positions):
    return {"name": name, "op": "rotary", "batch": batch, "n": tokens, "heads": heads, "dim": dim, "rot": rot, "x": kind,
            "layout": layout, "scaling": scaling, "inverse": inverse, "positions": positions}


def _distill(name, rows, vocab, kind, top, tail, grad, temperature, masked, id_bytes):
    return {"name": name, "op": "distill", "n": rows, "vocab": vocab, "x": kind, "top": top, "tail": tail, "grad": grad,
            "temperature": temperature, "masked": masked, "id_bytes": id_bytes}


def draw(rng):
    def log(lo, hi):
        return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))

    def kind():
        return rng.choice(["bf16", "bf16", "f16", "f32"])

    op = rng.choice(["norm", "normgrad", "normgrad", "rotary", "distill", "distill"])
    if op in ("norm", "normgrad"):
        width = log(16, 8192)
        if rng.random() < 0.6:
            width = max(16, width // 8 * 8)
        rows = log(1, min(131072, 131072 * 1024 // width))
        x = kind()
        if op == "norm":
            c = _norm("", rows, width, x, rng.choice([x, x, "bf16", "f32"]), rng.random() < 0.5)
        else:
            c = _normgrad("", rows, width, rng.choice([x, x, "bf16", "f32"]), x, rng.random() < 0.5, rng.random() < 0.5)
    elif op == "rotary":
        dim = 2 * log(16, 128)
        if rng.random() < 0.6:
            dim = dim // 16 * 16
        rot = dim if rng.random() < 0.6 else 2 * rng.randint(1, dim // 2)
        heads = rng.randint(1, 64)
        batch = log(1, 64)
        tokens = log(1, max(1, (1 << 27) // (batch * heads * dim)))
        c = _rotary("", batch, tokens, heads, dim, rot, kind(), rng.choice(["half", "interleaved"]),
                    rng.choice(["plain", "linear", "base", "parts"]), rng.random() < 0.4, rng.random() < 0.5)
    else:
        vocab = log(1000, 131072)
        if rng.random() < 0.5:
            vocab = vocab // 8 * 8
        x = kind()
        c = _distill("", log(1, min(65536, 8192 * 50257 * 2 // (vocab * SIZE[x]))), vocab, x, log(1, 128), rng.random() < 0.5,
                     rng.random() < 0.8, rng.choice([1.0, 1.0, 2.0, 4.0]), rng.choice([0.0, 0.25]), rng.choice([4, 8]))
    del c["name"]
    return c


# ---- inputs ----------------------------------------------------------------------------------
def _generator(seed):
    return torch.Generator(device="cuda").manual_seed(1000003 * int(seed) + 29)


def _normal(g, shape, kind, std=1.0, mean=0.0):
    return torch.empty(shape, dtype=TYPES[kind], device="cuda").normal_(mean, std, generator=g)


def prepare(case, seed):
    g = _generator(seed)
    c = dict(case)
    {"norm": _prepare_norm, "normgrad": _prepare_normgrad, "rotary": _prepare_rotary, "distill": _prepare_distill}[c["op"]](c, g)
    return c


def _activations(g, n, width, kind):
    """Rows of a residual stream: a few columns far from zero, as trained models have them."""
    x = _normal(g, (n, width), kind)
    loud = torch.randint(0, width, (max(1, width // 256),), generator=g, device="cuda")
    x[:, loud] += 8.0
    return x


def _prepare_norm(c, g):
    n, width = c["n"], c["width"]
    c["x_t"] = _activations(g, n, width, c["x"])
    c["add_t"] = _normal(g, (n, width), c["x"], 0.5) if c["add"] else None
    c["sum_t"] = torch.empty_like(c["x_t"]) if c["add"] else None
    c["gamma"], c["beta"] = _normal(g, (width,), "f32", 0.1, 1.0), _normal(g, (width,), "f32", 0.1)
    c["y_t"] = torch.empty((n, width), dtype=TYPES[c["y"]], device="cuda")
    c["mean"], c["rstd"] = torch.empty(n, device="cuda"), torch.empty(n, device="cuda")


def _prepare_normgrad(c, g):
    n, width = c["n"], c["width"]
    c["x_t"] = _activations(g, n, width, c["x"])
    c["dy_t"] = _normal(g, (n, width), c["dy"], 0.01)
    c["add_t"] = _normal(g, (n, width), c["x"], 0.01) if c["add"] else None
    c["gamma"] = _normal(g, (width,), "f32", 0.1, 1.0)
    c["dx_t"] = torch.empty_like(c["x_t"])
    # what the forward pass has kept
    c["mean"], c["rstd"] = torch.empty(n, device="cuda"), torch.empty(n, device="cuda")
    for a in range(0, n, 8192):
        x = c["x_t"][a:a + 8192].double()
        c["mean"][a:a + 8192] = x.mean(1)
        c["rstd"][a:a + 8192] = (x.var(1, unbiased=False) + EPS).rsqrt()
    # weight and bias follow one another in the flat vector
    c["flat"] = _normal(g, (2 * width,), "f32", 0.01)
    if own:
        from paper_2307_03500_b200 import deft
        c["ws"] = deft.alloc_layer_norm_workspace(n, width, "cuda")


# The rotary frequencies of each kind of case: base 10000, contexts eight times as long as the 2048 tokens trained on.
BASE, FACTOR, ORIGINAL, LOW, HIGH = 10000.0, 8.0, 2048, 1.0, 32.0


def _prepare_rotary(c, g):
    b, n, heads, dim = c["batch"], c["n"], c["heads"], c["dim"]
    # the rotated heads come first in the fused projection; the values' heads lie behind them
    fused = _normal(g, (b, n, heads + heads // 2, dim), c["x"])
    c["fused"], c["x_t"] = fused, fused[:, :, :heads]
    c["pos"] = None
    if c["positions"]:
        if n == 1:
            c["pos"] = torch.randint(0, int(ORIGINAL * FACTOR), (b, 1), generator=g, device="cuda")
        else:   # packed sequences: positions start again inside a row
            start = torch.randint(1, n + 1, (b, 1), generator=g, device="cuda")
            t = torch.arange(n, device="cuda").view(1, -1)
            c["pos"] = torch.where(t >= start, t - start, t).contiguous()
    c["y_t"] = torch.empty((b, n, heads, dim), dtype=TYPES[c["x"]], device="cuda")
    if own:
        from paper_2307_03500_b200 import deft
        turns = deft.deft_rotary_frequencies(c["rot"], BASE, scaling=c["scaling"], factor=FACTOR, original=ORIGINAL, low=LOW, high=HIGH)
        c["turns"] = torch.from_numpy(turns).cuda()


def _prepare_distill(c, g):
    n, vocab, top = c["n"], c["vocab"], c["top"]
    c["x_t"] = torch.empty((n, vocab), dtype=TYPES[c["x"]], device="cuda")
    c["ids"] = torch.empty((n, top), dtype=torch.int64 if c["id_bytes"] == 8 else torch.int32, device="cuda")
    c["teacher"] = torch.empty((n, top), dtype=torch.float32, device="cuda")
    c["teacher_lse"] = torch.empty(n, device="cuda") if c["tail"] else None
    step = max(1, (1 << 27) // vocab)
    for a in range(0, n, step):
        part = c["x_t"][a:a + step]
        part.normal_(0.0, 2.0, generator=g)
        # the student has learnt part of what the teacher says, and both favour a few tokens of a row
        peak = torch.randint(0, vocab, (part.shape[0], 4), generator=g, device="cuda")
        part.scatter_add_(1, peak, torch.full_like(peak, 9, dtype=part.dtype))
        t = part.float() + torch.empty(part.shape, device="cuda").normal_(0.0, 1.0, generator=g)
        c["teacher"][a:a + step], ids = t.topk(top, dim=1)
        c["ids"][a:a + step] = ids
        if c["tail"]:
            c["teacher_lse"][a:a + step] = torch.logsumexp(t / c["temperature"], 1)
    # rows of padding or prompts count nothing
    c["weight"] = (torch.rand(n, generator=g, device="cuda") >= c["masked"]).float() if c["masked"] else None
    # the mean over the rows, with the loss scale that keeps fp16 gradients in range
    c["scale"] = (65536.0 if c["x"] == "f16" else 1.0) / n
    c["loss"] = torch.empty(n, device="cuda")
    c["grad_t"] = torch.empty_like(c["x_t"]) if c["grad"] else None


# ---- one pass --------------------------------------------------------------------------------
def run(state):
    table = {"norm": (_norm_plain, _norm_own), "normgrad": (_normgrad_plain, _normgrad_own), "rotary": (_rotary_plain, _rotary_own),
             "distill": (_distill_plain, _distill_own)}
    return table[state["op"]][1 if own else 0](state)


def _norm_plain(c):
    s = c["x_t"].float()
    if c["add"]:
        s = s + c["add_t"].float()
    mean = s.mean(1)
    d = s - mean.view(-1, 1)
    rstd = 1.0 / (d.square().mean(1) + EPS).sqrt()
    out = {"y": (d * rstd.view(-1, 1) * c["gamma"] + c["beta"]).to(c["y_t"].dtype), "mean": mean, "rstd": rstd}
    if c["add"]:
        out["sum"] = s.to(c["x_t"].dtype)
    return out


def _norm_own(c):
    from paper_2307_03500_b200 import deft
    deft.deft_layer_norm(c["x_t"], c["y_t"], c["gamma"], c["beta"], eps=EPS, add=c["add_t"], sum=c["sum_t"], mean=c["mean"], rstd=c["rstd"])
    out = {"y": c["y_t"], "mean": c["mean"], "rstd": c["rstd"]}
    if c["add"]:
        out["sum"] = c["sum_t"]
    return out


def _normgrad_plain(c):
    dy, width = c["dy_t"].float(), c["width"]
    h = (c["x_t"].float() - c["mean"].view(-1, 1)) * c["rstd"].view(-1, 1)
    a = dy * c["gamma"]
    dx = (a - a.mean(1, keepdim=True) - h * (a * h).mean(1, keepdim=True)) * c["rstd"].view(-1, 1)
    if c["add"]:
        dx = dx + c["add_t"].float()
    got = torch.cat([(dy * h).sum(0), dy.sum(0)])
    flat = c["flat"].add_(got) if c["accumulate"] else c["flat"].copy_(got)
    return {"dx": dx.to(c["dx_t"].dtype), "gamma": flat[:width], "beta": flat[width:]}


def _normgrad_own(c):
    from paper_2307_03500_b200 import deft
    gamma, beta = c["flat"][:c["width"]], c["flat"][c["width"]:]
    deft.deft_layer_norm_grad(c["dy_t"], c["x_t"], c["mean"], c["rstd"], c["dx_t"], c["gamma"], add=c["add_t"], grad_gamma=gamma,
                              grad_beta=beta, ws=c["ws"], accumulate=c["accumulate"])
    return {"dx": c["dx_t"], "gamma": gamma, "beta": beta}


def _frequencies(c):
    """Radians per position of every pair."""
    rot = c["rot"]
    i = torch.arange(rot // 2, dtype=torch.float64, device="cuda")
    base = BASE * FACTOR ** (rot / (rot - 2.0)) if c["scaling"] == "base" and rot > 2 else BASE
    f = base ** (-2.0 * i / rot)
    if c["scaling"] == "linear":
        f = f / FACTOR
    elif c["scaling"] == "parts":
        keep = ((f * (ORIGINAL / (2.0 * math.pi)) - LOW) / (HIGH - LOW)).clamp(0.0, 1.0)
        f = f * keep + f / FACTOR * (1.0 - keep)
    return f


def _rotary_plain(c):
    n, rot = c["n"], c["rot"]
    x = c["x_t"].float()
    pos = torch.arange(n, device="cuda").view(1, -1) if c["pos"] is None else c["pos"]
    # angles of far positions need 64 bits
    angle = pos.double().unsqueeze(-1) * _frequencies(c)
    cos, sin = angle.cos().float().unsqueeze(2), angle.sin().float().unsqueeze(2)
    if c["inverse"]:
        sin = -sin
    if c["layout"] == "half":
        a, b = x[..., :rot // 2], x[..., rot // 2:rot]
        turned = torch.cat([a * cos - b * sin, a * sin + b * cos], -1)
    else:
        a, b = x[..., 0:rot:2], x[..., 1:rot:2]
        turned = torch.stack([a * cos - b * sin, a * sin + b * cos], -1).flatten(-2)
    return torch.cat([turned, x[..., rot:]], -1).to(c["y_t"].dtype)


def _rotary_own(c):
    from paper_2307_03500_b200 import deft
    deft.deft_rotary(c["x_t"], c["y_t"], c["turns"], positions=c["pos"], interleaved=c["layout"] == "interleaved", inverse=c["inverse"])
    return c["y_t"]


def _distill_plain(c):
    t = c["temperature"]
    z = c["x_t"].float() / t
    ids = c["ids"].long()
    # the loss is what is left of logarithms that nearly cancel: 64 bits for the entries, log q by the teacher's
    # normaliser or by that of its entries
    q = c["teacher"].double() / t
    q = q - (c["teacher_lse"].double().view(-1, 1) if c["tail"] else (q - q[:, :1]).exp().sum(1, keepdim=True).log() + q[:, :1])
    z = z - z.amax(1, keepdim=True)
    chosen = z.gather(1, ids)
    e = z.exp()
    total = e.sum(1, keepdim=True)
    prob = q.exp()
    loss = (prob * (q - chosen.double() + total.double().log())).sum(1)
    mass, rest = 1.0, 0.0
    if c["tail"]:
        outside = e.scatter(1, ids, 0.0).sum(1, keepdim=True)
        left = (1.0 - prob.sum(1, keepdim=True)).clamp(min=0.0)
        mass = prob.sum(1, keepdim=True) + left
        term = left * (left.log() - outside.double().log() + total.double().log())
        loss = loss + torch.where(left > 0, term, torch.zeros_like(term)).squeeze(1)
        mass, rest = mass.float(), (left / outside).float()
    weight = torch.ones(c["n"], device="cuda") if c["weight"] is None else c["weight"]
    out = {"loss": (loss * weight * (t * t)).float()}
    if c["grad"]:
        factor = weight.view(-1, 1) * (t * c["scale"])
        inside = e.gather(1, ids) * (mass / total) - prob.float()
        out["grad"] = e.mul_(mass / total - rest).scatter_(1, ids, inside).mul_(factor).to(c["x_t"].dtype)
    return out


def _distill_own(c):
    from paper_2307_03500_b200 import deft
    deft.deft_distill(c["x_t"], c["ids"], c["teacher"], loss=c["loss"], grad=c["grad_t"], teacher_lse=c["teacher_lse"],
                      temperature=c["temperature"], weight=c["weight"], scale=c["scale"])
    return {"loss": c["loss"], "grad": c["grad_t"]} if c["grad"] else {"loss": c["loss"]}


# ---- what one pass cannot do without -----------------------------------------------------------
def work(case):
    c = case
    if c["op"] == "norm":
        cells, x = c["n"] * c["width"], SIZE[c["x"]]
        return {"bytes": cells * (x + SIZE[c["y"]] + (2 * x if c["add"] else 0)) + 8 * (c["n"] + c["width"]), "flops": 8 * cells}
    if c["op"] == "normgrad":
        cells, x = c["n"] * c["width"], SIZE[c["x"]]
        return {"bytes": cells * (SIZE[c["dy"]] + 2 * x + (x if c["add"] else 0)) + 8 * c["n"] + (20 if c["accumulate"] else 12) * c["width"],
                "flops": 14 * cells}
    if c["op"] == "rotary":
        tokens, size = c["batch"] * c["n"], SIZE[c["x"]]
        return {"bytes": tokens * (2 * c["heads"] * c["dim"] * size + (8 if c["positions"] else 0)) + 4 * c["rot"],
                "flops": 3 * tokens * c["heads"] * c["rot"]}
    cells, size = c["n"] * c["vocab"], SIZE[c["x"]]
    read = (1.0 - c["masked"]) * (cells * size + c["n"] * c["top"] * (c["id_bytes"] + 4))
    return {"bytes": int(read + (cells * size if c["grad"] else 0) + c["n"] * (4 + (4 if c["tail"] else 0) + (4 if c["masked"] else 0))),
            "flops": int((1.0 - c["masked"]) * cells * (8 if c["grad"] else 5))}


# ---- the definition in 64 bits -----------------------------------------------------------------
def exact(case, seed):
    s = prepare(case, seed)
    return {"norm": _norm_exact, "normgrad": _normgrad_exact, "rotary": _rotary_exact, "distill": _distill_exact}[s["op"]](s)


def _blocks(n, width):
    step = max(1, (1 << 24) // width)
    return [(a, min(n, a + step)) for a in range(0, n, step)]


def _norm_exact(s):
    n, width = s["n"], s["width"]
    out = {k: torch.empty((n, width) if k in ("y", "sum") else n, dtype=torch.float64, device="cuda")
           for k in (("y", "mean", "rstd", "sum") if s["add"] else ("y", "mean", "rstd"))}
    for a, b in _blocks(n, width):
        v = s["x_t"][a:b].double()
        if s["add"]:
            v += s["add_t"][a:b].double()
            out["sum"][a:b] = v
        var, mean = torch.var_mean(v, 1, correction=0, keepdim=True)
        r = torch.rsqrt(var + EPS)
        out["y"][a:b] = torch.addcmul(s["beta"].double(), (v - mean) * r, s["gamma"].double())
        out["mean"][a:b], out["rstd"][a:b] = mean[:, 0], r[:, 0]
    return out


def _normgrad_exact(s):
    n, width = s["n"], s["width"]
    dx = torch.empty((n, width), dtype=torch.float64, device="cuda")
    gamma, beta = (s["flat"].double().view(2, width) if s["accumulate"] else torch.zeros((2, width), dtype=torch.float64, device="cuda"))
    gamma, beta = gamma.clone(), beta.clone()
    w = s["gamma"].double()
    for a, b in _blocks(n, width):
        r = s["rstd"][a:b, None].double()
        h = (s["x_t"][a:b].double() - s["mean"][a:b, None].double()) * r
        d = s["dy_t"][a:b].double()
        gamma += torch.einsum("rc,rc->c", d, h)
        beta += torch.einsum("rc->c", d)
        d *= w
        # the component of d along the row's constant and along h is taken out
        dx[a:b] = r * (d - (d @ d.new_ones(width, 1)) / width - h * (torch.einsum("rc,rc->r", d, h)[:, None] / width))
        if s["add"]:
            dx[a:b] += s["add_t"][a:b].double()
    return {"dx": dx, "gamma": gamma, "beta": beta}


def _rotary_exact(s):
    b, n, heads, dim, rot = s["batch"], s["n"], s["heads"], s["dim"], s["rot"]
    f = []
    for i in range(rot // 2):
        if s["scaling"] == "base" and rot > 2:
            v = math.exp(-2.0 * i / rot * math.log(BASE) - 2.0 * i / (rot - 2) * math.log(FACTOR))
        else:
            v = math.exp(-2.0 * i / rot * math.log(BASE))
        if s["scaling"] == "linear":
            v /= FACTOR
        if s["scaling"] == "parts":
            turns = v * ORIGINAL / (2.0 * math.pi)
            share = min(1.0, max(0.0, (turns - LOW) / (HIGH - LOW)))
            v *= share + (1.0 - share) / FACTOR
        f.append(v)
    f = torch.tensor(f, dtype=torch.float64, device="cuda")
    pos = (torch.arange(n, device="cuda").repeat(b, 1) if s["pos"] is None else s["pos"]).double()
    turn = torch.polar(torch.ones((b, n, rot // 2), dtype=torch.float64, device="cuda"), (-1.0 if s["inverse"] else 1.0) * pos[:, :, None] * f)
    out = torch.empty((b, n, heads, dim), dtype=torch.float64, device="cuda")
    for h in range(heads):
        x = s["x_t"][:, :, h].double()
        first, second = (slice(0, rot // 2), slice(rot // 2, rot)) if s["layout"] == "half" else (slice(0, rot, 2), slice(1, rot, 2))
        z = torch.complex(x[..., first].contiguous(), x[..., second].contiguous()) * turn
        out[:, :, h, first], out[:, :, h, second] = z.real, z.imag
        out[:, :, h, rot:] = x[..., rot:]
    return out


def _distill_exact(s):
    n, vocab, t = s["n"], s["vocab"], s["temperature"]
    loss = torch.empty(n, dtype=torch.float64, device="cuda")
    grad = torch.empty((n, vocab), dtype=torch.float64, device="cuda") if s["grad"] else None
    for a, b in _blocks(n, vocab):
        ids, top = s["ids"][a:b].long(), s["teacher"][a:b].double() / t
        log_p = torch.log_softmax(s["x_t"][a:b].double() / t, 1)
        log_q = top - s["teacher_lse"][a:b, None].double() if s["tail"] else torch.log_softmax(top, 1)
        q = log_q.exp()
        value = (q * (log_q - log_p.gather(1, ids))).sum(1)
        target = torch.zeros_like(log_p).scatter_(1, ids, q)
        if s["tail"]:
            beyond = log_p.scatter(1, ids, -math.inf)
            log_rest = torch.logsumexp(beyond, 1)
            rest = (1.0 - q.sum(1)).clamp_(min=0.0)
            value += torch.xlogy(rest, rest) - rest * log_rest
            target += (beyond - log_rest[:, None]).exp() * rest[:, None]
        w = torch.ones_like(value) if s["weight"] is None else s["weight"][a:b].double()
        loss[a:b] = value * w * t ** 2
        if grad is not None:
            grad[a:b] = (log_p.exp() * target.sum(1, keepdim=True) - target) * (w * t * s["scale"])[:, None]
    return {"loss": loss, "grad": grad} if grad is not None else {"loss": loss}
