"""The row-sparse front end of a language model, as measured cases.

Four operators that produce or consume what the sparsification step works on:

``embed``    token rows of a table, scaled, with position rows added and dropout applied
``grad``     the table's gradient: the rows of the incoming gradient summed by token, in fp32, into the
             table's part of the flat gradient vector (written) or of the residual (added)
``dropout``  dropout from a counter-based generator, optionally added to a residual stream
``step``     error-feedback accumulate and layer norms of a vector whose embedding gradient is row sparse

The dropout mask is a function of (seed, offset, row, column) alone: Philox4x32-10 (Salmon, Moraes, Dror and
Shaw, "Parallel random numbers: as easy as 1, 2, 3", SC 2011) with counter (column / 8, row, offset) and key
seed gives eight 16-bit numbers for eight columns; an element is kept when its number is at least
t = round(65536 p), and kept elements are multiplied by 65536 / (65536 - t).

With ``own = False`` the operators are computed in their plain form; with ``own = True`` by this repository's
library.
"""
import math

import numpy as np
import torch

own = False

TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
SIZE = {"f32": 4, "bf16": 2, "f16": 2}
MASK = 0xFFFFFFFF

# Tensor sizes of a two-layer LSTM language model, vocabulary 33278, width 1500 (the table first).
LSTM = [33278 * 1500] + 2 * [4 * 1500 * 1500, 4 * 1500 * 1500, 4 * 1500, 4 * 1500] + [1500 * 33278, 33278]


def listed():
    return [
        # one step of an LSTM language model: 20 sequences of 35 tokens, latency counts
        _embed("embed_lstm_700", 700, 33278, 1500, "f32", "f32", 0, 0.5, 1.0, 8),
        # a BERT-large batch: 32 sequences of 512 tokens, positions added, dropout 0.1
        _embed("embed_bert_16k", 16384, 30522, 1024, "bf16", "bf16", 512, 0.1, 1.0, 8),
        # a large GPT-2-medium batch from fp32 master weights, 128 sequences of 1024 tokens
        _embed("embed_gpt2_128k", 131072, 50257, 1024, "f32", "bf16", 1024, 0.1, 1.0, 8),
        # the LSTM step's gradient, added to the touched rows of the residual
        _grad("grad_lstm_700_add", 700, 33278, 1500, "f32", -1, 0.5, 1.0, 8, True),
        # the BERT batch's gradient written as a dense part of the gradient vector, padding token 0 left out
        _grad("grad_bert_16k_write", 16384, 30522, 1024, "bf16", 0, 0.1, 1.0, 8, False),
        # the large GPT-2 batch's gradient, added to what the tied output layer has left in the vector
        _grad("grad_gpt2_128k_add", 131072, 50257, 1024, "bf16", -1, 0.1, 1.0, 8, True),
        # odd sizes throughout, rows that start on no vector boundary, 32-bit ids, embeddings scaled by sqrt(width)
        _grad("grad_odd_5003_write", 5003, 10007, 1027, "f16", -1, 0.0, math.sqrt(1027.0), 4, False),
        # dropout between the layers of the LSTM model
        _dropout("dropout_lstm_700", 700, 1500, "f32", "f32", False, 0.5),
        # a transformer block's output dropout, added to the residual stream
        _dropout("dropout_bert_16k_add", 16384, 1024, "bf16", "bf16", True, 0.1),
        # the widest activations of a large batch: 65536 tokens, feed-forward width 4096
        _dropout("dropout_64k_4096", 65536, 4096, "bf16", "bf16", False, 0.1),
        # accumulate + norms of the whole LSTM vector with the embedding's gradient by rows
        _step("step_lstm_700", 700, 33278, 1500, LSTM[1:], "f32", 0.5),
        # the same of a small model, where the number of launches counts
        _step("step_small_1k", 1024, 8000, 512, [4 * 512 * 512, 512, 8 * 512 * 512, 2048, 777], "bf16", 0.1),
    ]


def _embed(name, n, rows, width, table, out, pos, p, scale, id_bytes):
    return {"name": name, "op": "embed", "n": n, "rows": rows, "width": width, "table": table, "out": out, "pos": pos, "p": p,
            "scale": scale, "id_bytes": id_bytes}


def _grad(name, n, rows, width, dy, skip_id, p, scale, id_bytes, add):
    return {"name": name, "op": "grad", "n": n, "rows": rows, "width": width, "dy": dy, "skip_id": skip_id, "p": p, "scale": scale,
            "id_bytes": id_bytes, "add": add}


def _dropout(name, rows, width, x, y, add, p):
    return {"name": name, "op": "dropout", "n": rows, "width": width, "x": x, "y": y, "add": add, "p": p}


def _step(name, n, rows, width, rest, dy, p):
    return {"name": name, "op": "step", "n": n, "rows": rows, "width": width, "rest": ",".join(str(s) for s in rest), "dy": dy, "p": p}


def draw(rng):
    def log(lo, hi):
        return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))

    def kind():
        return rng.choice(["f32", "bf16", "f16"])

    op = rng.choice(["embed", "grad", "grad", "dropout", "step"])
    width = log(8, 4096)
    if rng.random() < 0.6:
        width = max(8, width // 8 * 8)
    n = log(1, min(131072, 131072 * 1024 // width))
    rows = log(64, min(131072, 50257 * 1024 // width))
    p = rng.choice([0.0, 0.1, 0.1, 0.25, 0.5])
    scale = rng.choice([1.0, math.sqrt(width)])
    if op == "embed":
        c = _embed("", n, rows, width, kind(), kind(), rng.choice([0, max(1, n // 3)]), p, scale, rng.choice([4, 8]))
    elif op == "grad":
        c = _grad("", n, rows, width, kind(), rng.choice([-1, 0, rows // 2]), p, scale, rng.choice([4, 8]), rng.random() < 0.5)
    elif op == "dropout":
        x, add = kind(), rng.random() < 0.5
        y = rng.choice([x, "f32"])
        n = log(1, min(65536, (1 << 30) // (width * (SIZE[x] + SIZE[y] * (2 if add else 1)))))
        c = _dropout("", n, width, x, y, add, rng.choice([0.1, 0.1, 0.25, 0.5]))
    else:
        c = _step("", min(n, 16384), min(rows, 33278 * 1500 // width), width, [log(1, 20000000), log(1, 2000000), log(1, 5000)], kind(), p)
    del c["name"]
    return c


# ---- inputs ----------------------------------------------------------------------------------
def _generator(seed):
    return torch.Generator(device="cuda").manual_seed(1000003 * int(seed) + 17)


def _tokens(g, n, rows, id_bytes=8):
    """Token ids as text has them: the frequency falls with 1 / rank, the lowest ids are the most frequent."""
    u = torch.rand(n, generator=g, device="cuda", dtype=torch.float64)
    ids = (torch.exp(u * math.log(rows + 1.0)) - 1.0).floor().clamp_(0, rows - 1)
    return ids.to(torch.int64 if id_bytes == 8 else torch.int32)


def _normal(g, shape, kind, std=1.0):
    return torch.empty(shape, dtype=TYPES[kind], device="cuda").normal_(0.0, std, generator=g)


def prepare(case, seed):
    g = _generator(seed)
    c = dict(case, seed=int(seed) * 2654435761 % (1 << 63), offset=int(seed) * 7 + 3)
    n, width = c["n"], c["width"]
    if c["op"] == "embed":
        c["w"] = _normal(g, (c["rows"], width), c["table"], 0.02)
        c["ids"] = _tokens(g, n, c["rows"], c["id_bytes"])
        c["pos_w"] = _normal(g, (c["pos"], width), c["table"], 0.02) if c["pos"] else None
        c["y"] = torch.empty((n, width), dtype=TYPES[c["out"]], device="cuda")
    elif c["op"] == "grad":
        c["dy_t"] = _normal(g, (n, width), c["dy"], 0.01)
        c["ids"] = _tokens(g, n, c["rows"], c["id_bytes"])
        c["g"] = _normal(g, (c["rows"], width), "f32", 0.01)
    elif c["op"] == "dropout":
        c["x_t"] = _normal(g, (n, width), c["x"])
        c["add_t"] = _normal(g, (n, width), c["y"]) if c["add"] else None
        c["y_t"] = torch.empty((n, width), dtype=TYPES[c["y"]], device="cuda")
    else:
        sizes = _sizes(c)
        n_g = sum(sizes)
        c["dy_t"] = _normal(g, (n, width), c["dy"], 0.01)
        c["ids"] = _tokens(g, n, c["rows"])
        c["e"] = _normal(g, (n_g,), "f32", 0.003)
        # the dense tensors' gradient; the table's part of the vector holds none
        c["grad"] = _normal(g, (n_g,), "f32", 0.003)
        c["grad"][:sizes[0]] = 0.0
        start = torch.zeros(len(sizes) + 1, dtype=torch.int64)
        start[1:] = torch.tensor(sizes).cumsum(0)
        c["start"] = start.cuda()
        c["norms"] = torch.empty(len(sizes), dtype=torch.float64, device="cuda")
    if own and c["op"] in ("grad", "step"):   # the workspaces a program allocates once
        from paper_2307_03500_b200 import deft
        c["ws_rows"] = deft.alloc_embed_workspace(n, c["rows"], width, "cuda")
        if c["op"] == "step":
            c["ws"] = deft.alloc_workspace(c["e"].numel(), c["norms"].numel(), "cuda")
    return c


def _sizes(c):
    return [c["rows"] * c["width"]] + [int(s) for s in c["rest"].split(",")]


# ---- one pass --------------------------------------------------------------------------------
def run(state):
    if own:
        return _run_own(state)
    c = state
    if c["op"] == "embed":
        return _embed_plain(c)
    if c["op"] == "grad":
        got = _grad_plain(c, c["dy_t"], c["ids"], c["rows"], c["skip_id"], c["scale"])
        return c["g"].add_(got) if c["add"] else c["g"].copy_(got)
    if c["op"] == "dropout":
        x = c["x_t"].float()
        y = torch.where(_keep(c, c["n"], c["width"]), x * _rate(c["p"])[1], torch.zeros_like(x)) if c["p"] else x
        return (y + c["add_t"].float() if c["add_t"] is not None else y).to(c["y_t"].dtype)
    size = c["rows"] * c["width"]
    got = _grad_plain(c, c["dy_t"], c["ids"], c["rows"], -1, 1.0)
    e = c["e"].add_(torch.cat([got.view(-1), c["grad"][size:]]))
    norms = [part.double().square().sum().sqrt() for part in e.split(_sizes(c))]
    return {"e": e, "norms": torch.stack(norms).float()}


def _rate(p):
    t = min(65535, int(math.floor(p * 65536.0 + 0.5)))
    return t, 65536.0 / (65536 - t)


def _keep(c, n, width):
    """Which elements of an [n, width] matrix dropout keeps."""
    c0 = torch.arange((width + 7) // 8, device="cuda").view(1, -1)
    c1 = torch.arange(n, device="cuda").view(-1, 1)
    c2, c3 = c["offset"] & MASK, c["offset"] >> 32
    k0, k1 = c["seed"] & MASK, c["seed"] >> 32
    for _ in range(10):
        a, b = c0 * 0xD2511F53, c2 * 0xCD9E8D57
        c0, c1, c2, c3 = ((b >> 32) & MASK) ^ c1 ^ k0, b & MASK, ((a >> 32) & MASK) ^ c3 ^ k1, a & MASK
        k0, k1 = (k0 + 0x9E3779B9) & MASK, (k1 + 0xBB67AE85) & MASK
    words = torch.stack(torch.broadcast_tensors(c0, c1, c2, c3), -1)
    halves = torch.stack([words & 0xFFFF, words >> 16], -1).view(n, -1)
    return halves[:, :width] >= _rate(c["p"])[0]


def _embed_plain(c):
    y = c["w"][c["ids"].long()].float() * c["scale"]
    if c["pos"]:
        y = y + c["pos_w"].float()[torch.arange(c["n"], device="cuda") % c["pos"]]
    if c["p"]:
        y = torch.where(_keep(c, c["n"], c["width"]), y * _rate(c["p"])[1], torch.zeros_like(y))
    return y.to(TYPES[c["out"]])


def _grad_plain(c, dy, ids, rows, skip_id, scale):
    d = dy.float()
    if c["p"]:
        d = torch.where(_keep(c, c["n"], c["width"]), d, torch.zeros_like(d))
        scale = scale * _rate(c["p"])[1]
    if skip_id >= 0:
        d = torch.where((ids != skip_id).view(-1, 1), d, torch.zeros_like(d))
    return torch.zeros((rows, d.shape[1]), dtype=torch.float32, device="cuda").index_add_(0, ids.long(), d).mul_(scale)


def _run_own(c):
    from paper_2307_03500_b200 import deft
    drop = {"p": c["p"], "seed": c["seed"], "offset": c["offset"]}
    if c["op"] == "embed":
        deft.deft_embed(c["w"], c["ids"], c["y"], scale=c["scale"], pos=c["pos_w"], **drop)
        return c["y"]
    if c["op"] == "grad":
        deft.deft_embed_grad(c["dy_t"], c["ids"], c["g"], c["ws_rows"], accumulate=c["add"], skip_id=c["skip_id"], scale=c["scale"], **drop)
        return c["g"]
    if c["op"] == "dropout":
        deft.deft_dropout(c["x_t"], c["y_t"], add=c["add_t"], **drop)
        return c["y_t"]
    size = c["rows"] * c["width"]
    table = c["e"][:size].view(c["rows"], c["width"])
    deft.deft_embed_grad(c["dy_t"], c["ids"], table, c["ws_rows"], accumulate=True, **drop)
    deft.deft_layer_norms_part(c["e"], c["grad"], [(0, size)], c["start"], c["norms"], c["ws"])
    return {"e": c["e"], "norms": c["norms"].float()}


# ---- what one pass cannot do without -----------------------------------------------------------
def _distinct(n, rows):
    """The expected number of different tokens among n."""
    edges = np.log1p(np.arange(rows + 1, dtype=np.float64)) / math.log(rows + 1.0)
    return float((1.0 - np.exp(n * np.log1p(-np.minimum(np.diff(edges), 1 - 1e-16)))).sum())


def work(case):
    c, n, width = case, case["n"], case["width"]
    cells = n * width
    # a Philox call is ten rounds of two products and four exclusive ors, for eight elements
    random = cells // 8 * 60 if c["p"] else 0
    if c["op"] == "embed":
        read = n * c["id_bytes"] + (_distinct(n, c["rows"]) + c["pos"]) * width * SIZE[c["table"]]
        return {"bytes": int(read + cells * SIZE[c["out"]]), "flops": 3 * cells + random}
    if c["op"] == "grad":
        out = 8 * _distinct(n, c["rows"]) * width if c["add"] else 4 * c["rows"] * width
        return {"bytes": int(n * c["id_bytes"] + cells * SIZE[c["dy"]] + out), "flops": 2 * cells + random}
    if c["op"] == "dropout":
        return {"bytes": cells * (SIZE[c["x"]] + SIZE[c["y"]] * (2 if c["add"] else 1)), "flops": 2 * cells + random}
    sizes = _sizes(c)
    table, rest = sizes[0], sum(sizes[1:])
    touched = _distinct(n, c["rows"]) * width
    return {"bytes": int(n * 8 + cells * SIZE[c["dy"]] + 4 * touched + 4 * table + 12 * rest), "flops": 2 * cells + random + 2 * table + 3 * rest}


# ---- the definition in 64 bits -----------------------------------------------------------------
def _mul_32(a, m):
    """High and low 32 bits of a * m from 16-bit limbs."""
    a0, a1, m0, m1 = a & 0xFFFF, a >> 16, m & 0xFFFF, m >> 16
    low, mid1, mid2 = a0 * m0, a0 * m1, a1 * m0
    carry = (low >> 16) + (mid1 & 0xFFFF) + (mid2 & 0xFFFF)
    return a1 * m1 + (mid1 >> 16) + (mid2 >> 16) + (carry >> 16), ((carry & 0xFFFF) << 16) | (low & 0xFFFF)


def _kept_exact(s, row0, rows, width):
    """dropout's factor (0, or the survivors' gain) for the rows row0 .. row0 + rows."""
    if not s["p"]:
        return 1.0
    x = [torch.arange(-(-width // 8), device="cuda").repeat(rows, 1),
         (row0 + torch.arange(rows, device="cuda")).view(-1, 1).repeat(1, -(-width // 8))]
    x += [torch.full_like(x[0], s["offset"] % 2 ** 32), torch.full_like(x[0], s["offset"] // 2 ** 32)]
    key = [s["seed"] % 2 ** 32, s["seed"] // 2 ** 32]
    for r in range(10):
        h0, l0 = _mul_32(x[0], 0xD2511F53)
        h1, l1 = _mul_32(x[2], 0xCD9E8D57)
        x = [h1 ^ x[1] ^ ((key[0] + r * 0x9E3779B9) % 2 ** 32), l1, h0 ^ x[3] ^ ((key[1] + r * 0xBB67AE85) % 2 ** 32), l0]
    t = min(65535, round(s["p"] * 65536))
    out = torch.empty((rows, x[0].shape[1], 8), dtype=torch.float64, device="cuda")
    for i in range(4):
        out[:, :, 2 * i] = x[i] % 65536 >= t
        out[:, :, 2 * i + 1] = x[i] // 65536 >= t
    return out.view(rows, -1)[:, :width] * (65536.0 / (65536.0 - t))


def exact(case, seed):
    s = prepare(case, seed)
    n, width = s["n"], s["width"]
    step = max(1, (1 << 24) // width)   # rows at a time: the generator's words take 64 bytes for eight elements
    blocks = [(a, min(n, a + step)) for a in range(0, n, step)]
    if s["op"] == "embed":
        w, y = s["w"].double(), torch.empty((n, width), dtype=torch.float64, device="cuda")
        for a, b in blocks:
            v = w.index_select(0, s["ids"][a:b].long()) * s["scale"]
            if s["pos"]:
                v += s["pos_w"].double().index_select(0, torch.arange(a, b, device="cuda").remainder(s["pos"]))
            y[a:b] = v * _kept_exact(s, a, b - a, width)
        return y
    if s["op"] == "dropout":
        y = torch.empty((n, width), dtype=torch.float64, device="cuda")
        for a, b in blocks:
            y[a:b] = s["x_t"][a:b].double() * _kept_exact(s, a, b - a, width)
            if s["add"]:
                y[a:b] += s["add_t"][a:b].double()
        return y
    total = torch.zeros((s["rows"], width), dtype=torch.float64, device="cuda")
    for a, b in blocks:
        ids = s["ids"][a:b].long()
        d = s["dy_t"][a:b].double() * _kept_exact(s, a, b - a, width) * s.get("scale", 1.0)
        keep = ids != s.get("skip_id", -1)
        total.index_put_((ids[keep],), d[keep], accumulate=True)
    if s["op"] == "grad":
        return total + s["g"].double() if s["add"] else total
    e = s["e"].double() + s["grad"].double()
    e[:total.numel()] += total.view(-1)
    start = s["start"].tolist()
    norms = torch.stack([torch.linalg.vector_norm(e[a:b]) for a, b in zip(start, start[1:])])
    return {"e": e, "norms": norms}
