"""The row operators from their definitions, in numpy and 64 bits.  Used by the tests; shares no code with the library."""
import numpy as np

M32 = np.uint64(0xFFFFFFFF)


def philox(counter, key):
    """Philox4x32-10 (Salmon, Moraes, Dror, Shaw, SC 2011).  counter: four uint64 arrays below 2^32, key: two ints."""
    c = [np.asarray(x, dtype=np.uint64) for x in counter]
    k = [int(key[0]), int(key[1])]
    for _ in range(10):
        a, b = np.uint64(0xD2511F53) * c[0], np.uint64(0xCD9E8D57) * c[2]
        c = [(b >> np.uint64(32)) ^ c[1] ^ np.uint64(k[0]), b & M32, (a >> np.uint64(32)) ^ c[3] ^ np.uint64(k[1]), a & M32]
        k = [(k[0] + 0x9E3779B9) % 2 ** 32, (k[1] + 0xBB67AE85) % 2 ** 32]
    return c


def threshold(p):
    return min(65535, int(np.floor(p * 65536.0 + 0.5)))


def gain(p):
    return 65536.0 / (65536.0 - threshold(p))


def keep(rows, cols, p, seed, offset):
    """Boolean [rows, cols]: the elements dropout keeps."""
    if threshold(p) == 0:
        return np.ones((rows, cols), dtype=bool)
    g = -(-cols // 8)
    c0, c1 = np.meshgrid(np.arange(g, dtype=np.uint64), np.arange(rows, dtype=np.uint64))
    off = offset % 2 ** 64
    w = philox([c0, c1, np.full_like(c0, off % 2 ** 32), np.full_like(c0, off >> 32)], (seed % 2 ** 32, (seed >> 32) % 2 ** 32))
    w = np.stack(w, -1)
    halves = np.stack([w & np.uint64(0xFFFF), w >> np.uint64(16)], -1).reshape(rows, 8 * g)
    return halves[:, :cols] >= threshold(p)


def embed(table, ids, scale=1.0, pos=None, p=0.0, seed=0, offset=0):
    rows, width = table.shape
    out = np.zeros((ids.size, width))
    inside = (ids >= 0) & (ids < rows)
    out[inside] = table[ids[inside]].astype(np.float64) * scale
    if pos is not None:
        out = out + pos.astype(np.float64)[np.arange(ids.size) % pos.shape[0]]
    return np.where(keep(ids.size, width, p, seed, offset), out * gain(p), 0.0)


def embed_grad(grad_out, ids, rows, skip_id=-1, scale=1.0, p=0.0, seed=0, offset=0):
    """(G, sum of the absolute terms: what rounding errors are measured against, tokens per row)."""
    n, width = grad_out.shape
    d = np.where(keep(n, width, p, seed, offset), grad_out.astype(np.float64), 0.0) * gain(p) * scale
    inside = (ids >= 0) & (ids < rows) & (ids != skip_id)
    g, size = np.zeros((rows, width)), np.zeros((rows, width))
    np.add.at(g, ids[inside], d[inside])
    np.add.at(size, ids[inside], np.abs(d[inside]))
    return g, size, np.bincount(ids[inside], minlength=rows)


def dropout(x, add=None, p=0.5, seed=0, offset=0):
    y = np.where(keep(x.shape[0], x.shape[1], p, seed, offset), x.astype(np.float64) * gain(p), 0.0)
    return y if add is None else y + add.astype(np.float64)
