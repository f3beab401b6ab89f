"""Shared by the tests of the drafted-token cache path: 64-bit definitions, paged caches and error bounds (no GPU code)."""
import numpy as np

# half a step of each type, relative to the value
HALF = {"f32": 2.0 ** -24, "bf16": 2.0 ** -8, "f16": 2.0 ** -11}
F32 = 2.0 ** -24


def angles(rot, theta=10000.0):
    return theta ** (-2.0 * np.arange(rot // 2) / rot)


def table(n_pos, rot, theta=10000.0):
    """fp32 [n_pos, rot / 2, 2] as the stage makes it."""
    a = np.arange(n_pos)[:, None] * angles(rot, theta)[None]
    return np.stack([np.cos(a), np.sin(a)], -1).astype(np.float32)


def pair_index(rot, layout):
    i = np.arange(rot // 2)
    return (i, i + rot // 2) if layout == 0 else (2 * i, 2 * i + 1)


def turn(u, cs, rot, layout, sign=1.0):
    """u [T, heads, dh] turned by the angles cs [T, rot / 2, 2] of its rows."""
    if rot == 0:
        return u.copy()
    a, b = pair_index(rot, layout)
    c, s = cs[:, None, :, 0], sign * cs[:, None, :, 1]
    y = u.copy()
    y[..., a], y[..., b] = u[..., a] * c - u[..., b] * s, u[..., a] * s + u[..., b] * c
    return y


def norm_rope(x, gain, cs, rot, layout, norm=True, eps=1e-5):
    """x [T, heads, dh] float64 -> (y, largest |u| of every head vector)."""
    u = x / np.sqrt((x * x).mean(-1, keepdims=True) + eps) if norm else x
    if gain is not None:
        u = u * gain
    return turn(u, cs, rot, layout), np.abs(u).max(-1, keepdims=True)


def norm_rope_bwd(dy, x, gain, cs, rot, layout, norm=True, eps=1e-5):
    """(dx, a magnitude that dx's terms do not exceed, dgain, the same for dgain)."""
    du = turn(dy, cs, rot, layout, -1.0)
    if not norm:
        return du, np.abs(du).max(-1, keepdims=True) * np.ones_like(du), None, None
    r = 1.0 / np.sqrt((x * x).mean(-1, keepdims=True) + eps)
    n = x * r
    w = du * gain if gain is not None else du
    dx = r * (w - n * (w * n).mean(-1, keepdims=True))
    big = r * (np.abs(w).max(-1, keepdims=True) + np.abs(n) * np.abs(w * n).mean(-1, keepdims=True))
    return dx, big, (du * n).sum((0, 1)), np.abs(du * n).sum((0, 1))


def trees(rng, counts):
    """Parents of one random tree per count."""
    return [[int(i - 1 if rng.random() < 0.6 else rng.integers(-1, i)) for i in range(n)] for n in counts]


def ancestors(parents):
    out = []
    for i, p in enumerate(parents):
        out.append((out[p] if p >= 0 else []) + [i])
    return out


def mask_words(seen_lists, words):
    """Truth lists (nodes seen by each row) -> int64 [rows, words]."""
    m = np.zeros((len(seen_lists), words), np.uint64)
    for r, seen in enumerate(seen_lists):
        for j in seen:
            m[r, j // 64] |= np.uint64(1 << (j % 64))
    return m.view(np.int64)


def page_table(rng, tokens, page, spare=3, width=None):
    """Shuffled page ids [requests, width] and the number of pages; unused entries name a page out of the pool's range."""
    need = [(n + page - 1) // page for n in tokens]
    total = sum(need) + spare
    ids = rng.permutation(total)
    width = max(max(need), 1) if width is None else width
    out, at = np.full((len(tokens), width), 1 << 30, np.int64), 0
    for b, n in enumerate(need):
        out[b, :n] = ids[at:at + n]
        at += n
    return out.astype(np.int32), total


def attend(q, keys, values, seen, dtype, p_half):
    """One row and query head: q [dh], keys / values [n, dh] (all the row may see), seen: their indexes.
    Returns (o [dh], bound on the error of a kernel that keeps sums in fp32 and rounds the weights to p_half)."""
    dh = q.shape[0]
    if len(seen) == 0:
        return np.zeros(dh), np.zeros(dh)
    k, v = keys[seen], values[seen]
    s = k @ q / np.sqrt(dh)
    p = np.exp(s - s.max())
    w = p / p.sum()
    o, mag = w @ v, w @ np.abs(v)
    # scores: dh products and their sum, the scaling and the exponential's argument; sums over the keys in four parts or more
    ds = (dh + 8) * F32 * (np.abs(k) @ np.abs(q)).max() / np.sqrt(dh) + 8 * F32 * np.abs(s).max()
    rel = p_half + 2 * ds + (len(seen) / 4 + 80) * F32
    # fp16 weights below 2^-20 of the largest may be dropped: the matrix cores take subnormal operands for zero
    dropped = 2.0 ** -20 * w.max() * np.abs(v).sum(0) if dtype == "f16" else 0.0
    return o, 1.01 * rel * mag + 1.01 * HALF[dtype] * np.abs(o) + 2.0 ** -24 * (dtype == "f16") + dropped
