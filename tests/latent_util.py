"""Plain 64-bit implementations of rotary positions and of the latent cache's calls, straight from their definitions,
and makers of their inputs.  Nothing here is shared with the library."""
from __future__ import annotations

import numpy as np

import q8_util
from q8_util import to_dev  # noqa: F401

ROPE = 64


def trees(rng, sizes, kind="random"):
    """parents [B][max] (-1 past a tree, and for an empty one)."""
    par = q8_util.trees(rng, [max(n, 1) for n in sizes], kind)
    return par[:, :max(sizes)]


def frequencies(rot, base=10000.0):
    return base ** (-2.0 * np.arange(rot // 2) / rot)


def turn(x, pos, freq, inter, m=1.0):
    """x [..., rot] turned by pos [...] * freq, pairs as complex numbers."""
    x = np.asarray(x, np.float64)
    rot = x.shape[-1]
    a, b = (slice(0, rot, 2), slice(1, rot, 2)) if inter else (slice(0, rot // 2), slice(rot // 2, rot))
    angle = np.asarray(pos, np.longdouble)[..., None] * np.asarray(freq, np.longdouble)
    z = (x[..., a] + 1j * x[..., b]) * m * np.exp(1j * angle.astype(np.clongdouble)).astype(np.complex128)
    y = np.empty_like(x)
    y[..., a], y[..., b] = z.real, z.imag
    return y


def half_step(dtype):
    """Half a rounding step relative to the value."""
    return {"bfloat16": 2.0 ** -8, "float32": 2.0 ** -24}[str(dtype).split(".")[-1]]


def place(table, b, r, R):
    return (b, r) if table is None else (int(table[b, r // R]), r % R)


def make_table(rng, rows, block, extra=2):
    """Pages and block table of sequences with rows[b] rows."""
    per = [-(-r // block) for r in rows]
    pages = sum(per) + extra
    perm = rng.permutation(pages)
    table = np.full((len(rows), max(per) if per else 1), -7, np.int32)
    at = 0
    for b, n in enumerate(per):
        table[b, :n] = perm[at:at + n]
        at += n
    return pages, table


def gather(cache, table, b, n):
    """Logical rows 0 .. n - 1 of sequence b from a cache [pages][R][D]."""
    R = cache.shape[1]
    if table is None:
        return cache[b, :n]
    t = np.arange(n)
    return cache[table[b, t // R], t % R]


def root_path(par, i):
    out = []
    while i >= 0:
        out.append(i)
        i = int(par[i])
    return out


def attention(ql, qr, cache, table, prefix, par, sizes, scale):
    """Outputs [B][N][H][DL], the weighted means of |c| and the largest scaled sum of |q||x| of every row."""
    B, N, H, DL = ql.shape
    out, mean = np.zeros((B, N, H, DL)), np.zeros((B, N, H, DL))
    size = np.zeros((B, N, H))
    q = np.concatenate([ql, qr], -1).astype(np.float64)
    for b in range(B):
        P, n = int(prefix[b]), int(sizes[b])
        x = gather(cache, table, b, P + n).astype(np.float64)
        for i in range(n):
            seen = np.r_[np.arange(P), P + np.array(sorted(root_path(par[b], i)))].astype(int)
            rows = x[seen]
            s = q[b, i] @ rows.T * scale
            w = np.exp(s - s.max(1, keepdims=True))
            w /= w.sum(1, keepdims=True)
            out[b, i], mean[b, i] = w @ rows[:, :DL], w @ np.abs(rows[:, :DL])
            size[b, i] = (np.abs(q[b, i]) @ np.abs(rows).T).max(1) * scale
    return out, mean, size
