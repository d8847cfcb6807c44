"""Plain 64-bit implementations of the 8-bit KV cache's calls and of the sampling rules, straight from their
definitions, and makers of their inputs.  Nothing here is shared with the library."""
from __future__ import annotations

import numpy as np

import workloads as W

E_MIN, E_MAX = 27, 214


def _code_values():
    out = np.empty(256)
    for c in range(256):
        sign, e, f = -1.0 if c & 128 else 1.0, (c >> 3) & 15, c & 7
        out[c] = sign * (f * 2.0 ** -9 if e == 0 else (8 + f) * 2.0 ** (e - 10))
    out[0x7F] = out[0xFF] = np.nan
    return out


VALUES = _code_values()
_POS = VALUES[:127]  # ascending


def decode(codes, exps):
    """codes * 2^(exps - 127), exps broadcast."""
    return VALUES[codes] * np.exp2(np.asarray(exps, np.float64) - 127)


def encode(x):
    """The nearest code, ties to the even one; beyond the largest the largest; NaN the NaN code."""
    x = np.asarray(x, np.float64)
    mag = np.minimum(np.abs(x), 448.0)
    hi = np.clip(np.searchsorted(_POS, np.nan_to_num(mag)), 0, 126)
    lo = np.maximum(hi - 1, 0)
    dl, dh = mag - _POS[lo], _POS[hi] - mag
    up = (dh < dl) | ((dh == dl) & (hi % 2 == 0))
    c = np.where(up, hi, lo).astype(np.uint8)
    c = np.where(np.signbit(x), c | 128, c)
    return np.where(np.isnan(x), np.uint8(0x7F), c).astype(np.uint8)


def needed(x):
    """The scale byte of a block's new values."""
    a = np.abs(np.asarray(x, np.float64))
    a = a[~np.isnan(a)]
    top = a.max() if a.size else 0.0
    e = E_MIN
    while e < E_MAX and top > 448 * 2.0 ** (e - 127):
        e += 1
    return e


def place(table, b, r, R):
    return (b, r) if table is None else (int(table[b, r // R]), r % R)


def append(c, s, x, table, prefix, n_rows, sr):
    """codes c [pages][H][R][d], bytes s [pages][H][groups], new rows x [B][N][H][d]: in place."""
    R, H = c.shape[2], c.shape[1]
    for b in range(len(prefix)):
        P, n = int(prefix[b]), int(n_rows[b])
        first = P // sr * sr
        for r0 in range(first, P + n, sr):
            rows = [r for r in range(r0, min(r0 + sr, P + n)) if r >= P]
            if not rows:
                continue
            page, w0 = place(table, b, r0, R)
            for g in range(H):
                e = needed(x[b, [r - P for r in rows], g])
                if r0 < P:
                    old = int(s[page, g, w0 // sr])
                    e = max(e, old)
                    if e > old:
                        keep = slice(w0, w0 + P - r0)
                        c[page, g, keep] = encode(VALUES[c[page, g, keep]] * 2.0 ** (old - e))
                s[page, g, w0 // sr] = e
                for r in rows:
                    c[page, g, w0 + r - r0] = encode(np.asarray(x[b, r - P, g], np.float64) * 2.0 ** (127 - e))


def compact(c, s, table, prefix, path, n_acc, sr):
    """One layer's compaction, in place."""
    R, H = c.shape[2], c.shape[1]
    for b in range(len(prefix)):
        P, n = int(prefix[b]), int(n_acc[b])
        was_c, was_s = c.copy(), s.copy()
        for r0 in range(P // sr * sr, P + n, sr):
            page, w0 = place(table, b, r0, R)
            rows = [r for r in range(max(r0, P), min(r0 + sr, P + n))]
            src = [place(table, b, P + int(path[b, r - P]), R) for r in rows]
            for g in range(H):
                e_src = [int(was_s[p, g, w // sr]) for p, w in src]
                e = max(e_src)
                own = int(was_s[page, g, w0 // sr])
                if r0 < P:
                    e = max(e, own)
                    if e > own:
                        keep = slice(w0, w0 + P - r0)
                        c[page, g, keep] = encode(VALUES[was_c[page, g, keep]] * 2.0 ** (own - e))
                s[page, g, w0 // sr] = e
                for r, (p, w), es in zip(rows, src, e_src):
                    codes = was_c[p, g, w]
                    c[page, g, w0 + r - r0] = codes if es == e else encode(VALUES[codes] * 2.0 ** (es - e))


def paths(par):
    """For each node, the nodes of its root path, the root first."""
    out = []
    for i in range(len(par)):
        j, p = i, []
        while j >= 0:
            p.append(j)
            j = int(par[j])
        out.append(p[::-1])
    return out


def attention(q, k, v, prefix, parents, n_nodes, scale):
    """q [B][N][Hq][d]; k, v(b, rows) give [rows][H][d] values of logical rows.  Returns the outputs, the same with
    |v| in v's place, and the largest scaled sum of |q||k| over a row's keys (for the tolerances)."""
    B, N, Hq, d = q.shape
    out, mag, top = np.zeros(q.shape), np.zeros(q.shape), np.zeros(q.shape[:3])
    for b in range(B):
        P, n = int(prefix[b]), int(n_nodes[b])
        K, V = k(b, np.arange(P + n)), v(b, np.arange(P + n))
        G = Hq // K.shape[1]
        for i, path in enumerate(paths(parents[b, :n])):
            rows = np.concatenate([np.arange(P), P + np.asarray(path)]).astype(int)
            for h in range(Hq):
                kk, vv = K[rows, h // G], V[rows, h // G]
                x = kk @ q[b, i, h] * scale
                w = np.exp(x - x.max())
                w /= w.sum()
                out[b, i, h], mag[b, i, h] = w @ vv, w @ np.abs(vv)
                top[b, i, h] = scale * (np.abs(kk) @ np.abs(q[b, i, h])).max()
    return out, mag, top


def rules(logits, tokens, parents, n_nodes, counts, pen, bias, mask):
    """Processed logits in float64 (rows past the trees are NaN); counts int32 with bit 31 for the prompt;
    bias = (tokens, values, n) or None."""
    B, N, voc = logits.shape
    out = np.full(logits.shape, np.nan)
    for b in range(B):
        made = np.zeros(voc, np.int64) if counts is None else counts[b].astype(np.int64) & 0x7FFFFFFF
        seen = np.zeros(voc, bool) if counts is None else counts[b] < 0
        add, has = np.zeros(voc), np.zeros(voc, bool)
        if bias is not None:
            for t, x in list(zip(bias[0][b], bias[1][b]))[:int(bias[2][b])]:
                if 0 <= t < voc:
                    add[t] += float(x)
                    has[t] = True
        for i, path in enumerate(paths(parents[b, :int(n_nodes[b])])):
            x = logits[b, i].astype(np.float64)
            if pen is not None:
                r, f, p = (float(y) for y in pen[b])
                c = made.copy()
                for j in path[1:]:
                    if 0 <= tokens[b, j] < voc:
                        c[tokens[b, j]] += 1
                x = np.where(seen | (c > 0), np.where(x > 0, x / r, x * r), x)
                with np.errstate(invalid="ignore"):
                    x = np.where(c > 0, x - f * c - p, x)
            with np.errstate(invalid="ignore"):
                x = np.where(has, x + add, x)
            if mask is not None:
                v = np.arange(voc)
                x = np.where((mask[b, i].view(np.uint32)[v // 32] >> (v % 32)) & 1, x, -np.inf)
            out[b, i] = x
    return out


# ---------------------------------------------------------------- inputs

def cache(rng, B, H, d, sr, rows, block=0, layers=None, spread=2, extra=1):
    """A random 8-bit cache with room for `rows` rows a sequence: a dict of codes and bytes for K and V, the block
    table (pages in a random order, `extra` of them unused) and the geometry.  Unused rows hold NaN codes."""
    if block:
        per = [-(-x // block) for x in rows]
        pages = sum(per) + extra
        perm = rng.permutation(pages).astype(np.int32)
        table = np.full((B, max(per)), perm[0], np.int32)
        at = 0
        for b, n in enumerate(per):
            table[b, :n] = perm[at:at + n]
            at += n
        R = block
    else:
        table, pages, R = None, B, max(rows) + extra
    lead = () if layers is None else (layers,)
    out = dict(table=table, pages=pages, R=R, H=H, d=d, sr=sr)
    for k in ("k", "v"):
        c = rng.integers(0, 127, lead + (pages, H, R, d)).astype(np.uint8)
        c |= (rng.integers(0, 2, c.shape) << 7).astype(np.uint8)
        out[k] = c
        out[k + "s"] = rng.integers(119, 119 + spread + 1, lead + (pages, H, -(-R // sr))).astype(np.uint8)
    return out


def values(c, which, table, sr):
    """rows -> [rows][H][d] float64 values of sequence b's logical rows."""
    codes, exps = c[which], c[which + "s"]

    def get(b, rows):
        at = [place(table, b, int(r), codes.shape[2]) for r in rows]
        if not at:
            return np.zeros((0, codes.shape[1], codes.shape[3]))
        p, w = np.array([a[0] for a in at]), np.array([a[1] for a in at])
        return decode(codes[p, :, w], exps[p, :, w // sr][:, :, None])
    return get


def to_dev(a):
    import torch
    return None if a is None else torch.from_numpy(np.ascontiguousarray(a)).to("cuda")


def dev_cache(c):
    """The cache's tensors on the GPU: k, v, ks, vs, table."""
    return {k: to_dev(c[k]) for k in ("k", "v", "ks", "vs", "table")}


def trees(rng, sizes, kind="random"):
    """parents [B][max] (-1 past a tree)."""
    nmax = max(sizes)
    par = np.full((len(sizes), nmax), -1, np.int32)
    for b, n in enumerate(sizes):
        p = {"chain": W.tree_chain, "star": W.tree_star}.get(kind, lambda m: W.tree_uniform_parent(rng, m))(n)
        par[b, :n] = p
    return par
