"""YaRN over a latent cache: its factor multiplies whole queries and keys, of which a latent cache's rotations turn a part, so
it goes into the softmax scale, squared.  The calls as a program makes them against the definition in 64 bits.

Tolerances (float32, u = 2^-24), with S the largest sum of a row's products, each turned dim taken at its pair's length, times
the scale: rows and queries are stored within 15u (norm, its rounding) or 13u (turn) of these lengths, so a score is off by
S * (D + 8 + 2 * 16) u, which moves the output by 4 times that of A, the weighted mean of |c|; values are off by 16u of A; and
the attention's own 2 (T + 32) u + 4u of A as in its tests.
"""
import math

import numpy as np
import pytest

import latent_util as L
import paper_2603_01639_amd as ltd

pytestmark = pytest.mark.gpu

U = 2.0 ** -24


def pair_lengths(x, inter):
    a, b = (x[..., 0::2], x[..., 1::2]) if inter else np.split(x, 2, -1)
    r = np.hypot(a, b)
    return np.repeat(r, 2, -1) if inter else np.concatenate([r, r], -1)


@pytest.mark.parametrize("inter", [False, True])
@pytest.mark.parametrize("H, DL, N, prefix, block", [(16, 512, 1, [700, 33], 16), (4, 256, 9, [300, 65], 32), (8, 512, 20, [90], 8)])
def test_factor_in_the_scale(H, DL, N, prefix, block, inter):
    import torch
    rng = np.random.default_rng(H + N)
    B, D, factor, base_scale = len(prefix), DL + L.ROPE, 40.0, 192 ** -0.5
    par = L.trees(rng, [N] * B)
    dep = np.array([[len(L.root_path(p, i)) - 1 for i in range(N)] for p in par], np.int32)
    pages, table = L.make_table(rng, [p + N for p in prefix], block)
    freq, m = ltd.rope_frequencies(L.ROPE, 10000.0, scaling="yarn", factor=factor, trained_len=4096)
    assert m == pytest.approx(0.1 * math.log(factor) + 1)
    f32 = lambda *s: torch.from_numpy(rng.normal(size=s)).float()  # noqa: E731
    old, new, q, w = f32(B, max(prefix), D), f32(B, N, D), f32(B, N, H, D) * 1.5, 1 + 0.2 * f32(DL)
    i32 = lambda x: L.to_dev(np.asarray(x, np.int32))  # noqa: E731
    zero, P, n = i32([0] * B), i32(prefix), i32([N] * B)
    cache = torch.zeros((pages, block, D), device="cuda")
    kw = dict(norm_weight=w.cuda(), norm_eps=1e-6, interleaved=inter, block_table=L.to_dev(table), num_blocks=pages)
    ltd.latent_append(old.cuda(), cache, freq.cuda(), zero, P, **kw)
    ltd.latent_append(new.cuda(), cache, freq.cuda(), P, n, depth=i32(dep), **kw)
    turned = q.cuda()
    ltd.tree_rope(turned, turned, freq.cuda(), P, n, depth=i32(dep), rot_offset=DL, interleaved=inter)
    out = torch.zeros((B, N, H, DL), device="cuda")
    ltd.tree_verify_attn_latent(turned[..., :DL], turned[..., DL:], cache, P, i32(par), n, out, max_prefix=max(prefix),
                                scale=base_scale * m ** 2, block_table=L.to_dev(table), num_blocks=pages)
    torch.cuda.synchronize()

    f = freq.numpy()
    for b, p in enumerate(prefix):
        x = np.concatenate([old[b, :p].double().numpy(), new[b].double().numpy()])
        pos = np.r_[np.arange(p), p + dep[b]]
        c = x[:, :DL] / np.sqrt((x[:, :DL] ** 2).mean(1, keepdims=True) + 1e-6) * w.double().numpy()
        k, length_k = L.turn(x[:, DL:], pos, f, inter), pair_lengths(x[:, DL:], inter)
        for i in range(N):
            seen = np.r_[np.arange(p), p + np.array(sorted(L.root_path(par[b], i)))].astype(int)
            qd = q[b, i].double().numpy()
            t, length_q = L.turn(qd[:, DL:], np.full(H, p + dep[b, i]), f, inter), pair_lengths(qd[:, DL:], inter)
            # whole queries and keys times m
            both = (m * np.c_[qd[:, :DL], t]) @ (m * np.c_[c, k])[seen].T * base_scale
            part = (np.c_[qd[:, :DL], m * t]) @ (np.c_[c, m * k])[seen].T * base_scale

            def means(s):
                e = np.exp(s - s.max(1, keepdims=True))
                e /= e.sum(1, keepdims=True)
                return e @ c[seen], e @ np.abs(c[seen])

            want, A = means(both)
            S = (np.c_[np.abs(qd[:, :DL]), length_q] @ np.c_[np.abs(c), length_k][seen].T).max(1) * base_scale * m ** 2
            tol = (4 * S * (D + 40) * U)[:, None] * A + (2 * (len(seen) + 32) + 4 + 16) * U * A + 1e-30
            got = out[b, i].double().cpu().numpy()
            assert (np.abs(got - want) <= tol).all(), float((np.abs(got - want) / tol).max())
            # (the factor in the rotations alone is another attention)
            assert (np.abs(means(part)[0] - want) > 10 * tol).any()
