"""How many bits the weights of latent attention have that multiply the values, for calls of up to 16 rows a sequence in bfloat16.

Two kinds of keys, all with scores of one exact product: score 0 and values +v0, a lower score and values -v1, so that in some
dims the output nearly cancels, and what is left is the error of the weights' ratio.  Tolerance, with u = 2^-24, A the weighted
mean of |c|, o the output, S the largest |score| (scaled), T the keys: the exponent in powers of two is off by at most
3 * 2 * 1.45 S u (the scale's constant, the product, the maximum's), and the exponential by two steps of 2u: e = (9 S + 4) u, which moves
o by 4 e A; a weight is rounded in two parts to 2^-16 of itself and normalised by the parts' sum, 2^-16 (A + |o|); numerator and
denominator are sums of T + 32 terms, a whole step of 2u each at most, 4 (T + 32) u A; and the output rounds by 2^-8 |o|.
"""
import numpy as np
import pytest

import latent_util as L
from test_gpu_latent_attention import make, run

pytestmark = pytest.mark.gpu

U = 2.0 ** -24


@pytest.mark.parametrize("H, n", [(16, 1), (4, 4), (1, 1)])
@pytest.mark.parametrize("DL, P, block", [(512, 20, 0), (512, 300, 16), (256, 1500, 0), (256, 77, 8)])
def test_sixteen_bits(DL, P, block, H, n):
    import torch
    m = make(P + H, H, DL, [P, P // 2], [n, 1], block, nmax=n)
    rng = np.random.default_rng(P)
    t = m["q"].dtype
    q = torch.zeros_like(m["q"])
    q[..., DL] = (4 + torch.arange(H) / 8.0).to(t)  # (exact, one for each head)
    low = torch.from_numpy(rng.random(m["cache"].shape[:2]) < 0.5)
    v = torch.from_numpy(2.0 ** np.linspace(-2, 2, DL) * np.where(rng.random(DL) < 0.5, 1, -1))
    m["cache"][..., :DL] = torch.where(low[..., None], -v, torch.ones(DL, dtype=torch.float64) * v.sign()).to(t)
    m["cache"][..., DL] = torch.where(low, torch.tensor(-1.25, dtype=torch.float64), torch.tensor(0.0, dtype=torch.float64)).to(t)
    m["cache"][..., DL + 1:] = 1
    m.update(q=q, ql=q[..., :DL], qr=q[..., DL:], layout="rows")
    out = run(m).double().cpu().numpy()
    f = lambda x: x.double().numpy()  # noqa: E731
    want, A, S = L.attention(f(m["ql"]), f(m["qr"]), f(m["cache"]), m["table"], m["prefix"], m["par"], m["n"], m["scale"])
    for b, k in enumerate(m["n"]):
        w, a, s, T = want[b, :k], A[b, :k], S[b, :k, :, None], int(m["prefix"][b]) + k
        tol = 4 * (9 * s + 4) * U * a + 2.0 ** -16 * (a + np.abs(w)) + 4 * (T + 32) * U * a + 2.0 ** -8 * np.abs(w)
        err = np.abs(out[b, :k] - w)
        assert (err <= tol).all(), f"sequence {b}: {float((err / tol).max())} of the tolerance, {int((err > tol).sum())} values"
