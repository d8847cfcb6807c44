"""Latent attention whose rows are cut over workgroups: what the pieces hold and how they are joined.

Tolerances where all scores are 0, so that every weight is 1 and the output the mean of the values a row sees: products are
exact and their sums float32.  T + 32 additions (the pieces' among them) are off by at most a whole step of 2^-23 of the
mean of |c| each, and the output then rounds once, by half a step of bfloat16 at its own size.
"""
import numpy as np
import pytest

import latent_util as L
from test_gpu_latent_attention import make, run

pytestmark = pytest.mark.gpu

CUT = [  # heads, d_latent, prefix, sizes, block: every row lies on several workgroups
    (16, 512, [1500], [1], 0), (16, 512, [1500, 900], [1, 1], 16), (128, 512, [1500], [1], 64), (16, 512, [1400, 1000], [12, 5], 0),
    (4, 256, [2000], [3], 8), (40, 256, [1300], [7], 0), (128, 256, [700], [4], 16)]


def named(s):
    return "-".join(map(str, s)).replace(" ", "")


@pytest.mark.parametrize("shape", CUT, ids=named)
def test_equal_weights(shape):
    H, DL, prefix, sizes, block = shape
    m = make(sum(prefix) + H, H, DL, prefix, sizes, block)
    m["q"].zero_()
    m.update(ql=m["q"][..., :DL], qr=m["q"][..., DL:], layout="rows")
    m["cache"].abs_().add_(0.5)
    out = run(m).double().cpu().numpy()
    f = lambda t: t.double().numpy()  # noqa: E731
    want, A, _ = L.attention(f(m["ql"]), f(m["qr"]), f(m["cache"]), m["table"], m["prefix"], m["par"], m["n"], m["scale"])
    for b, n in enumerate(sizes):
        w, T = want[b, :n], prefix[b] + n
        tol = 2.0 ** (np.floor(np.log2(w)) - 8) + (T + 32) * 2.0 ** -23 * A[b, :n]
        err = np.abs(out[b, :n] - w)
        assert (err <= tol).all(), f"sequence {b}: {float((err / tol).max())} of the tolerance, {int((err > tol).sum())} values"


@pytest.mark.parametrize("shape", CUT, ids=named)
def test_infinities_leave_the_other_dims(shape):
    """A row of the prefix with eight infinite dims and a score of minus infinity: its weight is 0, so these dims have no
    number and the others are the attention over the other rows."""
    H, DL, prefix, sizes, block = shape
    m = make(sum(prefix) + 7, H, DL, prefix, sizes, block)
    m["q"][..., 8:16] = -m["q"][..., 8:16].abs() - 0.5
    m.update(ql=m["q"][..., :DL], qr=m["q"][..., DL:], layout="rows")
    cache = m["cache"].clone()
    for b, P in enumerate(prefix):
        page, at = L.place(m["table"], b, 3 * P // 5, cache.shape[1])
        cache[page, at, 8:16] = float("inf")
    out = run(m, cache=cache.to("cuda")).clone()
    for b, n in enumerate(sizes):
        assert not np.isfinite(out[b, :n, :, 8:16].float().cpu().numpy()).any()
    # the same attention without that row: a score that no weight is left of, and finite values
    for b, P in enumerate(prefix):
        page, at = L.place(m["table"], b, 3 * P // 5, cache.shape[1])
        m["cache"][page, at] = 0
        m["cache"][page, at, 8:16] = 2.0 ** 60
    clean = run(m).double().cpu().numpy()
    got = out.double().cpu().numpy()
    rest = np.r_[0:8, 16:DL]
    for b, n in enumerate(sizes):
        assert np.isfinite(got[b, :n][..., rest]).all()
        assert (got[b, :n][..., rest] == clean[b, :n][..., rest]).all()
