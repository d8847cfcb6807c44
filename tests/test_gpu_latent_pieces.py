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


@pytest.mark.parametrize("dtype", ["bfloat16", "float32"])
@pytest.mark.parametrize("rows", ["one far below", "the first half", "the first tile"])
@pytest.mark.parametrize("shape", CUT + [(16, 512, [40], [1], 0), (2, 256, [45, 70], [5, 1], 16), (20, 512, [70], [1], 0)], ids=named)
def test_infinities_of_no_weight_reach_the_outputs(shape, rows, dtype):
    """Rows of the prefix with infinite dims and a score of minus infinity, on a workgroup (or a wave) all of whose other
    weights are 0 beside the row's largest: the infinite dims of the outputs have no number, cut or not."""
    H, DL, prefix, sizes, block = shape
    m = make(sum(prefix) + 7, H, DL, prefix, sizes, block, dtype)
    m["q"][..., 8:16] = -m["q"][..., 8:16].abs() - 0.5
    m["q"][..., DL] = 16.0
    m.update(ql=m["q"][..., :DL], qr=m["q"][..., DL:], layout="rows")
    for b, P in enumerate(prefix):
        poison = {"one far below": [P // 5], "the first half": range(P // 2), "the first tile": range(16)}[rows]
        for r in range(P // 2):
            page, at = L.place(m["table"], b, r, m["cache"].shape[1])
            m["cache"][page, at, DL] = -1024.0  # (2^-1700 of the others' weight)
            if r in poison:
                m["cache"][page, at, 8:16] = float("inf")
    out = run(m)
    for b, n in enumerate(sizes):
        got = out[b, :n].float().cpu().numpy()
        assert not np.isfinite(got[..., 8:16]).any(), b
        assert np.isfinite(got[..., 16:]).all() and np.isfinite(got[..., :8]).all(), b
