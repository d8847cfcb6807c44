"""Attention over an 8-bit cache in many pieces: long prefixes for the kernels of more than 32 stacked rows, batches of
thousands of units, and what the pieces are held in.  (The reference and, where nothing else is said, the tolerance are
those of test_gpu_q8_attention.)"""
import numpy as np
import pytest

import q8_util as Q
from test_gpu_q8_attention import check, make, run

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("B, Hq, Hkv, d, prefix, sizes, block", [
    (1, 8, 2, 128, [16384], [60], 0), (1, 8, 1, 128, [16383], [13], 16), (1, 4, 2, 64, [15000], [200], 64),
    (4, 8, 2, 128, [5000, 64, 3001, 1000], [20, 64, 9, 33], 16), (3, 16, 2, 64, [6000, 0, 777], [12, 40, 1], 0)])
def test_long_prefixes(B, Hq, Hkv, d, prefix, sizes, block):
    m = make(B + d, B, Hq, Hkv, d, 16, prefix, sizes, block)
    check(m, run(m), label="long")


@pytest.mark.parametrize("block", [0, 16])
def test_thousands_of_units(block):
    """256 sequences of 8 kv heads are 2048 units of up to 34 rows, some of them long enough to be cut."""
    rng = np.random.default_rng(3)
    B = 256
    prefix = [int(x) for x in rng.integers(0, 200, B)]
    for b in (0, 17, 100, 255):
        prefix[b] = 3000 if block else 500  # (a contiguous cache has room for the longest in every sequence)
    sizes = [int(x) for x in rng.integers(1, 5, B)]
    sizes[3], sizes[100] = 17, 9
    m = make(9, B, 16, 8, 64, 16, prefix, sizes, block)
    check(m, run(m), label="units")


@pytest.mark.parametrize("B, Hq, Hkv, n, P", [(1, 8, 2, 60, 16384), (1, 8, 2, 13, 4096), (5, 8, 2, 60, 4096), (1, 8, 2, 1, 16384),
                                              (8, 8, 4, 4, 4096)])
@pytest.mark.parametrize("d", [64, 128])
def test_pieces_keep_eleven_bits(B, Hq, Hkv, n, P, d):
    """Keys of zero, so that weights (all 1) and sums (of few bits) are exact, and values whose mean is 1 + 3 * 2^-9 over
    each 64 keys of a prefix's first half and -1 over the second: the halves all but cancel, and what is left of a
    piece's rounding shows.  Half a step of fp16 is 2^-11 of a piece's mean, so at most 2^-11 * A in all; the quotients by
    the sums and the merge's products and sums are off by 2^-24 of A each, less than 64 of them; the output is rounded
    (2^-8 * |o|).  Pieces in bf16 would move the result by 2^-10 * A, for 1 + 3 * 2^-9 lies a quarter of a step from
    its neighbour."""
    m = make(1, B, Hq, Hkv, d, 16, [P] * B, [n] * B, 0)
    c = m["c"]
    one, more, minus = (int(Q.encode(np.array(x))) for x in (1.0, 1.125, -1.0))
    c["k"][:] = 0
    c["v"][:] = 0
    c["v"][:, :, :P // 2] = one
    for r in (5, 20, 41):
        c["v"][:, :, r:P // 2:64] = more
    c["v"][:, :, P // 2:P] = minus
    c["ks"][:] = c["vs"][:] = 127
    k, v = (Q.values(c, w, None, 16) for w in "kv")
    want, A, _ = Q.attention(m["q"].double().numpy(), k, v, m["prefix"], m["par"], m["n"], d ** -0.5)
    got = run(m).double().cpu().numpy()
    tol = 2.0 ** -11 * A + 64 * 2.0 ** -24 * A + 2.0 ** -8 * np.abs(want)
    assert (np.abs(got - want) <= tol).all(), float((np.abs(got - want) / tol).max())
