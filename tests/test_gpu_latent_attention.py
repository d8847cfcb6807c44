"""Tree attention over a latent cache on the GPU against softmax attention in 64 bits.

Tolerances, per output element, with A the same weighted mean of |c|, o the output, S the largest scaled sum of
|q||x| of its row, T its keys and D = d_latent + 64.  Scores are float32 sums of exact products: off by at most
e = S * (D + 8) * 2^-24, which moves a weight by a factor within e^(+-2e), so the output by about 4e * A; the exponent's
own rounding is of the size of |m * c| * 2^-24 <= 2S * 2^-24 and is covered by the 8 in e.
bfloat16 (half a step is 2^-8): weights are rounded once and normalised by the rounded ones' sum (2^-8 * (A + |o|)),
pieces of a row may be stored rounded (2^-8 * A), the output is rounded (2^-8 * |o|).
float32 (half a step is 2^-24): T + 32 additions of weights and products, 2 * (T + 32) * 2^-24 * A, and the exponential
within 2 ulp, 4 * 2^-24 * A.
"""
import numpy as np
import pytest

import latent_util as L
import paper_2603_01639_amd as ltd

pytestmark = pytest.mark.gpu


def tolerance(bf16, o, A, S, T, D):
    e = (S * (D + 8) * 2.0 ** -24)[..., None]
    base = 4 * e * A
    if bf16:
        return 1.02 * (base + 2.0 ** -8 * (2 * A + 2 * np.abs(o))) + 1e-30
    return base + (2 * (T + 32) + 4) * 2.0 ** -24 * A + 1e-30


def make(seed, H, DL, prefix, sizes, block=0, dtype="bfloat16", kind="random", qstd=1.5, nmax=None, layout="rows", slack=3):
    import torch
    rng = np.random.default_rng(seed)
    B, D = len(prefix), DL + L.ROPE
    rows = [p + n for p, n in zip(prefix, sizes)]
    t = getattr(torch, dtype)
    if block:
        pages, table = L.make_table(rng, rows, block)
        shape = (pages, block, D)
    else:
        table, shape = None, (B, max(rows) + slack, D)
    cache = torch.from_numpy(rng.normal(size=shape)).to(t)
    par = L.trees(rng, sizes, kind)
    if nmax:
        par = np.pad(par, ((0, 0), (0, nmax - par.shape[1])), constant_values=-7)
    N = par.shape[1]
    q = torch.from_numpy(rng.normal(size=(B, N, H, D)) * qstd).to(t)
    if layout == "rows":  # one tensor, both parts views of it
        ql, qr = q[..., :DL], q[..., DL:]
    else:  # a product per head's output, and the rotated part beside it
        ql, qr = q[..., :DL].permute(2, 0, 1, 3).contiguous().permute(1, 2, 0, 3), q[..., DL:].contiguous()
    return dict(cache=cache, table=table, par=par, q=q, ql=ql, qr=qr, layout=layout, prefix=np.array(prefix, np.int32),
                n=np.array(sizes, np.int32), scale=(128 + L.ROPE) ** -0.5, DL=DL)


def parts(m):
    """The query parts on the GPU, laid out as the case says."""
    q = m["q"].to("cuda")
    if m["layout"] == "rows":
        return q[..., :m["DL"]], q[..., m["DL"]:]
    return (q[..., :m["DL"]].permute(2, 0, 1, 3).contiguous().permute(1, 2, 0, 3), q[..., m["DL"]:].contiguous())


def run(m, fill=7.0, max_prefix=None, scale=None, cache=None, out=None, **more):
    import torch
    ql, qr = parts(m)
    B, N, H, DL = ql.shape
    out = torch.full((B, N, H, DL), fill, dtype=ql.dtype, device="cuda") if out is None else out
    table = None if m["table"] is None else L.to_dev(m["table"])
    ltd.tree_verify_attn_latent(ql, qr, m["cache"].to("cuda") if cache is None else cache, L.to_dev(m["prefix"]),
                                L.to_dev(m["par"]), L.to_dev(m["n"]), out,
                                max_prefix=int(m["prefix"].max()) if max_prefix is None else max_prefix,
                                scale=m["scale"] if scale is None else scale, block_table=table,
                                num_blocks=0 if table is None else m["cache"].shape[0], **more)
    torch.cuda.synchronize()
    return out


def check(m, out, scale=None, fill=7.0, label=""):
    DL = m["DL"]
    f = lambda t: t.double().numpy()  # noqa: E731
    want, A, S = L.attention(f(m["ql"]), f(m["qr"]), f(m["cache"]), m["table"], m["prefix"], m["par"], m["n"],
                             m["scale"] if scale is None else scale)
    got = out.double().cpu().numpy()
    bf16 = str(m["q"].dtype) == "torch.bfloat16"
    for b, n in enumerate(m["n"]):
        tol = tolerance(bf16, want[b, :n], A[b, :n], S[b, :n], int(m["prefix"][b]) + n, DL + L.ROPE)
        err = np.abs(got[b, :n] - want[b, :n])
        assert np.isfinite(got[b, :n]).all(), f"{label} sequence {b}: not finite"
        assert (err <= tol).all(), f"{label} sequence {b}: {float((err / tol).max())} of the tolerance"
        assert (got[b, n:] == fill).all(), f"{label} sequence {b}: rows past the tree were written"


SHAPES = [
    # heads, d_latent, prefix, sizes, block
    (16, 512, [0], [1], 0),
    (16, 512, [1], [1], 0),
    (1, 512, [31], [1], 0),
    (1, 512, [32], [1], 16),
    (128, 512, [100], [1], 64),
    (128, 512, [0], [3], 0),
    (16, 512, [63], [2], 0),
    (16, 512, [500], [60], 0),
    (16, 512, [700], [9], 1),
    (5, 512, [130], [65], 48),
    (16, 256, [300], [33], 64),
    (7, 256, [129], [100], 0),
    (3, 512, [257], [43], 128),
    (16, 512, [0, 1, 500], [5, 64, 17], 16),
    (16, 512, [100, 0, 64, 1000], [1, 1, 1, 1], 0),
    (8, 256, [65, 300], [70, 12], 16),
    (32, 512, [10, 200, 333, 64, 900], [40, 3, 9, 1, 16], 64),
    (128, 512, [90, 31], [9, 30], 0),
    (16, 256, [1500], [16], 0),
    (16, 512, [2100, 40], [1, 1], 64),
]


@pytest.mark.parametrize("dtype", ["bfloat16", "float32"])
@pytest.mark.parametrize("shape", SHAPES, ids=lambda s: "-".join(map(str, s)).replace(" ", ""))
def test_attention(shape, dtype):
    H, DL, prefix, sizes, block = shape
    m = make(sum(prefix) + H + DL, H, DL, prefix, sizes, block, dtype, layout="rows" if sum(sizes) % 2 else "heads")
    check(m, run(m), label=str(shape))


@pytest.mark.parametrize("kind", ["chain", "star"])
@pytest.mark.parametrize("dtype", ["bfloat16", "float32"])
@pytest.mark.parametrize("B", [1, 2])
def test_chains_and_stars_of_the_largest_size(kind, dtype, B):
    m = make(4, 2, 512, [100, 37][:B], [256, 130][:B], 32, dtype, kind)
    check(m, run(m), label=kind)
