"""Tree attention over an 8-bit cache on the GPU against softmax attention in 64 bits over the values that the codes
stand for.

Tolerances, per output element, with A the same weighted mean of |v|, o the output, S the largest scaled sum of
|q||k| of its row and T its keys.  Scores are float32 sums of exact products: off by at most
e = S * (d + 8) * 2^-24, which moves a weight by a factor within e^(+-2e), so the output by about 4e * A; the
exponent's own rounding is of the size of |m * c| * 2^-24 <= 2S * 2^-24 and is covered by the 8 in e.
bfloat16 (half a step is 2^-8): weights are rounded once and normalised by the rounded ones' sum (2^-8 * (A + |o|)),
pieces of a row are stored rounded (2^-8 * A), the output is rounded (2^-8 * |o|).
float32 (half a step is 2^-24): T + 32 additions of weights and products, 2 * (T + 32) * 2^-24 * A, and the exponential
within 2 ulp, 4 * 2^-24 * A.
"""
import numpy as np
import pytest

import paper_2603_01639_amd as ltd
import q8_util as Q

pytestmark = pytest.mark.gpu


def tolerance(bf16, o, A, S, T, d):
    e = (S * (d + 8) * 2.0 ** -24)[..., None]
    base = 4 * e * A
    if bf16:
        return 1.02 * (base + 2.0 ** -8 * (2 * A + 2 * np.abs(o))) + 1e-30
    return base + (2 * (T + 32) + 4) * 2.0 ** -24 * A + 1e-30


def make(seed, B, Hq, Hkv, d, sr, prefix, sizes, block=0, dtype="bfloat16", kind="random", qstd=1.5, spread=2, nmax=None,
         extra=1):
    import torch
    rng = np.random.default_rng(seed)
    c = Q.cache(rng, B, Hkv, d, sr, [p + n for p, n in zip(prefix, sizes)], block, spread=spread, extra=extra)
    for k in "kv":  # values spread as a cache's: few codes near the largest
        x = np.clip(rng.normal(size=c[k].shape) * 110, -448, 448)
        c[k] = Q.encode(x)
    par = Q.trees(rng, sizes, kind)
    if nmax:
        par = np.pad(par, ((0, 0), (0, nmax - par.shape[1])), constant_values=-7)
    q = torch.from_numpy(rng.normal(size=(B, par.shape[1], Hq, d)) * qstd).to(getattr(torch, dtype))
    return dict(c=c, par=par, q=q, prefix=np.array(prefix, np.int32), n=np.array(sizes, np.int32), sr=sr)


def run(m, fill=7.0, max_prefix=None, scale=None, dev=None, out=None, workspace=None, **more):
    import torch
    dev = dev or Q.dev_cache(m["c"])
    q = m["q"].to("cuda")
    out = torch.full_like(q, fill) if out is None else out
    ltd.tree_verify_attn_q8(q, dev["k"], dev["v"], dev["ks"], dev["vs"], Q.to_dev(m["prefix"]), Q.to_dev(m["par"]),
                            Q.to_dev(m["n"]), out, max_prefix=int(m["prefix"].max()) if max_prefix is None else max_prefix,
                            scale_rows=m["sr"], block_table=dev["table"], num_blocks=m["c"]["pages"], scale=scale,
                            workspace=workspace, **more)
    torch.cuda.synchronize()
    return out


def check(m, out, scale=None, fill=7.0, label=""):
    d, sr = m["q"].shape[-1], m["sr"]
    k, v = (Q.values(m["c"], w, m["c"]["table"], sr) for w in "kv")
    q = m["q"].double().numpy()
    want, A, S = Q.attention(q, k, v, m["prefix"], m["par"], m["n"], d ** -0.5 if scale is None else scale)
    got = out.double().cpu().numpy()
    bf16 = str(m["q"].dtype) == "torch.bfloat16"
    for b, n in enumerate(m["n"]):
        tol = tolerance(bf16, want[b, :n], A[b, :n], S[b, :n], int(m["prefix"][b]) + n, d)
        err = np.abs(got[b, :n] - want[b, :n])
        assert np.isfinite(got[b, :n]).all(), f"{label} sequence {b}: not finite"
        assert (err <= tol).all(), f"{label} sequence {b}: {float((err / tol).max())} of the tolerance"
        assert (got[b, n:] == fill).all(), f"{label} sequence {b}: rows past the tree were written"


SHAPES = [
    # B, Hq, Hkv, d, sr, prefix, sizes, block
    (1, 8, 2, 128, 16, [0], [1], 0),
    (1, 8, 2, 128, 16, [1], [1], 0),
    (1, 8, 2, 128, 64, [63], [2], 0),
    (1, 4, 4, 128, 32, [64], [64], 32),
    (1, 8, 1, 128, 16, [130], [65], 16),
    (1, 32, 8, 128, 128, [700], [60], 0),
    (1, 8, 2, 64, 16, [300], [33], 48),
    (1, 8, 8, 64, 64, [129], [7], 64),
    (1, 64, 8, 128, 64, [1000], [8], 128),
    (1, 5, 1, 128, 16, [257], [100], 16),
    (3, 8, 2, 128, 16, [0, 1, 500], [5, 64, 17], 16),
    (4, 8, 2, 128, 32, [100, 0, 64, 1000], [1, 1, 1, 1], 0),
    (2, 8, 4, 64, 16, [65, 300], [70, 12], 16),
    (5, 16, 2, 128, 64, [10, 200, 333, 64, 900], [40, 3, 90, 1, 16], 64),
    (2, 8, 1, 64, 128, [500, 128], [256, 100], 128),
    (2, 3, 3, 128, 16, [90, 31], [9, 30], 48),
]


@pytest.mark.parametrize("dtype", ["bfloat16", "float32"])
@pytest.mark.parametrize("shape", SHAPES, ids=lambda s: "-".join(map(str, s)).replace(" ", ""))
def test_attention(shape, dtype):
    B, Hq, Hkv, d, sr, prefix, sizes, block = shape
    m = make(sum(prefix) + sr + d, B, Hq, Hkv, d, sr, prefix, sizes, block, dtype)
    check(m, run(m), label=str(shape))


@pytest.mark.parametrize("kind", ["chain", "star"])
@pytest.mark.parametrize("dtype", ["bfloat16", "float32"])
@pytest.mark.parametrize("B", [1, 2])
def test_chains_and_stars_of_the_largest_size(kind, dtype, B):
    m = make(4, B, 4, 2, 128, 32, [100, 37][:B], [256, 130][:B], 32, dtype, kind)
    check(m, run(m), label=kind)


@pytest.mark.parametrize("spread", [0, 40])
def test_scales_far_apart(spread):
    """Blocks whose scales differ by up to 2^40, K's and V's apart: exact powers of two, whatever their size."""
    m = make(9, 2, 8, 2, 128, 16, [200, 77], [12, 30], 16, spread=2)
    rng = np.random.default_rng(2)
    c = m["c"]
    c["vs"] = rng.integers(127 - 8 - spread // 2, 127 - 8 + spread // 2 + 1, c["vs"].shape).astype(np.uint8)
    c["ks"] = rng.integers(110, 121, c["ks"].shape).astype(np.uint8)
    check(m, run(m), label=f"spread {spread}")


@pytest.mark.parametrize("dtype", ["bfloat16", "float32"])
def test_smallest_and_largest_scale_bytes(dtype):
    """Blocks at both ends of what an append writes; V at 2^-100 and 2^87 exactly."""
    for byte, qs in ((Q.E_MIN, 2.0 ** 60), (Q.E_MAX, 2.0 ** -60)):
        m = make(byte, 1, 4, 1, 128, 16, [90], [6], 0, dtype)
        c = m["c"]
        c["vs"][:] = byte
        c["ks"][:] = byte
        k = c["k"]
        q = m["q"].double() * qs
        m["q"] = q.to(m["q"].dtype)
        scale = float(2.0 ** (119 - byte) / qs / 11)
        check(m, run(m, scale=scale), scale=scale, label=f"byte {byte}")


@pytest.mark.parametrize("dtype", ["bfloat16", "float32"])
@pytest.mark.parametrize("B", [1, 3])
def test_rows_outside_the_sequences_may_hold_nan(dtype, B):
    """Rows past a tree, unused pages and rows of padded nodes hold NaN codes and wild scale bytes."""
    m = make(31, B, 8, 2, 128, 16, [70, 20, 131][:B], [5, 9, 30][:B], 16, dtype, nmax=40)
    c = m["c"]
    for w in "kv":
        used = np.zeros(c[w].shape[:3], bool)
        groups = np.zeros(c[w + "s"].shape, bool)
        for b in range(B):
            for r in range(int(m["prefix"][b] + m["n"][b])):
                p, x = Q.place(c["table"], b, r, c["R"])
                used[p, :, x] = True
                groups[p, :, x // 16] = True
        c[w][~used] = 0x7F
        c[w + "s"][~groups] = 255
    m["q"][:, -1] = float("nan")
    check(m, run(m), label="nan outside")


@pytest.mark.parametrize("dtype", ["bfloat16", "float32"])
@pytest.mark.parametrize("B, n", [(1, 12), (1, 70), (2, 12), (2, 130)])
def test_nan_in_a_tree_row_reaches_its_descendants_only(dtype, B, n):
    m = make(n, B, 4, 2, 128, 32, [100, 9][:B], [n, n - 3][:B], 0, dtype)
    c, bad = m["c"], 4
    for w in "kv":
        for b in range(B):
            p, x = Q.place(c["table"], b, int(m["prefix"][b]) + bad, c["R"])
            c[w][p, 1, x, 7] = 0x7F
    out = run(m).double().cpu().numpy()
    clean = {w: c[w].copy() for w in "kv"}
    for w in "kv":
        clean[w][np.isnan(Q.VALUES[c[w]])] = 0
    k, v = (Q.values(dict(c, **clean), w, c["table"], m["sr"]) for w in "kv")
    want, A, S = Q.attention(m["q"].double().numpy(), k, v, m["prefix"], m["par"], m["n"], 128 ** -0.5)
    for b in range(B):
        nb = int(m["n"][b])
        sees = np.array([bad in p for p in Q.paths(m["par"][b, :nb])])
        got = out[b, :nb]
        assert np.isnan(got[sees][:, 2:]).any(-1).all()  # kv head 1 serves query heads 2 and 3
        calm = got.copy()
        calm[sees, 2:] = want[b, :nb][sees, 2:]
        tol = tolerance(dtype == "bfloat16", want[b, :nb], A[b, :nb], S[b, :nb], int(m["prefix"][b]) + nb, 128)
        assert (np.abs(calm - want[b, :nb]) <= tol).all()


@pytest.mark.parametrize("dtype", ["bfloat16", "float32"])
def test_large_scores(dtype):
    """Rows whose softmax is all but one key's."""
    m = make(6, 2, 8, 2, 128, 16, [300, 64], [20, 33], 16, dtype, qstd=40.0)
    check(m, run(m), label="large")


def test_loose_bounds_and_a_dirty_workspace():
    import torch
    m = make(14, 3, 16, 2, 128, 32, [64, 5, 400], [7, 1, 33], 32, nmax=256)
    size = ltd.attn_q8_workspace_size(3, 256, 16, 2, 128, 9000, ltd.DTYPE_BF16)
    ws = torch.full((max(16, size),), 0xFF, dtype=torch.uint8, device="cuda")
    check(m, run(m, max_prefix=9000, workspace=ws), label="loose")


def test_same_answer_twice_and_from_a_graph():
    """Two runs are bit-identical, and so is every replay of a captured one between eager calls on other data."""
    import torch
    m = make(77, 4, 32, 8, 128, 16, [700, 30, 333, 64], [20, 1, 64, 33], 16)
    other = make(78, 4, 32, 8, 128, 16, [700, 30, 333, 64], [20, 1, 64, 33], 16)
    dev = Q.dev_cache(m["c"])
    first, second = run(m, dev=dev), run(m, dev=dev)
    assert torch.equal(first.view(torch.int16), second.view(torch.int16))
    size = ltd.attn_q8_workspace_size(4, 64, 32, 8, 128, 700, ltd.DTYPE_BF16)
    ws = torch.empty(size, dtype=torch.uint8, device="cuda")
    ints = [Q.to_dev(m[k]) for k in ("prefix", "par", "n")]
    q, out = m["q"].to("cuda"), torch.full_like(first, 7.0)
    call = lambda: ltd.tree_verify_attn_q8(q, dev["k"], dev["v"], dev["ks"], dev["vs"], *ints, out, max_prefix=700,  # noqa: E731
                                           scale_rows=16, block_table=dev["table"], num_blocks=m["c"]["pages"], workspace=ws)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.stream(side):
        call()
        side.synchronize()
        with torch.cuda.graph(graph, stream=side):
            call()
    for _ in range(4):
        out.fill_(7.0)
        ws.fill_(0xFF)
        run(other)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out.view(torch.int16), first.view(torch.int16))


def test_validation_reports_bad_data_and_writes_nothing():
    import torch
    m = make(3, 2, 4, 2, 64, 16, [40, 20], [6, 9], 16)
    status = torch.full((1,), 9, dtype=torch.int32, device="cuda")
    check(m, run(m, validate=True, status=status))
    assert int(status.cpu()[0]) == 0
    m["par"][1, 4] = 4
    out = run(m, validate=True, status=status)
    assert int(status.cpu()[0]) == ltd.STATUS_BAD_PARENT
    assert (out == 7.0).all()


@pytest.mark.parametrize("B, prefix, sizes, Hq, Hkv, d", [
    (1, [5000], [4], 8, 1, 128), (70, None, None, 8, 8, 64), (130, None, None, 4, 4, 128), (3, [0, 0, 0], [1, 2, 3], 8, 1, 128),
    (2, [9000, 1], [1, 4], 8, 1, 128), (5, [128, 129, 127, 64, 4000], [8, 1, 8, 3, 2], 4, 1, 64)])
def test_short_units(B, prefix, sizes, Hq, Hkv, d):
    """At most 32 stacked rows a unit, cut into splits of one length on the GPU: one sequence, more than 64 of them,
    empty and very different prefixes, lengths around a split's."""
    rng = np.random.default_rng(B)
    prefix = prefix or [int(x) for x in rng.integers(0, 400, B)]
    sizes = sizes or [int(x) for x in rng.integers(1, 9, B)]
    m = make(B + d, B, Hq, Hkv, d, 16, prefix, sizes, 16)
    check(m, run(m), label="short units")
    check(m, run(m, max_prefix=40000), label="short units, loose bound")


@pytest.mark.parametrize("sizes", [[3, 1], [40, 9]])
def test_bounds_beyond_the_matrix_kernels(sizes):
    """A max_prefix past what the matrix-core kernels plan for with such pages: the vector kernel takes the calls."""
    m = make(1, 2, 8, 2, 128, 32, [90, 33], sizes, 32)
    check(m, run(m, max_prefix=9_000_000), label="far bound")
