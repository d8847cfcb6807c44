"""Rotary positions on the GPU against products of complex numbers in extended precision.

Tolerances, per element, with X the larger magnitude of its pair and m = |mscale|, h half a step of the type: the cosine
and the sine are off by at most 4 * 2^-24 (the reduced angle's rounding moves them by at most pi / 4 * 2^-24, the sums
by less than 2 * 2^-24, their product with m by 2^-24), and two products and a sum round by another 2 * 2^-24 of 2X; in
all 12 * 2^-24 * X * m, and the output rounds by h of itself.  The angle's own error in revolutions (float64) is below
2^-50 of a revolution per position in 2^30: nothing beside these.
"""
import numpy as np
import pytest

import latent_util as L
import paper_2603_01639_amd as ltd

pytestmark = pytest.mark.gpu


def make(seed, H, Hk, d, rot, off=0, inter=False, prefix=(5,), sizes=(3,), depth="tree", dtype="bfloat16", base=10000.0,
         m=1.0, N=None):
    import torch
    rng = np.random.default_rng(seed)
    B, N = len(prefix), N or max(max(sizes), 1)
    t = getattr(torch, dtype)
    x = lambda h: torch.from_numpy(rng.normal(size=(B, N, h, d)) * 3).to(t)  # noqa: E731
    dep = rng.integers(0, 9, (B, N)).astype(np.int32) if depth == "tree" else None
    return dict(q=x(H), k=x(Hk) if Hk else None, freq=L.frequencies(rot, base), rot=rot, off=off, inter=inter,
                prefix=np.array(prefix, np.int32), n=np.array(sizes, np.int32), dep=dep, m=m)


def want(c, x, fill):
    y = x.double().numpy().copy()
    B, N = y.shape[:2]
    pos = c["prefix"][:, None].astype(np.int64) + (np.arange(N) if c["dep"] is None else c["dep"])
    a, b = c["off"], c["off"] + c["rot"]
    tol = L.half_step(x.dtype) * np.abs(y)
    tol[..., :a] = tol[..., b:] = 0
    part = y[..., a:b]
    pair = np.abs(part).reshape(*part.shape[:-1], -1, 2).max(-1) if c["inter"] else np.maximum(*np.split(np.abs(part), 2, -1))
    pair = np.repeat(pair, 2, -1) if c["inter"] else np.concatenate([pair, pair], -1)
    y[..., a:b] = L.turn(part, pos[:, :, None], c["freq"], c["inter"], c["m"])
    tol[..., a:b] = 1.01 * L.half_step(x.dtype) * np.abs(y[..., a:b]) + 12 * 2.0 ** -24 * pair * abs(c["m"])
    past = np.arange(N) >= c["n"][:, None]
    y[past], tol[past] = fill, 0
    return y, tol


def call(c, q, q_out, k=None, k_out=None, **more):
    import torch
    ltd.tree_rope(q, q_out, L.to_dev(c["freq"]), L.to_dev(c["prefix"]), L.to_dev(c["n"]), k=k, k_out=k_out,
                  depth=L.to_dev(c["dep"]), rot_offset=c["off"], interleaved=c["inter"], mscale=c["m"], **more)
    torch.cuda.synchronize()


def compare(c, x, out, fill, label):
    y, tol = want(c, x, fill)
    err = np.abs(out.double().cpu().numpy() - y)
    assert (err <= tol).all(), f"{label}: {float((err / np.maximum(tol, 1e-300)).max())} of the tolerance"


CASES = [
    dict(H=1, Hk=0, d=2, rot=2),
    dict(H=8, Hk=2, d=128, rot=128, prefix=(2041,), sizes=(60,)),
    dict(H=8, Hk=2, d=128, rot=128, inter=True, prefix=(2041, 0), sizes=(33, 7)),
    dict(H=5, Hk=5, d=64, rot=32, prefix=(0, 1, 70), sizes=(1, 0, 9)),
    dict(H=4, Hk=1, d=96, rot=36, inter=True, off=8, prefix=(11,), sizes=(20,)),
    dict(H=4, Hk=1, d=96, rot=36, off=3, prefix=(11,), sizes=(20,)),
    dict(H=3, Hk=2, d=33, rot=6, inter=True, off=5, prefix=(3, 4), sizes=(6, 2)),
    dict(H=16, Hk=0, d=64, rot=64, prefix=(1000000,), sizes=(256,), m=1.3, base=500000.0),
    dict(H=2, Hk=2, d=128, rot=64, inter=True, prefix=((1 << 30) - 300,), sizes=(200,), depth="rows", base=1e6),
    dict(H=2, Hk=1, d=256, rot=256, prefix=(0, 100), sizes=(4100, 77), depth="rows"),
    dict(H=1, Hk=1, d=4096, rot=4096, prefix=(17,), sizes=(3,)),
    dict(H=40, Hk=40, d=128, rot=128, prefix=(9,) * 5, sizes=(700, 1, 0, 1300, 999), depth="rows"),
]


@pytest.mark.parametrize("dtype", ["bfloat16", "float32"])
@pytest.mark.parametrize("case", CASES, ids=lambda c: "-".join(f"{k}{v}" for k, v in c.items()).replace(" ", ""))
def test_rope(case, dtype):
    import torch
    c = make(case["d"] + case["rot"], dtype=dtype, **case)
    q, k = c["q"].to("cuda"), None if c["k"] is None else c["k"].to("cuda")
    qo, ko = torch.full_like(q, 7.0), None if k is None else torch.full_like(k, 7.0)
    call(c, q, qo, k, ko)
    compare(c, c["q"], qo, 7.0, "q")
    if k is not None:
        compare(c, c["k"], ko, 7.0, "k")
        # in place, and the same result to the bit (rows past the count keep what they held)
        call(c, q, q, k, k)
        for x, out, was in ((q, qo, c["q"]), (k, ko, c["k"])):
            past = torch.arange(x.shape[1]) >= torch.from_numpy(c["n"])[:, None]
            assert torch.equal(x.cpu()[~past], out.cpu()[~past])
            assert torch.equal(x.cpu()[past], was[past])


@pytest.mark.parametrize("inter", [False, True])
@pytest.mark.parametrize("dtype", ["bfloat16", "float32"])
@pytest.mark.parametrize("lead", [0, 8, 3])
def test_views_of_a_fused_projection(lead, inter, dtype):
    """q and k as slices of one buffer, in place; what lies between them stays.  A lead of 3 elements leaves
    nothing aligned."""
    import torch
    c = make(9, 4, 2, 64, 64, inter=inter, prefix=(100, 7), sizes=(17, 30), dtype=dtype)
    B, N = c["q"].shape[:2]
    width = lead + 4 * 64 + 2 * 64 + 128
    buf = torch.full((B, N, width), 3.0, dtype=c["q"].dtype, device="cuda")
    qv = buf[:, :, lead:lead + 256].unflatten(2, (4, 64))
    kv = buf[:, :, lead + 256:lead + 384].unflatten(2, (2, 64))
    qv.copy_(c["q"])
    kv.copy_(c["k"])
    call(c, qv, qv, kv, kv)
    for x, v in (("q", qv), ("k", kv)):
        y, tol = want(c, c[x], 0)
        past = np.arange(N) >= c["n"][:, None]
        y[past] = c[x].double().numpy()[past]
        assert (np.abs(v.double().cpu().numpy() - y) <= tol).all(), x
    assert (buf[:, :, :lead] == 3).all() and (buf[:, :, lead + 384:] == 3).all()


def test_heads_before_rows():
    """[Hq][B][Nmax][d] storage, as a product per head leaves it, into rows."""
    import torch
    c = make(12, 6, 0, 64, 64, prefix=(8, 9), sizes=(5, 12))
    q = c["q"].to("cuda").permute(2, 0, 1, 3).contiguous().permute(1, 2, 0, 3)
    out = torch.full_like(c["q"], 7.0, device="cuda")
    call(c, q, out)
    compare(c, c["q"], out, 7.0, "q")


def test_nan_and_infinity_stay_in_their_pairs():
    import torch
    c = make(5, 2, 0, 64, 64, prefix=(3,), sizes=(4,))
    c["q"][0, 1, 0, 5], c["q"][0, 2, 1, 40] = float("nan"), float("inf")
    q = c["q"].to("cuda")
    out = torch.full_like(q, 7.0)
    call(c, q, out)
    bad = ~torch.isfinite(out.cpu())
    want_bad = torch.zeros_like(bad)
    want_bad[0, 1, 0, [5, 37]] = want_bad[0, 2, 1, [8, 40]] = True
    assert torch.equal(bad, want_bad)


def test_validation():
    import torch
    c = make(6, 2, 1, 64, 64, prefix=(3, 4), sizes=(4, 2))
    q, k = c["q"].to("cuda"), c["k"].to("cuda")

    def status(**kw):
        d = dict(c, **kw)
        st = torch.full((1,), -9, dtype=torch.int32, device="cuda")
        qo, ko = torch.full_like(q, 7.0), torch.full_like(k, 7.0)
        call(d, q, qo, k, ko, validate=True, status=st)
        wrote = bool((qo != 7).any() or (ko != 7).any())
        return int(st), wrote

    i = lambda *v: np.array(v, np.int32)  # noqa: E731
    assert status() == (ltd.STATUS_OK, True)
    assert status(n=i(4, 5)) == (ltd.STATUS_BAD_NNODES, False)
    assert status(n=i(-1, 1)) == (ltd.STATUS_BAD_NNODES, False)
    assert status(prefix=i(3, -1)) == (ltd.STATUS_BAD_PREFIX, False)
    assert status(prefix=i((1 << 30) - 2, 0)) == (ltd.STATUS_BAD_PREFIX, False)
    dep = c["dep"].copy()
    dep[1, 1] = -1
    assert status(dep=dep) == (ltd.STATUS_BAD_PREFIX, False)
    assert status(dep=dep, n=i(4, 1)) == (ltd.STATUS_OK, True)
    assert status(prefix=i(-1, 0), n=i(4, 9)) == (ltd.STATUS_BAD_PREFIX, False)  # the lowest sequence's
