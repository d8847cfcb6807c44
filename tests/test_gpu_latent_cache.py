"""The latent cache's writes on the GPU: appending rows (norm, rotation) and moving the accepted ones.

Tolerances, per element, h half a step of the type: the mean square is a float32 sum of 512 or 256 squares (each rounds,
and the sum's tree of additions by at most 16 steps: 20 * 2^-24 relative at most), its root and reciprocal another 3 *
2^-24, and two products 2 * 2^-24: 0.5 * 20 + 3 + 2 = 15 * 2^-24 of the value, which then rounds by h.  The rotated part
as in the rotary positions' tests: 12 * 2^-24 of the pair's larger magnitude, and h of the value.
"""
import numpy as np
import pytest

import latent_util as L
import paper_2603_01639_amd as ltd

pytestmark = pytest.mark.gpu


def make(seed, DL, prefix, sizes, block=0, dtype="bfloat16", norm=True, inter=True, depth=True, lead=0, m=1.0):
    import torch
    rng = np.random.default_rng(seed)
    B, N, D = len(prefix), max(max(sizes), 1), DL + L.ROPE
    rows = [p + n for p, n in zip(prefix, sizes)]
    t = getattr(torch, dtype)
    pages, table = L.make_table(rng, rows, block) if block else (B, None)
    R = block or max(rows) + 3
    buf = torch.from_numpy(rng.normal(size=(B, N, lead + D)) * np.exp(rng.normal(size=(B, N, 1)))).to(t)
    return dict(cache=torch.from_numpy(rng.normal(size=(pages, R, D))).to(t), table=table, buf=buf, lead=lead, DL=DL,
                w=torch.from_numpy(1 + 0.3 * rng.normal(size=DL)).to(t) if norm else None, freq=L.frequencies(L.ROPE),
                prefix=np.array(prefix, np.int32), n=np.array(sizes, np.int32), inter=inter, eps=1e-5, m=m,
                dep=rng.integers(0, 9, (B, N)).astype(np.int32) if depth else None)


def call(c, cache, buf=None, **more):
    import torch
    new = (c["buf"].to("cuda") if buf is None else buf)[:, :, c["lead"]:]
    table = L.to_dev(c["table"])
    ltd.latent_append(new, cache, L.to_dev(c["freq"]), L.to_dev(c["prefix"]), L.to_dev(c["n"]), depth=L.to_dev(c["dep"]),
                      norm_weight=None if c["w"] is None else c["w"].to("cuda"), norm_eps=c["eps"],
                      interleaved=c["inter"], mscale=c["m"], block_table=table,
                      num_blocks=0 if table is None else cache.shape[0], **more)
    torch.cuda.synchronize()


def want(c):
    """The cache after the append, and the tolerance (0 where no row is written)."""
    y = c["cache"].double().numpy().copy()
    tol = np.zeros_like(y)
    h, DL = L.half_step(c["buf"].dtype), c["DL"]
    x = c["buf"][:, :, c["lead"]:].double().numpy()
    for b, n in enumerate(c["n"]):
        for i in range(n):
            page, r = L.place(c["table"], b, int(c["prefix"][b]) + i, y.shape[1])
            lat = x[b, i, :DL]
            if c["w"] is not None:
                lat = lat / np.sqrt((lat ** 2).mean() + c["eps"]) * c["w"].double().numpy()
                tol[page, r, :DL] = 1.01 * (h + 15 * 2.0 ** -24) * np.abs(lat)
            part = x[b, i, DL:]
            pos = int(c["prefix"][b]) + (i if c["dep"] is None else int(c["dep"][b, i]))
            rot = L.turn(part, np.int64(pos), c["freq"], c["inter"], c["m"])
            pair = np.abs(part).reshape(-1, 2).max(-1) if c["inter"] else np.maximum(*np.split(np.abs(part), 2))
            pair = np.repeat(pair, 2) if c["inter"] else np.concatenate([pair, pair])
            tol[page, r, DL:] = 1.01 * h * np.abs(rot) + 12 * 2.0 ** -24 * pair * abs(c["m"])
            y[page, r] = np.concatenate([lat, rot])
    return y, tol


CASES = [
    dict(DL=512, prefix=(0,), sizes=(1,)),
    dict(DL=512, prefix=(2041,), sizes=(60,)),
    dict(DL=256, prefix=(7,), sizes=(33,), inter=False, lead=8),
    dict(DL=512, prefix=(0, 5, 100), sizes=(9, 0, 17), block=16, inter=False),
    dict(DL=512, prefix=(63, 64), sizes=(2, 65), block=64, norm=False),
    dict(DL=256, prefix=(1, 2, 3, 4), sizes=(1, 1, 1, 1), block=1, m=0.7),
    dict(DL=512, prefix=(0, 0), sizes=(700, 1111), depth=False, block=48, lead=1024),
]


@pytest.mark.parametrize("dtype", ["bfloat16", "float32"])
@pytest.mark.parametrize("case", CASES, ids=lambda c: "-".join(f"{k}{v}" for k, v in c.items()).replace(" ", ""))
def test_append(case, dtype):
    c = make(case["DL"] + sum(case["sizes"]), dtype=dtype, **case)
    cache = c["cache"].to("cuda")
    call(c, cache)
    y, tol = want(c)
    err = np.abs(cache.double().cpu().numpy() - y)
    assert (err <= tol).all(), f"{float((err / np.maximum(tol, 1e-300)).max())} of the tolerance"


def test_append_of_zero_rows_and_nan():
    """A row of zeros stays zeros under the norm; a NaN stays in its row."""
    import torch
    c = make(3, 512, (4,), (3,))
    c["buf"][0, 0] = 0
    c["buf"][0, 1, 17] = float("nan")
    cache = c["cache"].to("cuda")
    call(c, cache)
    assert (cache[0, 4] == 0).all()
    assert torch.isnan(cache[0, 5, :512]).all() and torch.isfinite(cache[0, 5, 512:]).all()
    assert torch.isfinite(cache[0, 6]).all()


def test_append_validation():
    import torch
    c = make(4, 512, (3, 20), (4, 2), block=16)

    def status(**kw):
        d = dict(c, **kw)
        st = torch.full((1,), -9, dtype=torch.int32, device="cuda")
        cache = c["cache"].to("cuda")
        call(d, cache, validate=True, status=st)
        return int(st), not torch.equal(cache.cpu(), c["cache"])

    i = lambda *v: np.array(v, np.int32)  # noqa: E731
    assert status() == (ltd.STATUS_OK, True)
    assert status(n=i(5, 2)) == (ltd.STATUS_BAD_NNODES, False)
    assert status(prefix=i(-1, 20)) == (ltd.STATUS_BAD_PREFIX, False)
    assert status(prefix=i(3, 31)) == (ltd.STATUS_BAD_PREFIX, False)
    bad = c["table"].copy()
    bad[1, 1] = c["cache"].shape[0]
    assert status(table=bad) == (ltd.STATUS_BAD_BLOCK, False)


@pytest.mark.parametrize("dtype", ["bfloat16", "float32"])
@pytest.mark.parametrize("layers, DL, prefix, sizes, block", [
    (1, 512, (5,), (8,), 0), (3, 512, (0, 63, 10), (40, 60, 1), 16), (2, 256, (100, 7), (256, 130), 64),
    (1, 512, (9,), (256,), 1), (4, 256, (3, 3), (17, 20), 0)])
def test_compact(layers, DL, prefix, sizes, block, dtype):
    import torch
    rng = np.random.default_rng(layers + DL + sum(sizes))
    B, N, D = len(prefix), max(sizes), DL + L.ROPE
    pages, table = L.make_table(rng, [p + n for p, n in zip(prefix, sizes)], block) if block else (B, None)
    R = block or max(p + n for p, n in zip(prefix, sizes)) + 2
    cache = torch.from_numpy(rng.normal(size=(layers, pages, R, D))).to(getattr(torch, dtype))
    path, nacc = np.full((B, N), -5, np.int32), np.zeros(B, np.int32)
    for b, n in enumerate(sizes):
        k = int(rng.integers(1, n + 1)) if n < 200 else n // 2
        path[b, :k] = np.r_[0, np.sort(rng.choice(np.arange(1, n), k - 1, replace=False))] if k > 1 else [0]
        nacc[b] = k
    want = cache.clone()
    for b, P in enumerate(prefix):
        for j in range(nacc[b]):
            sp, sr = L.place(table, b, P + int(path[b, j]), R)
            dp, dr = L.place(table, b, P + j, R)
            want[:, dp, dr] = cache[:, sp, sr]
    got = cache.to("cuda") if layers > 1 else cache[0].to("cuda")
    new = torch.full((B,), -1, dtype=torch.int32, device="cuda")
    ltd.latent_compact(got, L.to_dev(np.array(prefix, np.int32)), new, L.to_dev(path), L.to_dev(nacc),
                       block_table=L.to_dev(table), num_blocks=pages if block else 0)
    torch.cuda.synchronize()
    # (rows past the accepted ones keep what they held: the whole cache is compared)
    assert torch.equal(got.cpu().reshape(want.shape), want)
    assert new.cpu().tolist() == [p + int(k) for p, k in zip(prefix, nacc)]


def test_compact_validation():
    import torch
    cache = torch.randn((1, 40, 576), device="cuda").bfloat16()
    was = cache.clone()
    i = lambda *v: torch.tensor(v, dtype=torch.int32, device="cuda")  # noqa: E731
    for path, n, P, code in (([0, 2, 1, 0], 3, 5, ltd.STATUS_BAD_PATH), ([0, 2, 3, 0], 5, 5, ltd.STATUS_BAD_PATH),
                             ([0, 2, 3, 0], 3, 37, ltd.STATUS_BAD_PREFIX)):
        st, new = i(-9), i(-1)
        ltd.latent_compact(cache, i(P), new, i(*path)[None], i(n), validate=True, status=st)
        torch.cuda.synchronize()
        assert int(st) == code and int(new) == -1 and torch.equal(cache, was)


# ---- caches that 32 bits do not reach: only the rows of the case are filled

@pytest.mark.parametrize("block", [0, 1, 48])
@pytest.mark.parametrize("dtype", ["bfloat16", "float32"])
def test_append_past_32_bits(dtype, block):
    import torch
    c = make(21, 512, (40, 3, 100), (9, 30, 1), block=block, dtype=dtype)
    size = c["cache"].element_size()
    if block:
        pages, used = 5 * 10 ** 9 // (576 * block * size), c["cache"].shape[0]
        big = torch.empty((pages, block, 576), dtype=c["cache"].dtype, device="cuda")
        view = big[pages - used:]
        c["moved"] = dict(c, table=np.where(c["table"] < 0, c["table"], c["table"] + pages - used).astype(np.int32))
    else:
        R, used = 5 * 10 ** 9 // (2 * 576 * size) + 3, c["cache"].shape[1]
        big = torch.empty((3, R, 576), dtype=c["cache"].dtype, device="cuda")
        view = big[:, :used]
        c["moved"] = c
    view.copy_(c["cache"])
    call(c["moved"], big)
    y, tol = want(c)
    assert (np.abs(view.double().cpu().numpy() - y) <= tol).all()


@pytest.mark.parametrize("block", [0, 16])
def test_compact_past_32_bits(block):
    """The second of two layers begins past 2^32 bytes, and the pages in use are a layer's last."""
    import torch
    rng = np.random.default_rng(22)
    P, n, acc = 45, 20, [0, 3, 4, 11, 19]
    R = block or 2_000_003
    pages = 250_000 if block else 1
    cache = torch.empty((2, pages, R, 576), dtype=torch.bfloat16, device="cuda")
    cache = cache if block else torch.empty((2, 2, R, 576), dtype=torch.bfloat16, device="cuda")
    assert cache[1].data_ptr() - cache.data_ptr() > 2 ** 32
    rows = torch.from_numpy(rng.normal(size=(2, 64 + 16, 576))).bfloat16().cuda()
    if block:
        table = (pages - 1 - rng.permutation(5)).astype(np.int32)[None]
        for k, page in enumerate(table[0]):
            cache[:, page] = rows[:, 16 * k:16 * k + 16]
        one = lambda v: L.to_dev(np.array([v], np.int32))  # noqa: E731
    else:
        table = None
        cache[:, 1, :80] = rows
        cache[:, 0, :80] = 0
        one = lambda v: L.to_dev(np.array([0, v], np.int32))  # noqa: E731
    B = 1 if block else 2
    path = np.zeros((B, n), np.int32)
    path[B - 1, :len(acc)] = acc
    new = torch.zeros((B,), dtype=torch.int32, device="cuda")
    nacc = one(len(acc)) if block else L.to_dev(np.array([1, len(acc)], np.int32))
    ltd.latent_compact(cache, one(P), new, L.to_dev(path), nacc, block_table=L.to_dev(table), num_blocks=pages if block else 0)
    torch.cuda.synchronize()
    want = rows.clone()
    for j, a in enumerate(acc):
        want[:, P + j] = rows[:, P + a]
    got = torch.cat([cache[:, p] for p in table[0]], 1) if block else cache[:, 1, :80]
    assert torch.equal(got, want)
    assert int(new[-1]) == P + len(acc)
