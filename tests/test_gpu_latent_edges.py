"""Latent attention on the GPU where it can go wrong: what masked rows hold, scores that move the running maximum, batches
longer than a wave, a few rows a sequence, large caches, layouts, streams and validation.  Tolerances are those of the
attention tests beside this file."""
import numpy as np
import pytest

import latent_util as L
import paper_2603_01639_amd as ltd
from test_gpu_latent_attention import check, make, parts, run

pytestmark = pytest.mark.gpu

FEW = [  # heads, nodes: up to 16 rows a sequence
    (1, 16), (2, 8), (3, 5), (4, 4), (5, 3), (8, 2), (16, 1), (1, 1), (7, 2)]


@pytest.mark.parametrize("kind", ["random", "chain", "star"])
@pytest.mark.parametrize("H, n", FEW)
def test_few_rows(H, n, kind):
    """Trees that begin at every place of a tile, in shares of every length."""
    for DL, block, prefix in ((512, 0, [0, 15, 16, 17, 130, 4000]), (256, 24, [1, 2, 3, 29, 640, 20]), (512, 7, [2500] * 3)):
        sizes = [n, max(n - 1, 0), n, 1, n, 0][:len(prefix)]
        m = make(H * 100 + n + DL, H, DL, prefix, sizes, block, kind=kind, nmax=n)
        check(m, run(m), label=f"{H} heads, {n} nodes, d {DL}, blocks {block}")


def poisoned(m, rows_of):
    """The case's cache with rows_of(sequence) = {row: (first dim, value)} overwritten."""
    import torch
    cache = m["cache"].clone()
    for b in range(len(m["n"])):
        for r, (dim, v) in rows_of(b).items():
            page, at = L.place(m["table"], b, r, cache.shape[1])
            cache[page, at, dim] = v
    return cache.to("cuda"), torch


SIZES = [(16, 512, [37, 200], [9, 33], 16), (128, 512, [64], [40], 0), (3, 256, [0, 5, 1000], [5, 5, 3], 8),
         (16, 512, [3000, 11], [1, 1], 0), (40, 256, [90, 700], [4, 77], 0)]


@pytest.mark.parametrize("value", [float("nan"), float("inf"), float("-inf")])
@pytest.mark.parametrize("dtype", ["bfloat16", "float32"])
@pytest.mark.parametrize("shape", SIZES, ids=lambda s: "-".join(map(str, s)).replace(" ", ""))
def test_tree_rows_that_hold_no_number(shape, dtype, value):
    """A node's NaN or infinity, in either part of its row, reaches the nodes below it and no others."""
    H, DL, prefix, sizes, block = shape
    m = make(DL + H, H, DL, prefix, sizes, block, dtype)
    for dim in (0, DL - 1, DL + 3):
        at = [n // 2 for n in sizes]
        cache, torch = poisoned(m, lambda b: {int(m["prefix"][b]) + at[b]: (dim, value)})
        out = run(m, cache=cache)
        clean = run(m)
        for b, n in enumerate(sizes):
            below = np.array([at[b] in L.root_path(m["par"][b], i) for i in range(n)])
            got = out[b, :n].double().cpu().numpy()
            if dim < DL:
                # the poisoned dimension of every head of a node that sees the row (its weight is above 0, or its
                # product with the value has no number either)
                assert not np.isfinite(got[below][:, :, dim]).any(), (b, dim)
            elif np.isnan(value):
                assert np.isnan(got[below]).all(), (b, dim)
            assert torch.equal(out[b, :n][torch.from_numpy(~below)], clean[b, :n][torch.from_numpy(~below)]), (b, dim)


@pytest.mark.parametrize("dtype", ["bfloat16", "float32"])
@pytest.mark.parametrize("shape", SIZES, ids=lambda s: "-".join(map(str, s)).replace(" ", ""))
def test_rows_past_the_tree_hold_no_number(shape, dtype):
    import torch
    H, DL, prefix, sizes, block = shape
    m = make(DL + H + 1, H, DL, prefix, sizes, block, dtype)
    cache = torch.full_like(m["cache"], float("nan"))
    for b, n in enumerate(sizes):
        for r in range(int(m["prefix"][b]) + n):
            page, at = L.place(m["table"], b, r, cache.shape[1])
            cache[page, at] = m["cache"][page, at]
    check(m, run(m, cache=cache.to("cuda")))


@pytest.mark.parametrize("dtype", ["bfloat16", "float32"])
@pytest.mark.parametrize("H, sizes", [(16, [1, 1, 1]), (16, [60, 7, 33]), (128, [3, 1, 20])])
@pytest.mark.parametrize("way", ["up", "down", "both"])
def test_scores_that_climb_and_fall(way, H, sizes, dtype):
    """Scores that pass the running maximum by a little or by far in every tile, or fall away from it: every key's scaled
    score is steps of up to 12 (17 in powers of two) from the last tile's."""
    import torch
    m = make(5, H, 512, [900, 31, 500], sizes, 0, dtype)
    rng = np.random.default_rng(1)
    steps = rng.choice([0.5, 3.0, 11.0, 12.0], size=64)
    climb = np.repeat(np.cumsum(steps), 16)[:m["cache"].shape[1]]
    climb = {"up": climb, "down": climb[::-1].copy(), "both": np.minimum(climb, climb[::-1])}[way]
    climb -= climb.mean()
    # one dim of the queries is 8, the others small, so that this dim of a key sets its score
    q = m["q"] * 0.05
    q[..., 512] = 8.0
    m["cache"][:, :, 512] = torch.from_numpy(climb / (8.0 * m["scale"])).to(m["cache"].dtype)
    m.update(q=q, ql=q[..., :512], qr=q[..., 512:], layout="rows")
    check(m, run(m), label=way)


@pytest.mark.parametrize("dtype", ["bfloat16", "float32"])
@pytest.mark.parametrize("scale", [1e-44, 1e-30, 1e-3, 3.0])
@pytest.mark.parametrize("H", [4, 16])
def test_scales(H, scale, dtype):
    m = make(6, H, 256, [300, 2000], [4, 3], 16, dtype, qstd=0.3)
    check(m, run(m, scale=scale), scale=scale)


@pytest.mark.parametrize("dtype", ["bfloat16", "float32"])
def test_large_values(dtype):
    """Latent values of 2^60 with scores of usual size."""
    m = make(7, 16, 512, [500, 40], [20, 1], 0, dtype)
    big = 2.0 ** 60
    m["cache"][..., :512] *= big
    m["q"][..., :512] /= big
    m.update(ql=m["q"][..., :512], qr=m["q"][..., 512:], layout="rows")
    check(m, run(m))


@pytest.mark.parametrize("H, n", [(16, 1), (2, 9), (16, 12)])
@pytest.mark.parametrize("B", [65, 200])
def test_more_sequences_than_lanes(B, H, n):
    rng = np.random.default_rng(B + H)
    prefix = [int(p) for p in rng.choice([0, 1, 31, 32, 33, 100, 700], size=B)]
    sizes = [int(s) for s in rng.integers(0, n + 1, size=B)]
    sizes[64:] = [0 if b % 2 else n for b in range(64, B)]
    m = make(B, H, 256, prefix, sizes, 16, nmax=n)
    check(m, run(m))


@pytest.mark.parametrize("H, n", [(16, 1), (16, 30)])
def test_all_but_the_last_sequence_are_empty(H, n):
    m = make(3, H, 512, [50] * 129 + [3000], [0] * 129 + [n], 64)
    check(m, run(m))
    m = make(3, H, 512, [50] * 70, [0] * 70, 64, nmax=n)
    check(m, run(m))


@pytest.mark.parametrize("H, sizes", [(16, [1, 1]), (16, [30, 2]), (128, [5, 9])])
def test_a_loose_longest_prefix_changes_nothing_but_the_split(H, sizes):
    m = make(8, H, 512, [700, 3], sizes, 32)
    tight = run(m)
    loose = run(m, max_prefix=ltd.MAX_LENGTH)
    check(m, tight)
    check(m, loose)


@pytest.mark.parametrize("H, n", [(16, 1), (16, 20)])
def test_the_same_call_gives_the_same_bits(H, n):
    import torch
    m = make(9, H, 512, [900, 5, 4000], [n, n, 1], 16, nmax=n)
    first = run(m)
    for _ in range(3):
        assert torch.equal(run(m), first)


@pytest.mark.parametrize("dtype", ["bfloat16", "float32"])
@pytest.mark.parametrize("H, n", [(2, 3), (16, 9)])
def test_query_layouts(H, n, dtype):
    """Padded rows, heads first, heads in reverse storage and shared by all heads."""
    import torch
    m = make(10, H, 256, [33, 150], [n, 2], 0, dtype, nmax=n)
    base = run(m)
    B, N, D = 2, n, 256 + L.ROPE
    q = m["q"].to("cuda")
    out = torch.empty_like(base)

    def go(ql, qr):
        out.fill_(7.0)
        ltd.tree_verify_attn_latent(ql, qr, m["cache"].to("cuda"), L.to_dev(m["prefix"]), L.to_dev(m["par"]), L.to_dev(m["n"]),
                                    out, max_prefix=150, scale=m["scale"])
        torch.cuda.synchronize()
        return out

    wide = torch.zeros((B, N, H + 3, D + 24), dtype=q.dtype, device="cuda")
    wide[:, :, 2:H + 2, 8:D + 8] = q
    assert torch.equal(go(wide[:, :, 2:H + 2, 8:264], wide[:, :, 2:H + 2, 264:D + 8]), base)
    first = q.permute(2, 0, 1, 3).contiguous().permute(1, 2, 0, 3)
    assert torch.equal(go(first[..., :256], first[..., 256:].contiguous()), base)
    shared = q[:, :, :1].expand(B, N, H, D)
    same = go(shared[..., :256], shared[..., 256:]).clone()
    assert torch.equal(same, go(shared[..., :256].contiguous(), shared[..., 256:].contiguous()))


def test_another_stream():
    import torch
    m = make(11, 16, 512, [2000, 77], [33, 5], 64)
    base = run(m)
    s = torch.cuda.Stream()
    ql, qr = parts(m)
    cache, table = m["cache"].to("cuda"), L.to_dev(m["table"])
    args = (L.to_dev(m["prefix"]), L.to_dev(m["par"]), L.to_dev(m["n"]))
    out = torch.full_like(base, 7.0)
    torch.cuda.synchronize()
    with torch.cuda.stream(s):
        for _ in range(3):
            ltd.tree_verify_attn_latent(ql, qr, cache, *args, out, max_prefix=2000, scale=m["scale"], block_table=table,
                                        num_blocks=cache.shape[0])
    s.synchronize()
    assert torch.equal(out, base)


@pytest.mark.parametrize("H, sizes", [(16, [1, 1]), (16, [6, 3])])
@pytest.mark.parametrize("dtype", ["bfloat16", "float32"])
def test_validation(dtype, H, sizes):
    import torch
    n = max(sizes)

    def status(**change):
        m = make(12, H, 512, [40, 90], sizes, 16, dtype, nmax=n)
        m["par"] = np.where(m["par"] == -7, -1, m["par"])
        top = change.pop("max_prefix", 90)
        for k, f in change.items():
            m[k] = m[k].copy()
            f(m[k])
        st = torch.full((1,), -1, dtype=torch.int32, device="cuda")
        out = run(m, max_prefix=top, validate=True, status=st)
        if int(st) != ltd.STATUS_OK:
            assert bool((out == 7.0).all()), "written in spite of the status"
        else:
            check(m, out)
        return int(st)

    def put(i, v):
        return lambda a: a.__setitem__(i, v)

    assert status() == ltd.STATUS_OK
    assert status(n=put(0, 0)) == ltd.STATUS_BAD_NNODES
    assert status(n=put(1, n + 1)) == ltd.STATUS_BAD_NNODES
    assert status(par=put((0, 0), 0)) == ltd.STATUS_BAD_PARENT
    if n > 1:
        assert status(par=put((0, 2), 2)) == ltd.STATUS_BAD_PARENT
        assert status(par=put((1, 1), -1)) == ltd.STATUS_BAD_PARENT
    assert status(prefix=put(0, -1)) == ltd.STATUS_BAD_PREFIX
    assert status(max_prefix=89) == ltd.STATUS_BAD_PREFIX
    assert status(prefix=put(1, 16 * 6 - sizes[1] + 1), max_prefix=200) == ltd.STATUS_BAD_PREFIX
    assert status(table=put((0, 1), -1)) == ltd.STATUS_BAD_BLOCK
    assert status(table=put((1, 2), 10 ** 6)) == ltd.STATUS_BAD_BLOCK


# ---- caches that 32 bits do not reach (2^31 elements, 2^32 bytes): only the rows of the case are filled

def large(B, R, D, t):
    import torch
    return torch.empty((B, R, D), dtype=getattr(torch, t), device="cuda")


@pytest.mark.parametrize("H, sizes", [(16, [1, 1, 1]), (16, [8, 20, 3])])
@pytest.mark.parametrize("dtype", ["bfloat16", "float32"])
def test_contiguous_cache_past_32_bits(dtype, H, sizes):
    m = make(13, H, 512, [300, 10, 77], sizes, 0, dtype)
    R = 2_000_003 if dtype == "bfloat16" else 1_000_003
    cache = large(3, R, 576, dtype)
    cache[:, :m["cache"].shape[1]] = m["cache"].to("cuda")
    assert cache[2].data_ptr() - cache.data_ptr() > 2 ** 32
    check(m, run(m, cache=cache))


@pytest.mark.parametrize("block", [16, 1, 100])
@pytest.mark.parametrize("H, sizes", [(16, [1, 1]), (16, [8, 20])])
@pytest.mark.parametrize("dtype", ["bfloat16", "float32"])
def test_pages_past_32_bits(dtype, H, sizes, block):
    m = make(14, H, 512, [300, 77], sizes, block, dtype)
    pages = 5 * 10 ** 9 // (576 * block * m["cache"].element_size())
    cache = large(pages, block, 576, dtype)
    used = m["cache"].shape[0]
    cache[pages - used:] = m["cache"].to("cuda")
    table = np.where(m["table"] < 0, m["table"], m["table"] + pages - used).astype(np.int32)
    assert (pages - used) * block * 576 > 2 ** 31 or dtype == "float32"
    ql, qr = parts(m)
    import torch
    out = torch.full(ql.shape, 7.0, dtype=ql.dtype, device="cuda")
    ltd.tree_verify_attn_latent(ql, qr, cache, L.to_dev(m["prefix"]), L.to_dev(m["par"]), L.to_dev(m["n"]), out,
                                max_prefix=300, scale=m["scale"], block_table=L.to_dev(table), num_blocks=pages)
    torch.cuda.synchronize()
    check(m, out)


@pytest.mark.parametrize("H", [16, 24])
def test_a_long_prefix(H):
    """One sequence of 300000 rows on two pages that its table repeats."""
    import torch
    rng = np.random.default_rng(15)
    P, n, R, DL = 300_000, 1, 4096, 512
    cache = torch.from_numpy(rng.normal(size=(3, R, DL + L.ROPE))).to(torch.bfloat16)
    table = np.array([[0, 1] * 37], np.int32)
    table[0, P // R] = 2
    q = torch.from_numpy(rng.normal(size=(1, n, H, DL + L.ROPE)) * 1.5).to(torch.bfloat16)
    m = dict(cache=cache, table=table, par=np.array([[-1]], np.int32), q=q, ql=q[..., :DL], qr=q[..., DL:], layout="rows",
             prefix=np.array([P], np.int32), n=np.array([1], np.int32), scale=192 ** -0.5, DL=DL)
    check(m, run(m))


@pytest.mark.parametrize("H, sizes", [(16, [1, 1]), (16, [20, 1])])
@pytest.mark.parametrize("DL", [256, 512])
def test_dims_of_different_sizes(DL, H, sizes):
    """Latent dims from 2^-12 to 2^12 in turn, rows of sequences from 2^-60 to 2^60: split rows keep every dim's bits."""
    import torch
    m = make(16, H, DL, [3000, 700], sizes, 0)
    by_dim = 2.0 ** torch.from_numpy(np.random.default_rng(2).integers(-12, 13, DL)).double()
    by_seq = torch.tensor([2.0 ** 60, 2.0 ** -60]).double()
    lat = m["cache"][..., :DL].double() * by_dim
    m["cache"][..., :DL] = (lat * by_seq[:, None, None]).bfloat16()
    m["q"][..., :DL] = (m["q"][..., :DL].double() / by_dim / by_seq[:, None, None, None]).bfloat16()
    m.update(ql=m["q"][..., :DL], qr=m["q"][..., DL:], layout="rows")
    check(m, run(m))


@pytest.mark.parametrize("H, n", [(16, 1), (128, 1), (16, 12)])
@pytest.mark.parametrize("others", [1, 17, 40])
def test_one_long_sequence_among_short_ones(others, H, n):
    """Rows that many workgroups have pieces of, beside rows of one: up to a hundred pieces are joined."""
    prefix = [40, 12000] + [int(p) for p in np.random.default_rng(others).choice([0, 3, 31, 64, 90], size=others)]
    m = make(others + H, H, 512, prefix, [n] * len(prefix), 16)
    check(m, run(m), label=f"{H} heads, {n} nodes, {others} others")


@pytest.mark.parametrize("DL", [256, 512])
@pytest.mark.parametrize("H", [16, 20])
def test_prefixes_around_the_shortest_share(DL, H):
    """Shares that lie within a unit's own cost, end with it, or have one tile."""
    for tiles in (1, 2, 3, 4, 5, 8, 9, 12, 13, 16, 17, 20):
        for prefix in ([32 * tiles - 1], [32 * tiles], [32 * tiles - 1, 32 * tiles + 100, 5]):
            m = make(tiles + H, H, DL, prefix, [1] * len(prefix), 0)
            check(m, run(m), label=f"{H} heads over {prefix}")
