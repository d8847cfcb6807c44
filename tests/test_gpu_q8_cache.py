"""The 8-bit KV cache's writes on the GPU against their definitions: every code and scale byte of every row in use,
and every byte that has to stay."""
import numpy as np
import pytest

import paper_2603_01639_amd as ltd
import q8_util as Q

pytestmark = pytest.mark.gpu


def _live(c, which, b_rows):
    """Codes and scale bytes of the logical rows in use, in order."""
    out = []
    for b, rows in b_rows:
        for r in range(rows):
            p, w = Q.place(c["table"], b, r, c["R"])
            out.append((c[which][p, :, w].copy(), c[which + "s"][p, :, w // c["sr"]].copy()))
    return out


def _same(got, want, label):
    for i, ((gc, ge), (wc, we)) in enumerate(zip(got, want)):
        np.testing.assert_array_equal(ge, we, err_msg=f"{label}: scale bytes of live row {i}")
        nan = np.isnan(Q.VALUES[wc])
        assert np.array_equal(np.isnan(Q.VALUES[gc]), nan), f"{label}: NaN codes of live row {i}"
        np.testing.assert_array_equal(gc[~nan], wc[~nan], err_msg=f"{label}: codes of live row {i}")


def _rows(rng, B, N, H, d, dtype, wild=1.0):
    """New rows as a float64 array of values that dtype holds, and the tensor."""
    import torch
    x = rng.normal(size=(B, N, H, d)) * np.exp(wild * rng.normal(size=(B, N, H, 1)))
    t = torch.from_numpy(x).to(dtype)
    return t.double().numpy(), t.to("cuda")


def _untouched(c, before, which, written):
    """Pages outside `written` keep every byte."""
    keep = [p for p in range(c["pages"]) if p not in written]
    np.testing.assert_array_equal(c[which][keep], before[which][keep])
    np.testing.assert_array_equal(c[which + "s"][keep], before[which + "s"][keep])


@pytest.mark.parametrize("dtype", ["bfloat16", "float32"])
@pytest.mark.parametrize("d, sr, block", [(128, 16, 16), (128, 16, 0), (128, 32, 64), (128, 64, 0), (128, 128, 128),
                                          (64, 16, 48), (64, 32, 0), (64, 64, 64), (64, 128, 0)])
def test_append(dtype, d, sr, block):
    import torch
    rng = np.random.default_rng(sr * 1000 + d + block)
    prefix = [0, 1, sr - 1, sr, sr + 3, 5 * sr + 7, 40, 0]
    n = [1, 2 * sr + 3, 1, sr, 3, 0, 2 * sr, 3 * sr]
    B, H, N = len(prefix), 3, max(n)
    c = Q.cache(rng, B, H, d, sr, [p + m for p, m in zip(prefix, n)], block)
    x, xt = {}, {}
    for w in "kv":
        x[w], xt[w] = _rows(rng, B, N, H, d, getattr(torch, dtype))
    dev = Q.dev_cache(c)
    args = [Q.to_dev(np.array(a, np.int32)) for a in (prefix, n)]
    ltd.kv_append_q8(xt["k"], xt["v"], dev["k"], dev["v"], dev["ks"], dev["vs"], *args, scale_rows=sr,
                     block_table=dev["table"], num_blocks=c["pages"])
    torch.cuda.synchronize()
    for w in "kv":
        got = dict(c, **{w: dev[w].cpu().numpy(), w + "s": dev[w + "s"].cpu().numpy()})
        want = dict(c, **{w: c[w].copy(), w + "s": c[w + "s"].copy()})
        Q.append(want[w], want[w + "s"], x[w], c["table"], prefix, n, sr)
        live = [(b, p + m) for b, (p, m) in enumerate(zip(prefix, n))]
        _same(_live(got, w, live), _live(want, w, live), f"{w} sr={sr} d={d}")
        written = {Q.place(c["table"], b, r, c["R"])[0] for b, (p, m) in enumerate(zip(prefix, n))
                   for r in range(p, p + m)}
        _untouched(got, c, w, written)


def test_append_of_extreme_values():
    """Zeros, the smallest and largest magnitudes, values on the format's border, infinities and NaN: each in a block
    of its own."""
    import torch
    sr, d, H = 16, 64, 1
    rows = [0.0, 1e-38, 2.0 ** -101, 447.9, 448.0, 448.1, 464.0, 480.0, 2.0 ** 95, 2.0 ** 96, 3.0e38, np.inf, np.nan,
            1.75, 1.7500001, -1e-45, 2.0 ** 86 * 448]
    B = len(rows)
    x = np.zeros((B, sr, H, d), np.float32)
    rng = np.random.default_rng(5)
    for b, r in enumerate(rows):
        top = abs(r) if np.isfinite(r) else 3.0
        x[b] = (rng.uniform(-1, 1, (sr, H, d)) * top).astype(np.float32)
        x[b, 3, 0, 5] = r
    c = Q.cache(rng, B, H, d, sr, [sr] * B)
    dev = Q.dev_cache(c)
    args = [Q.to_dev(np.array(a, np.int32)) for a in ([0] * B, [sr] * B)]
    xt = Q.to_dev(x)
    ltd.kv_append_q8(xt, xt, dev["k"], dev["v"], dev["ks"], dev["vs"], *args, scale_rows=sr)
    torch.cuda.synchronize()
    got = dict(c, k=dev["k"].cpu().numpy(), ks=dev["ks"].cpu().numpy())
    want = dict(c, k=c["k"].copy(), ks=c["ks"].copy())
    Q.append(want["k"], want["ks"], x, None, [0] * B, [sr] * B, sr)
    live = [(b, sr) for b in range(B)]
    _same(_live(got, "k", live), _live(want, "k", live), "extremes")
    assert got["ks"].min() >= Q.E_MIN and got["ks"].max() <= Q.E_MAX


@pytest.mark.parametrize("dtype", ["bfloat16", "float32"])
def test_append_of_strided_views(dtype):
    """K and V as slices of a fused projection's output."""
    import torch
    rng = np.random.default_rng(8)
    B, N, H, d, sr, Hq = 2, 21, 2, 128, 32, 4
    t = torch.from_numpy(rng.normal(size=(B, N, (Hq + 2 * H) * d))).to(getattr(torch, dtype)).to("cuda")
    kn = t[:, :, Hq * d:(Hq + H) * d].view(B, N, H, d)
    vn = t[:, :, (Hq + H) * d:].view(B, N, H, d)
    c = Q.cache(rng, B, H, d, sr, [70, 70])
    args = [Q.to_dev(np.array(a, np.int32)) for a in ([40, 7], [21, 20])]
    outs = []
    for k, v in ((kn, vn), (kn.contiguous(), vn.contiguous())):
        dev = Q.dev_cache(c)
        ltd.kv_append_q8(k, v, dev["k"], dev["v"], dev["ks"], dev["vs"], *args, scale_rows=sr)
        outs.append([dev[x].cpu().numpy() for x in ("k", "v", "ks", "vs")])
    for a, b in zip(*outs):
        np.testing.assert_array_equal(a, b)


def test_appending_twice_grows_the_scale_of_a_shared_block():
    """Two appends to one block: a small row, then one a thousand times larger, then a smaller one again."""
    import torch
    rng = np.random.default_rng(11)
    d, sr, H = 128, 64, 2
    c = Q.cache(rng, 1, H, d, sr, [64])
    dev = Q.dev_cache(c)
    want = dict(c, k=c["k"].copy(), ks=c["ks"].copy())
    for P, scale in ((0, 1e-3), (3, 1.0), (7, 900.0), (11, 0.1)):
        x = (rng.normal(size=(1, 4, H, d)) * scale).astype(np.float32)
        xt = Q.to_dev(x)
        args = [Q.to_dev(np.array([a], np.int32)) for a in (P, 4)]
        ltd.kv_append_q8(xt, xt, dev["k"], dev["v"], dev["ks"], dev["vs"], *args, scale_rows=sr)
        Q.append(want["k"], want["ks"], x, None, [P], [4], sr)
    torch.cuda.synchronize()
    got = dict(c, k=dev["k"].cpu().numpy(), ks=dev["ks"].cpu().numpy())
    _same(_live(got, "k", [(0, 15)]), _live(want, "k", [(0, 15)]), "twice")


@pytest.mark.parametrize("d, sr, block, layers", [(128, 16, 16, 1), (128, 16, 0, 3), (128, 32, 96, 2), (128, 64, 0, 1),
                                                  (128, 128, 128, 2), (64, 16, 0, 1), (64, 32, 32, 2), (64, 128, 0, 1)])
@pytest.mark.parametrize("spread", [0, 6])
def test_compact(d, sr, block, layers, spread):
    import torch
    rng = np.random.default_rng(sr + d + block + layers + spread)
    prefix = [0, 1, sr - 2, sr, 3 * sr + 5, 17, 2 * sr + 1]
    paths = [[0], [0, 1, 2], [0, 3, 5, 6, 30], list(range(40)), [0, 1, 3, 6], [0] + list(range(5, 5 + min(2 * sr, 240))), [0, 200]]
    B, H, N = len(prefix), 2, 256
    n = [len(p) for p in paths]
    path = np.zeros((B, N), np.int32)
    for b, p in enumerate(paths):
        path[b, :len(p)] = p
    c = Q.cache(rng, B, H, d, sr, [P + max(p) + 1 for P, p in zip(prefix, paths)], block, layers=layers, spread=spread)
    dev = Q.dev_cache(c)
    new = torch.zeros(B, dtype=torch.int32, device="cuda")
    args = [Q.to_dev(np.array(a, np.int32)) for a in (prefix, path, n)]
    ltd.kv_compact_q8(dev["k"], dev["v"], dev["ks"], dev["vs"], args[0], new, args[1], args[2], scale_rows=sr,
                      block_table=dev["table"], num_blocks=c["pages"], num_layers=layers)
    torch.cuda.synchronize()
    np.testing.assert_array_equal(new.cpu().numpy(), np.array(prefix) + n)
    live = [(b, p + m) for b, (p, m) in enumerate(zip(prefix, n))]
    for w in "kv":
        gk, gs = dev[w].cpu().numpy(), dev[w + "s"].cpu().numpy()
        for x in range(layers):
            got = dict(c, **{w: gk[x], w + "s": gs[x]})
            want = dict(c, **{w: c[w][x].copy(), w + "s": c[w + "s"][x].copy()})
            Q.compact(want[w], want[w + "s"], c["table"], prefix, path, n, sr)
            _same(_live(got, w, live), _live(want, w, live), f"{w} layer {x} sr={sr} d={d}")
            written = {Q.place(c["table"], b, r, c["R"])[0] for b, (p, m) in enumerate(zip(prefix, n))
                       for r in range(p, p + m)}
            _untouched(got, dict(c, **{w: c[w][x], w + "s": c[w + "s"][x]}), w, written)


def test_compaction_leaves_gaps_between_layers_alone():
    """Layers inside a larger buffer: strides beyond a layer's size."""
    import torch
    rng = np.random.default_rng(21)
    H, d, sr, L = 2, 64, 16, 3
    c = Q.cache(rng, 1, H, d, sr, [60], layers=L)
    size, ssize = c["k"][0].size, c["ks"][0].size
    gap, sgap = 4096, 64
    buf = {w: torch.full(((size + gap) * L,), 0x55, dtype=torch.uint8, device="cuda") for w in "kv"}
    sbuf = {w: torch.full(((ssize + sgap) * L,), 0x66, dtype=torch.uint8, device="cuda") for w in "kv"}
    for w in "kv":
        for x in range(L):
            buf[w][x * (size + gap):][:size] = Q.to_dev(c[w][x].ravel())
            sbuf[w][x * (ssize + sgap):][:ssize] = Q.to_dev(c[w + "s"][x].ravel())
    path = np.array([[0, 2, 9, 20, 21]], np.int32)
    args = [Q.to_dev(np.array(a, np.int32)) for a in ([30], path, [5])]
    new = torch.zeros(1, dtype=torch.int32, device="cuda")
    view = [buf[w][:size].view(c[w][0].shape) for w in "kv"] + [sbuf[w][:ssize].view(c[w + "s"][0].shape) for w in "kv"]
    ltd.kv_compact_q8(*view, args[0], new, args[1], args[2], scale_rows=sr, num_layers=L, layer_stride_elems=size + gap,
                      scale_stride_elems=ssize + sgap)
    torch.cuda.synchronize()
    for w in "kv":
        got, gots = buf[w].cpu().numpy().reshape(L, -1), sbuf[w].cpu().numpy().reshape(L, -1)
        assert (got[:, size:] == 0x55).all() and (gots[:, ssize:] == 0x66).all()
        for x in range(L):
            want, ws = c[w][x].copy(), c[w + "s"][x].copy()
            Q.compact(want, ws, None, [30], path, [5], sr)
            one = dict(c, **{w: got[x, :size].reshape(want.shape), w + "s": gots[x, :ssize].reshape(ws.shape)})
            _same(_live(one, w, [(0, 35)]), _live(dict(c, **{w: want, w + "s": ws}), w, [(0, 35)]), f"{w} {x}")


@pytest.mark.parametrize("what, code", [("n", ltd.STATUS_BAD_NNODES), ("prefix", ltd.STATUS_BAD_PREFIX),
                                        ("block", ltd.STATUS_BAD_BLOCK), ("none", 0)])
def test_append_validation_writes_nothing_on_bad_data(what, code):
    import torch
    rng = np.random.default_rng(3)
    c = Q.cache(rng, 2, 2, 64, 16, [40, 40], 16)
    prefix, n = [20, 30], [10, 10]
    if what == "n":
        n[1] = 11
    elif what == "prefix":
        prefix[1] = 48 - 9
    elif what == "block":
        c["table"][1, 2] = c["pages"]
    dev = Q.dev_cache(c)
    x = torch.randn((2, 10, 2, 64), device="cuda", dtype=torch.bfloat16)
    status = torch.full((1,), 77, dtype=torch.int32, device="cuda")
    args = [Q.to_dev(np.array(a, np.int32)) for a in (prefix, n)]
    ltd.kv_append_q8(x, x, dev["k"], dev["v"], dev["ks"], dev["vs"], *args, scale_rows=16, block_table=dev["table"],
                     num_blocks=c["pages"], validate=True, status=status)
    assert int(status.cpu()[0]) == code
    changed = any(not np.array_equal(dev[k].cpu().numpy(), c[k]) for k in ("k", "v", "ks", "vs"))
    assert changed == (code == 0)


def test_pages_past_4_gib():
    """Codes whose offsets pass 2^32: append, attention and compaction on pages at the end of a large cache give what
    they give on a small one."""
    import torch
    rng = np.random.default_rng(17)
    H, d, sr, block, far = 8, 128, 16, 16, 280000  # 280000 pages of 16 KiB: 4.6 GB
    prefix, n = [40, 7], [9, 5]
    c = Q.cache(rng, 2, H, d, sr, [64, 64], block)
    for k in "kv":
        c[k] &= 0xBF  # (moderate values)
    x = torch.from_numpy(rng.normal(size=(2, 9, H, d))).to(torch.bfloat16).to("cuda")
    q = torch.from_numpy(rng.normal(size=(2, 9, 16, d))).to(torch.bfloat16).to("cuda")
    par = Q.to_dev(Q.trees(rng, n))
    path = np.zeros((2, 9), np.int32)
    path[0, :3], path[1, :2] = [0, 4, 8], [0, 3]
    ints = [Q.to_dev(np.array(a, np.int32)) for a in (prefix, n, path, [3, 2])]
    outs = []
    for shift in (0, far):
        dev = Q.dev_cache(c)
        table, pages = dev["table"], c["pages"]
        if shift:
            big = {k: torch.empty((far + pages,) + tuple(dev[k].shape[1:]), dtype=torch.uint8, device="cuda")
                   for k in ("k", "v", "ks", "vs")}
            for k, t in big.items():
                t[far:] = dev[k]
            dev, table, pages = big, table + far, far + pages
        cache = (dev["k"], dev["v"], dev["ks"], dev["vs"])
        paged = dict(scale_rows=sr, block_table=table, num_blocks=pages)
        ltd.kv_append_q8(x, x, *cache, ints[0], ints[1], **paged)
        out, new = torch.zeros_like(q), torch.zeros(2, dtype=torch.int32, device="cuda")
        ltd.tree_verify_attn_q8(q, *cache, ints[0], par, ints[1], out, max_prefix=40, **paged)
        short = torch.zeros_like(q[:, :1])  # (one node: the kernel of short units)
        ltd.tree_verify_attn_q8(q[:, :1].contiguous(), *cache, ints[0], par[:, :1].contiguous(),
                                torch.ones_like(ints[1]), short, max_prefix=40, **paged)
        f32 = torch.zeros_like(q, dtype=torch.float32)
        ltd.tree_verify_attn_q8(q.float(), *cache, ints[0], par, ints[1], f32, max_prefix=40, **paged)
        ltd.kv_compact_q8(*cache, ints[0], new, ints[2], ints[3], **paged)
        torch.cuda.synchronize()
        outs.append([out.float().cpu(), short.float().cpu(), f32.cpu(), new.cpu()] + [t[shift:].cpu() for t in cache])
        del dev, cache
    for a, b in zip(*outs):
        assert torch.equal(a, b)
