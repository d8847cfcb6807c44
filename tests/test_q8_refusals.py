"""What the 8-bit cache's calls and the rules' calls refuse, on the CPU: scalars and pointers in the C ABI, and types,
shapes and layouts in the binding (nothing is launched)."""
import pytest

import paper_2603_01639_amd as ltd
import q8_util as Q

X = 4096  # a pointer that no refused call follows
FN = ltd.lib


def append(**kw):
    a = dict(k=X, v=X, stride=512, kc=X, vc=X, ks=X, vs=X, table=None, prefix=X, n=X, B=1, N=4, H=4, d=128, rows=64, mb=0,
             nb=0, sr=16, dtype=1, validate=0, status=None)
    a.update(kw)
    return FN().ltd_kv_append_q8(*a.values(), None)


def attn(**kw):
    a = dict(q=X, kc=X, vc=X, ks=X, vs=X, table=None, prefix=X, par=X, n=X, out=X, B=1, N=4, Hq=8, H=4, d=128, mp=16, rows=64,
             mb=0, nb=0, sr=16, scale=0.1, dtype=0, ws=None, wsb=0, validate=0, status=None)
    a.update(kw)
    return FN().ltd_tree_verify_attn_q8(*a.values(), None)


def compact(**kw):
    a = dict(kc=X, vc=X, ks=X, vs=X, table=None, prefix=X, new=X + 64, path=X, n=X, B=1, N=4, H=4, d=128, rows=64, mb=0, nb=0,
             sr=16, layers=1, ls=0, ss=0, validate=0, status=None)
    a.update(kw)
    return FN().ltd_kv_compact_q8(*a.values(), None)


def process(**kw):
    a = dict(lg=X, tok=X, par=X, n=X, counts=None, pen=None, bt=None, bv=None, bn=None, mask=None, B=1, N=4, V=100, mb=0,
             out=X, validate=0, status=None)
    a.update(kw)
    return FN().ltd_tree_process_logits(*a.values(), None)


def accept(**kw):
    a = dict(lg=X, tok=X, par=X, n=X, counts=None, pen=None, bt=None, bv=None, bn=None, mask=None, B=1, N=4, V=100, mb=0,
             pred=X, acc=X, toks=X, nacc=X, ws=X, wsb=1 << 20, validate=0, status=None)
    a.update(kw)
    return FN().ltd_tree_accept_processed(*a.values(), None)


BAD, NO, WS = ltd.LTD_EINVAL, ltd.LTD_EUNSUPPORTED, ltd.LTD_EWORKSPACE


@pytest.mark.parametrize("kw, code", [
    (dict(B=-1), BAD), (dict(N=0), BAD), (dict(H=0), BAD), (dict(rows=0), BAD), (dict(d=96), NO), (dict(sr=8), NO),
    (dict(sr=48), NO), (dict(dtype=2), NO), (dict(table=X, mb=1, nb=1, rows=40), NO), (dict(table=X, mb=0, nb=1), BAD),
    (dict(stride=511), BAD), (dict(stride=516), BAD), (dict(k=X + 2), BAD), (dict(kc=X + 8), BAD), (dict(vs=None), BAD),
    (dict(n=None), BAD), (dict(validate=1), BAD), (dict(B=0, k=None), 0)])
def test_append(kw, code):
    assert append(**kw) == code


@pytest.mark.parametrize("kw, code", [
    (dict(B=-1), BAD), (dict(N=257), BAD), (dict(Hq=6), BAD), (dict(mp=-1), BAD), (dict(rows=0), BAD), (dict(scale=0.0), BAD),
    (dict(scale=float("nan")), BAD), (dict(d=96), NO), (dict(sr=256), NO), (dict(dtype=7), NO),
    (dict(table=X, mb=1, nb=1, rows=24), NO), (dict(table=X, mb=1, nb=0), BAD), (dict(ks=None), BAD), (dict(q=X + 4), BAD),
    (dict(out=X + 2), BAD), (dict(validate=1), BAD), (dict(dtype=1, N=60, mp=4096, rows=8192), WS),
    (dict(dtype=1, N=60, mp=4096, rows=8192, ws=X, wsb=64), WS), (dict(dtype=1, N=60, mp=4096, rows=8192, ws=X + 8, wsb=1 << 30), WS),
    (dict(B=0, q=None), 0)])
def test_attention(kw, code):
    assert attn(**kw) == code


@pytest.mark.parametrize("kw, code", [
    (dict(B=-1), BAD), (dict(N=257), BAD), (dict(layers=0), BAD), (dict(d=32), NO), (dict(sr=0), NO), (dict(new=X), BAD),
    (dict(layers=2), BAD), (dict(layers=2, ls=4096), BAD), (dict(layers=2, ls=4104, ss=16), BAD), (dict(ss=-1), BAD),
    (dict(kc=None), BAD), (dict(vc=X + 4), BAD), (dict(validate=1), BAD), (dict(B=0, kc=None), 0)])
def test_compact(kw, code):
    assert compact(**kw) == code


@pytest.mark.parametrize("call", [process, accept])
@pytest.mark.parametrize("kw, code", [
    (dict(B=-1), BAD), (dict(N=0), BAD), (dict(N=257), BAD), (dict(V=0), BAD), (dict(mb=-1), BAD),
    (dict(mb=ltd.MAX_BIAS + 1), BAD), (dict(mb=4), BAD), (dict(mb=4, bt=X, bv=X), BAD), (dict(lg=None), BAD),
    (dict(par=None), BAD), (dict(validate=1), BAD), (dict(B=0, lg=None), 0)])
def test_rules(call, kw, code):
    assert call(**kw) == code


def test_rules_outputs_and_workspace():
    assert process(out=None) == BAD
    assert accept(pred=None) == BAD
    assert accept(ws=None) == WS
    assert accept(wsb=4 * 8 - 1) == WS


@pytest.mark.parametrize("args, code", [((X, X, -1, 4, 100, 0, 0, X), BAD), ((X, X, 1, -1, 100, 0, 0, X), BAD),
                                        ((X, X, 1, 4, 0, 0, 0, X), BAD), ((X, X, 1, 4, 100, 0, 0, None), BAD),
                                        ((None, X, 1, 4, 100, 0, 0, X), BAD), ((None, None, 0, 4, 100, 0, 0, None), 0)])
def test_token_counts(args, code):
    assert FN().ltd_token_counts(*args, None) == code


def test_workspace_query():
    size = ltd.attn_q8_workspace_size
    assert size(1, 60, 32, 8, 96, 2048, ltd.DTYPE_BF16) == 0
    assert size(1, 300, 32, 8, 128, 2048, ltd.DTYPE_BF16) == 0
    assert size(1, 16, 8, 8, 64, 128, ltd.DTYPE_F32) == 0
    assert isinstance(size(1, 60, 32, 8, 128, 2048, ltd.DTYPE_BF16), int)


# ---- the binding's checks, with CPU tensors

def _cache(torch, B=2, H=2, rows=32, d=64, sr=16):
    z = lambda *s, t=torch.uint8: torch.zeros(s, dtype=t)  # noqa: E731
    return dict(k=z(B, H, rows, d), v=z(B, H, rows, d), ks=z(B, H, rows // sr), vs=z(B, H, rows // sr))


def _append(torch, c=None, x=None, n=None, B=2, **kw):
    c = c or _cache(torch)
    x = torch.zeros((B, 4, 2, 64), dtype=torch.bfloat16) if x is None else x
    i = torch.zeros(B, dtype=torch.int32)
    kw.setdefault("scale_rows", 16)
    ltd.kv_append_q8(x, x, c["k"], c["v"], c["ks"], c["vs"], i, i if n is None else n, **kw)


def test_binding_append():
    import torch
    with pytest.raises(ValueError, match="needs tensors on a GPU"):
        _append(torch)
    with pytest.raises(ValueError, match="scale_rows"):
        _append(torch, scale_rows=24)
    with pytest.raises(ValueError, match="k_scale has shape"):
        _append(torch, scale_rows=32)
    with pytest.raises(TypeError, match="k_cache has type"):
        _append(torch, dict(_cache(torch), k=torch.zeros((2, 2, 32, 64), dtype=torch.int32)))
    with pytest.raises(TypeError, match="unsupported dtype"):
        _append(torch, x=torch.zeros((2, 4, 2, 64), dtype=torch.float16))
    with pytest.raises(ValueError, match="are not both"):
        _append(torch, x=torch.zeros((2, 4, 3, 64), dtype=torch.bfloat16))
    with pytest.raises(ValueError, match="not contiguous"):
        _append(torch, x=torch.zeros((2, 4, 64, 2), dtype=torch.bfloat16).transpose(2, 3))
    with pytest.raises(ValueError, match="evenly spaced"):
        _append(torch, x=torch.zeros((2, 8, 2, 64), dtype=torch.bfloat16)[:, :4])
    with pytest.raises(TypeError, match="n_rows"):
        _append(torch, n=torch.zeros(2, dtype=torch.int64))
    with pytest.raises(ValueError, match="holds 2 sequences"):
        _append(torch, B=3)
    with pytest.raises(ValueError, match="num_blocks"):
        _append(torch, block_table=torch.zeros((2, 2), dtype=torch.int32), num_blocks=3)
    with pytest.raises(ValueError, match="rows for 2 sequences"):
        _append(torch, block_table=torch.zeros((1, 2), dtype=torch.int32), num_blocks=2)


def test_binding_attention_and_compaction():
    import torch
    c = _cache(torch)
    i = torch.zeros(2, dtype=torch.int32)
    q = torch.zeros((2, 4, 4, 64), dtype=torch.bfloat16)
    par = torch.zeros((2, 4), dtype=torch.int32)
    run = lambda q=q, out=q, par=par, **kw: ltd.tree_verify_attn_q8(  # noqa: E731
        q, c["k"], c["v"], c["ks"], c["vs"], i, par, i, out, max_prefix=8, scale_rows=16, **kw)
    with pytest.raises(ValueError, match="on a GPU"):
        run()
    with pytest.raises(TypeError, match="out has type"):
        run(out=q.float())
    with pytest.raises(ValueError, match="out has shape"):
        run(out=q[:, :3])
    with pytest.raises(ValueError, match="q has shape"):
        run(q=torch.zeros((2, 4, 4, 128), dtype=torch.bfloat16))
    with pytest.raises(ValueError, match="parents has shape"):
        run(par=par[:, :2])
    move = lambda c=c, i=i, path=par, **kw: ltd.kv_compact_q8(c["k"], c["v"], c["ks"], c["vs"], i, i.clone(), path, i,  # noqa: E731
                                                              scale_rows=16, **kw)
    with pytest.raises(ValueError, match="on a GPU"):
        move()
    with pytest.raises(ValueError, match="dimensions"):
        move(dict(c, k=c["k"][0]))
    with pytest.raises(ValueError, match="num_layers"):
        move({k: v[None].clone() for k, v in c.items()}, num_layers=2)


def test_binding_rules():
    import torch
    lg = torch.zeros((2, 3, 100))
    i, t = torch.ones(2, dtype=torch.int32), torch.zeros((2, 3), dtype=torch.int32)
    run = lambda lg=lg, out=lg, **kw: ltd.tree_process_logits(lg, t, t, i, out, **kw)  # noqa: E731
    with pytest.raises(ValueError, match="on a GPU"):
        run()
    with pytest.raises(TypeError, match="logits has type"):
        run(lg=lg.bfloat16())
    with pytest.raises(ValueError, match="mask has shape"):
        run(mask=torch.zeros((2, 3, 3), dtype=torch.int32))
    with pytest.raises(ValueError, match="penalties has shape"):
        run(penalties=torch.ones(3))
    with pytest.raises(ValueError, match="needs bias_values"):
        run(bias_tokens=t)
    with pytest.raises(ValueError, match="need bias_tokens"):
        run(n_bias=i)
    with pytest.raises(TypeError, match="counts has type"):
        run(counts=torch.zeros((2, 100), dtype=torch.int64))
    with pytest.raises(ValueError, match="out has shape"):
        run(out=lg[:, :2])
    with pytest.raises(ValueError, match="pred has shape"):
        ltd.tree_accept_processed(lg, t, t, i, i, t, t, i)


def test_lengths_past_the_limit():
    """Rows, tokens and vocabularies whose last index, rounded up to a block or a chunk, would pass 32 bits."""
    top = ltd.MAX_LENGTH
    assert append(N=top + 1) == NO and append(N=2**31 - 1) == NO
    assert attn(mp=top + 1, rows=2**31 - 1) == NO and attn(mp=2**31 - 1, rows=2**31 - 1) == NO
    assert ltd.attn_q8_workspace_size(1, 60, 32, 8, 128, 2**31 - 1, ltd.DTYPE_BF16) == 0
    for call in (process, accept):
        assert call(V=top + 1) == NO and call(V=2**31 - 1) == NO
    counts = FN().ltd_token_counts
    assert counts(X, X, 1, top + 1, 100, 0, 0, X, None) == NO
    assert counts(X, X, 1, 4, 2**31 - 1, 0, 1, X, None) == NO


@pytest.mark.parametrize("off", [4, 100 * 4, 399 * 4, -4, -399 * 4])
def test_overlapping_output(off):
    """1 x 4 nodes of 100 tokens are 1600 bytes: an output that begins inside them, or reaches into them."""
    assert process(lg=X, out=X + off) == BAD


def test_binding_status_strides_and_workspace():
    import torch
    c = {k: torch.stack([v] * 3) for k, v in _cache(torch).items()}
    i, path = torch.zeros(2, dtype=torch.int32), torch.zeros((2, 4), dtype=torch.int32)
    move = lambda **kw: ltd.kv_compact_q8(c["k"], c["v"], c["ks"], c["vs"], i, i.clone(), path, i, scale_rows=16, **kw)  # noqa: E731
    for kw in (dict(layer_stride_elems=8193), dict(scale_stride_elems=9), dict(num_layers=2, layer_stride_elems=16385)):
        with pytest.raises(ValueError, match="pass the tensors' end"):
            move(**kw)
    for kw in ({}, dict(num_layers=2), dict(num_layers=2, layer_stride_elems=16384)):
        with pytest.raises(ValueError, match="on a GPU"):
            move(**kw)
    for status in (torch.zeros(1), torch.zeros(1, dtype=torch.uint8), torch.zeros(0, dtype=torch.int32)):
        with pytest.raises(TypeError, match="status"):
            move(validate=True, status=status)
    lg, t = torch.zeros((2, 3, 100)), torch.zeros((2, 3), dtype=torch.int32)
    with pytest.raises(ValueError, match="workspace"):
        ltd.tree_accept_processed(lg, t, t, i, t, t, t, i, workspace=torch.zeros(4096, dtype=torch.uint8)[::2])


def test_the_reference_rounds_as_the_format_does():
    """The test's own encoder against torch's conversion, and its decoder against torch's values."""
    import numpy as np
    import torch
    codes = np.arange(256, dtype=np.uint8)
    want = torch.from_numpy(codes).view(torch.float8_e4m3fn).double().numpy()
    np.testing.assert_array_equal(Q.VALUES, want)
    rng = np.random.default_rng(0)
    x = np.concatenate([rng.normal(size=4000) * np.exp2(rng.integers(-12, 9, 4000)), Q.VALUES[~np.isnan(Q.VALUES)],
                        (Q.VALUES[:126] + Q.VALUES[1:127]) / 2]).astype(np.float32)
    x = x[np.abs(x) <= 448]
    got = Q.encode(x)
    ref = torch.from_numpy(x).to(torch.float8_e4m3fn).view(torch.uint8).numpy()
    np.testing.assert_array_equal(got, ref)
    for top, byte in ((448.0, 127), (448.1, 128), (224.0, 126), (1.75, 119), (1.7500001, 120), (0.0, 27), (np.inf, 214)):
        assert Q.needed(np.array([top], np.float32)) == byte, top
