"""What rotary positions' and the latent cache's calls refuse, on the CPU: scalars and pointers in the C ABI, and types,
shapes and layouts in the binding (nothing is launched)."""
import pytest

import paper_2603_01639_amd as ltd

X = 4096  # a pointer that no refused call follows
FN = ltd.lib
BAD, NO, WS = ltd.LTD_EINVAL, ltd.LTD_EUNSUPPORTED, ltd.LTD_EWORKSPACE
TOP = ltd.MAX_LENGTH


def rope(**kw):
    a = dict(q=X, qr=512, qh=64, qo=2 * X, qor=512, qoh=64, k=X, kr=128, kh=64, ko=2 * X, kor=128, koh=64, freq=X, prefix=X,
             depth=None, n=X, B=1, N=4, Hq=8, Hk=2, d=64, off=0, rot=64, inter=0, m=1.0, dtype=1, validate=0, status=None)
    a.update(kw)
    return FN().ltd_tree_rope(*a.values(), None)


def append(**kw):
    a = dict(x=X, stride=576, w=X, eps=1e-6, freq=X, inter=1, m=1.0, cache=X, table=None, prefix=X, depth=None, n=X, B=1, N=4,
             dl=512, dr=64, rows=64, mb=0, nb=0, dtype=1, validate=0, status=None)
    a.update(kw)
    return FN().ltd_latent_append(*a.values(), None)


def attn(**kw):
    a = dict(ql=X, qlr=8192, qlh=512, qr=X, qrr=1024, qrh=64, cache=X, table=None, prefix=X, par=X, n=X, out=X, B=1, N=4, Hq=16,
             dl=512, dr=64, mp=16, rows=64, mb=0, nb=0, scale=0.1, dtype=0, ws=None, wsb=0, validate=0, status=None)
    a.update(kw)
    return FN().ltd_tree_verify_attn_latent(*a.values(), None)


def compact(**kw):
    a = dict(cache=X, table=None, prefix=X, new=X + 64, path=X, n=X, B=1, N=4, dl=512, dr=64, rows=64, mb=0, nb=0, layers=1,
             ls=0, dtype=1, validate=0, status=None)
    a.update(kw)
    return FN().ltd_latent_compact(*a.values(), None)


@pytest.mark.parametrize("kw, code", [
    (dict(B=-1), BAD), (dict(N=0), BAD), (dict(Hq=0), BAD), (dict(Hk=-1), BAD), (dict(rot=63), BAD), (dict(rot=0), BAD),
    (dict(off=-2), BAD), (dict(off=2), BAD), (dict(off=2**31 - 1), BAD), (dict(m=float("nan")), BAD), (dict(m=float("inf")), BAD),
    (dict(dtype=2), NO), (dict(d=4098, rot=2), NO), (dict(N=TOP + 1), NO), (dict(Hq=2**31 - 1), NO), (dict(q=None), BAD),
    (dict(qo=None), BAD), (dict(k=None), BAD), (dict(freq=None), BAD), (dict(prefix=None), BAD), (dict(n=None), BAD),
    (dict(qo=X, qor=640), BAD), (dict(ko=X, koh=128), BAD), (dict(validate=1), BAD), (dict(B=0, q=None), 0),
    (dict(qor=511), BAD), (dict(qoh=0), BAD), (dict(qor=0), BAD), (dict(qor=-512), BAD), (dict(koh=63), BAD), (dict(kor=127), BAD),
    (dict(qor=64, qoh=255), BAD), (dict(qor=2**62, qoh=2**62, Hq=100), BAD), (dict(q=2 * X, qr=512, qh=0), BAD)])
def test_rope(kw, code):
    assert rope(**kw) == code


@pytest.mark.parametrize("kw, code", [
    (dict(B=-1), BAD), (dict(N=0), BAD), (dict(rows=0), BAD), (dict(eps=-1.0), BAD), (dict(eps=float("nan")), BAD),
    (dict(m=float("inf")), BAD), (dict(dl=128), NO), (dict(dl=576), NO), (dict(dr=32), NO), (dict(dtype=3), NO),
    (dict(N=TOP + 1), NO), (dict(table=X, mb=0, nb=1), BAD), (dict(table=X, mb=1, nb=0), BAD), (dict(stride=575), BAD),
    (dict(stride=580), BAD), (dict(stride=578, dtype=0), BAD), (dict(x=X + 2), BAD), (dict(cache=X + 8), BAD), (dict(w=X + 4), BAD), (dict(x=None), BAD),
    (dict(cache=None), BAD), (dict(freq=None), BAD), (dict(n=None), BAD), (dict(validate=1), BAD), (dict(B=0, x=None), 0)])
def test_append(kw, code):
    assert append(**kw) == code


@pytest.mark.parametrize("kw, code", [
    (dict(B=-1), BAD), (dict(N=0), BAD), (dict(N=257), BAD), (dict(Hq=0), BAD), (dict(mp=-1), BAD), (dict(rows=0), BAD),
    (dict(scale=0.0), BAD), (dict(scale=-1.0), BAD), (dict(scale=float("nan")), BAD), (dict(dl=384), NO), (dict(dr=128), NO),
    (dict(dtype=7), NO), (dict(mp=TOP + 1), NO), (dict(B=65536), NO), (dict(table=X, mb=1, nb=0), BAD), (dict(ql=None), BAD),
    (dict(qr=None), BAD), (dict(out=None), BAD), (dict(par=None), BAD), (dict(cache=X + 8), BAD), (dict(out=X + 4), BAD),
    (dict(dtype=1, ql=X + 2), BAD), (dict(dtype=1, qrh=60), BAD), (dict(dtype=1, qlr=516), BAD), (dict(validate=1), BAD),
    (dict(dtype=1, N=60, mp=4096, rows=8192), WS), (dict(dtype=1, N=60, mp=4096, rows=8192, ws=X, wsb=64), WS),
    (dict(dtype=1, N=60, mp=4096, rows=8192, ws=X + 8, wsb=1 << 40), WS), (dict(B=0, ql=None), 0)])
def test_attention(kw, code):
    assert attn(**kw) == code


@pytest.mark.parametrize("kw, code", [
    (dict(B=-1), BAD), (dict(N=257), BAD), (dict(layers=0), BAD), (dict(layers=65536, ls=64), BAD), (dict(ls=-8), BAD),
    (dict(dl=64), NO), (dict(dr=0), NO), (dict(dtype=2), NO), (dict(new=X), BAD), (dict(layers=2), BAD),
    (dict(layers=2, ls=36), BAD), (dict(cache=None), BAD), (dict(cache=X + 4), BAD), (dict(path=None), BAD),
    (dict(table=X, mb=0, nb=1), BAD), (dict(validate=1), BAD), (dict(B=0, cache=None), 0)])
def test_compact(kw, code):
    assert compact(**kw) == code


F = 1 << 20  # bytes that no case below reaches


@pytest.mark.parametrize("kw", [
    dict(qo=F, ko=F), dict(qo=X, q=F, k=X, ko=2 * F), dict(ko=X, q=X, qo=F, k=2 * F)])
def test_rope_refuses_queries_and_keys_in_one_place(kw):
    assert rope(**kw) == BAD


# rows of 576 bfloat16 elements are 1152 bytes: 4 of them 4608; a cache of one sequence is 64 rows, 73728
@pytest.mark.parametrize("kw", [
    dict(x=F, cache=F), dict(x=F, cache=F + 4608 - 16), dict(x=F + 73728 - 16, cache=F),
    dict(x=F + 73728 * 3 - 16, cache=F, table=X, mb=1, nb=3), dict(x=F, cache=F + 3 * 1152, stride=1152),
    dict(x=F + 147456 - 16, cache=F, dtype=0)])
def test_append_refuses_rows_of_the_cache(kw):
    assert append(**kw) == BAD


# four rows of 16 heads of 512 float32 elements are 131072 bytes, those of 64 dims 16384
@pytest.mark.parametrize("kw", [
    dict(ql=F, out=F), dict(ql=F, out=F + 131072 - 16), dict(ql=F + 131072 - 16, out=F),
    dict(qr=F, out=F + 16384 - 16, ql=8 * F), dict(qr=F + 131072 - 16, out=F, ql=8 * F),
    dict(ql=F, qlr=512, qlh=4 * 512, out=F + 65536), dict(ql=F, qlr=0, qlh=0, out=F + 2048 - 16),
    dict(ql=F, qlr=-8192, out=F - 3 * 32768)])
def test_attention_refuses_outputs_over_its_queries(kw):
    assert attn(**kw) == BAD


def test_workspace_query():
    size = ltd.attn_latent_workspace_size
    assert size(1, 60, 16, 384, 64, 2048, ltd.DTYPE_BF16) == 0
    assert size(1, 300, 16, 512, 64, 2048, ltd.DTYPE_BF16) == 0
    assert size(1, 60, 16, 512, 64, TOP + 1, ltd.DTYPE_BF16) == 0
    assert size(1, 60, 16, 512, 64, 2048, ltd.DTYPE_F32) == 0
    assert size(1, 60, 16, 512, 64, 2048, ltd.DTYPE_BF16) > 0
    assert size(0, 60, 16, 512, 64, 2048, ltd.DTYPE_BF16) == 0


# ---- the binding's checks, with CPU tensors

def _i(torch, *shape):
    return torch.zeros(shape, dtype=torch.int32)


def test_binding_rope():
    import torch
    q, k = torch.zeros((2, 4, 8, 64), dtype=torch.bfloat16), torch.zeros((2, 4, 2, 64), dtype=torch.bfloat16)
    f, i = torch.zeros(32, dtype=torch.float64), _i(torch, 2)

    def run(q=q, q_out=None, f=f, i=i, n=i, **kw):
        ltd.tree_rope(q, torch.zeros_like(q) if q_out is None else q_out, f, i, n, **kw)

    with pytest.raises(ValueError, match="on a GPU"):
        run()
    with pytest.raises(ValueError, match="on a GPU"):
        run(q_out=q, k=k, k_out=k)
    with pytest.raises(TypeError, match="unsupported dtype"):
        run(q=q.half())
    with pytest.raises(TypeError, match="q_out have types"):
        run(q_out=q.float())
    with pytest.raises(ValueError, match="q_out has shape"):
        run(q_out=q[:, :3])
    with pytest.raises(ValueError, match="come together"):
        run(k=k)
    with pytest.raises(ValueError, match="k has shape"):
        run(k=k[:, :3], k_out=k[:, :3])
    with pytest.raises(TypeError, match="inv_freq has type"):
        run(f=f.float())
    with pytest.raises(ValueError, match="dims 0 to 66 of 64"):
        run(f=torch.zeros(33, dtype=torch.float64))
    with pytest.raises(ValueError, match="dims 8 to 72 of 64"):
        run(rot_offset=8)
    with pytest.raises(ValueError, match="depth has shape"):
        run(depth=_i(torch, 2, 3))
    with pytest.raises(TypeError, match="n_rows has type"):
        run(n=i.long())
    with pytest.raises(ValueError, match="evenly spaced"):
        run(q=torch.zeros((2, 8, 8, 64), dtype=torch.bfloat16)[:, :4])
    with pytest.raises(ValueError, match="not contiguous"):
        run(q=torch.zeros((2, 4, 64, 8), dtype=torch.bfloat16).transpose(2, 3))
    buf = torch.zeros((2, 4, 9, 64), dtype=torch.bfloat16)
    with pytest.raises(ValueError, match="q_out overlaps q"):
        run(q=buf[:, :, :8], q_out=buf[:, :, 1:])


def _cache(torch, pages=2, rows=32, d=576, dtype="bfloat16"):
    return torch.zeros((pages, rows, d), dtype=getattr(torch, dtype))


def test_binding_append():
    import torch
    x, f, i = torch.zeros((2, 4, 576), dtype=torch.bfloat16), torch.zeros(32, dtype=torch.float64), _i(torch, 2)

    def run(x=x, cache=None, f=f, n=i, **kw):
        ltd.latent_append(x, _cache(torch) if cache is None else cache, f, i, n, **kw)

    with pytest.raises(ValueError, match="on a GPU"):
        run()
    with pytest.raises(TypeError, match="kv_new has type"):
        run(cache=_cache(torch, dtype="float32"))
    with pytest.raises(ValueError, match="the cache's have 576"):
        run(x=x[:, :, :512])
    with pytest.raises(ValueError, match="norm_weight has shape"):
        run(norm_weight=torch.ones(576, dtype=torch.bfloat16))
    with pytest.raises(TypeError, match="norm_weight has type"):
        run(norm_weight=torch.ones(512))
    with pytest.raises(ValueError, match="cache is not contiguous"):
        run(cache=_cache(torch, rows=64)[:, ::2])
    with pytest.raises(ValueError, match="holds 1 sequences"):
        run(cache=_cache(torch, pages=1))
    with pytest.raises(ValueError, match="num_blocks"):
        run(block_table=_i(torch, 2, 2), num_blocks=3)
    with pytest.raises(ValueError, match="rows for 2 sequences"):
        run(block_table=_i(torch, 1, 2), num_blocks=2)
    with pytest.raises(ValueError, match="evenly spaced"):
        run(x=torch.zeros((2, 8, 576), dtype=torch.bfloat16)[:, :4])


def test_binding_attention_and_compaction():
    import torch
    ql, qr = torch.zeros((2, 4, 16, 512), dtype=torch.bfloat16), torch.zeros((2, 4, 16, 64), dtype=torch.bfloat16)
    i, par = _i(torch, 2), _i(torch, 2, 4)

    def run(ql=ql, qr=qr, cache=None, par=par, out=None, **kw):
        ltd.tree_verify_attn_latent(ql, qr, _cache(torch) if cache is None else cache, i, par, i,
                                    torch.zeros_like(ql, memory_format=torch.contiguous_format) if out is None else out,
                                    max_prefix=8, scale=0.1, **kw)

    with pytest.raises(ValueError, match="on a GPU"):
        run()
    with pytest.raises(ValueError, match="on a GPU"):
        run(ql=ql.permute(2, 0, 1, 3).contiguous().permute(1, 2, 0, 3))
    with pytest.raises(TypeError, match="cache torch.float32"):
        run(cache=_cache(torch, dtype="float32"))
    with pytest.raises(ValueError, match="cache rows of 576"):
        run(ql=ql[..., :256], out=ql[..., :256].contiguous())
    with pytest.raises(ValueError, match="out has shape"):
        run(out=ql[:, :, :8].contiguous())
    with pytest.raises(ValueError, match="parents has shape"):
        run(par=par[:, :3])
    with pytest.raises(ValueError, match="not contiguous"):
        run(qr=torch.zeros((2, 4, 64, 16), dtype=torch.bfloat16).transpose(2, 3))
    with pytest.raises(ValueError, match="workspace"):
        run(workspace=torch.zeros(4096, dtype=torch.uint8)[::2])
    with pytest.raises(TypeError):  # the scale has no default
        ltd.tree_verify_attn_latent(ql, qr, _cache(torch), i, par, i, ql, max_prefix=8)
    move = lambda c, new=None, path=par: ltd.latent_compact(c, i, i.clone() if new is None else new, path, i)  # noqa: E731
    with pytest.raises(ValueError, match="on a GPU"):
        move(_cache(torch))
    with pytest.raises(ValueError, match="on a GPU"):
        move(_cache(torch)[None])
    with pytest.raises(ValueError, match="dimensions"):
        move(_cache(torch)[0])
    with pytest.raises(ValueError, match="accepted_nodes has shape"):
        move(_cache(torch), path=i)
    with pytest.raises(TypeError, match="status"):
        ltd.latent_compact(_cache(torch), i, i.clone(), par, i, validate=True, status=torch.zeros(1))
