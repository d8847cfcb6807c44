"""Which places rotary positions' and the latent cache's calls may share, on the CPU: what they refuse in the C ABI, and that
the binding lets other parts of one buffer through (to its refusal of CPU tensors; nothing is launched)."""
import pytest

import paper_2603_01639_amd as ltd
from test_latent_refusals import BAD, attn, rope

F = 1 << 20  # bytes that no case reaches by chance

# 4 rows of 8 + 2 + 8 + 2 heads of 64 bfloat16 elements: rows of 2560 bytes, heads of 128
ROW, HEAD = 1280, 128
AT = dict(q=F, k=F + 8 * HEAD, qo=F + 10 * HEAD, ko=F + 18 * HEAD)


def fused(**heads):
    """Places in heads of the fused buffer, from AT where not given."""
    at = {k: F + HEAD * heads[k] if k in heads else v for k, v in AT.items()}
    return rope(**at, qr=ROW, kr=ROW, qor=ROW, kor=ROW)


@pytest.mark.parametrize("heads", [
    dict(qo=9), dict(qo=7), dict(qo=1), dict(ko=9), dict(ko=7), dict(ko=17), dict(ko=10), dict(k=11), dict(k=17), dict(q=11),
    dict(q=17), dict(qo=13), dict(ko=8 + 20 * 2 + 1), dict(qo=-20 + 18, ko=19)])
def test_rope_refuses_shared_heads(heads):
    assert fused(**heads) == BAD


@pytest.mark.parametrize("kw", [
    dict(qo=F + 64), dict(qo=F + 126, ko=3 * F), dict(qo=F + 2),
    # (rows of 1024 bytes 2048 apart: from 1024 on they would lie between)
    dict(qr=1024, qo=F + 1022, qor=1024), dict(qr=1024, qo=F + 1026, qor=1024)])
def test_rope_refuses_outputs_that_meet_inputs(kw):
    assert rope(**{**dict(q=F, k=5 * F, ko=7 * F), **kw}) == BAD


def test_binding_takes_other_parts_of_one_buffer():
    import torch
    f, i = torch.zeros(32, dtype=torch.float64), torch.zeros(2, dtype=torch.int32)
    buf = torch.zeros((2, 4, 20, 64), dtype=torch.bfloat16)

    def run(q, q_out, **kw):
        ltd.tree_rope(q, q_out, f, i, i, **kw)

    with pytest.raises(ValueError, match="on a GPU"):
        run(buf[:, :, :8], buf[:, :, 8:16])
    with pytest.raises(ValueError, match="on a GPU"):
        run(buf[:, :, :8], buf[:, :, 10:18], k=buf[:, :, 8:10], k_out=buf[:, :, 18:])
    with pytest.raises(ValueError, match="on a GPU"):
        run(buf[:, :, 0:16:2], buf[:, :, 1:16:2])
    with pytest.raises(ValueError, match="on a GPU"):
        run(buf[:, :, 0:16:2], buf[:, :, 16:].reshape(2, 4, 4, 64)[:, :, :1].expand(2, 4, 8, 64).contiguous())
    wide = torch.zeros((2, 4, 8, 128), dtype=torch.float32)
    with pytest.raises(ValueError, match="on a GPU"):
        run(wide[..., :64], wide[..., 64:])
    with pytest.raises(ValueError, match="q_out overlaps q"):
        run(wide[..., :64], wide[..., 32:96])
    with pytest.raises(ValueError, match="k_out overlaps k"):
        run(buf[:, :, :8], buf[:, :, :8], k=buf[:, :, 8:12], k_out=buf[:, :, 9:13])
    with pytest.raises(ValueError, match="q_out overlaps q"):
        run(buf[:, :, :8], buf[:, :, 7:15])
    with pytest.raises(ValueError, match="q_out overlaps q"):  # heads two apart and one apart
        run(buf[:, :, 0:16:2], buf[:, :, 8:16])


# A sequence's 64 cache rows of 576 float32 elements are 147456 bytes, four rows of 16 heads of 512 131072, of 64 16384.
APART = dict(ql=F, qr=2 * F, cache=3 * F, out=4 * F)


@pytest.mark.parametrize("kw", [
    dict(out=3 * F), dict(out=3 * F + 147456 - 16), dict(out=3 * F - 131072 + 16), dict(out=3 * F + 1024),
    dict(B=2, out=3 * F + 2 * 147456 - 16), dict(table=F, mb=1, nb=5, out=3 * F + 5 * 147456 - 16)])
def test_attention_refuses_outputs_over_its_cache(kw):
    assert attn(**{**APART, **kw}) == BAD


def size():
    n = ltd.attn_latent_workspace_size(1, 60, 16, 512, 64, 4096, ltd.DTYPE_BF16)
    assert n > 0
    return n


# bfloat16, 60 nodes, one sequence of 8192 rows: out and q_latent 983040 bytes, q_rope 122880, cache 9437184
@pytest.mark.parametrize("over, at", [("ql", 0), ("ql", 983040 - 16), ("qr", 0), ("qr", 122880 - 16), ("cache", 0),
                                      ("cache", 9437184 - 16), ("out", 0), ("out", 983040 - 16), ("ql", None), ("out", None)])
def test_attention_refuses_a_workspace_over_its_tensors(over, at):
    """From byte `at` of the tensor on, or with its last 16 bytes over the tensor's first."""
    place = dict(ql=1 << 40, qr=2 << 40, cache=3 << 40, out=4 << 40)
    ws = place[over] + (16 - size() // 16 * 16 if at is None else at)
    assert attn(**place, dtype=1, N=60, mp=4096, rows=8192, qlr=8192, ws=ws, wsb=1 << 38) == BAD
