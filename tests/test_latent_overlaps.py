"""Which places rotary positions' and the latent cache's calls may share, on the CPU: what they refuse in the C ABI, and that
the binding lets other parts of one buffer through (to its refusal of CPU tensors; nothing is launched)."""
import pytest

import paper_2603_01639_amd as ltd
from test_latent_refusals import BAD, rope

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
