"""Latent attention at the ends of what its documentation takes: the largest latent values, head strides of either sign, and
batches of more sequences than the shares that a GPU's workgroups could have.  Tolerances are those of the attention tests."""
import numpy as np
import pytest

import latent_util as L
import paper_2603_01639_amd as ltd
from test_gpu_latent_attention import check, make, run

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["bfloat16", "float32"])
@pytest.mark.parametrize("H, DL, prefix, sizes", [(16, 512, [3000, 40], [1, 1]), (16, 512, [2500], [20]), (128, 256, [1500], [1])])
def test_latent_values_of_2_to_the_80(H, DL, prefix, sizes, dtype):
    """In rows that are cut, with most scores 14.9 powers of two above the first tile's of their piece: the maximum stays
    behind, and weights of up to 2^15 multiply the values."""
    import torch
    m = make(21, H, DL, prefix, sizes, 0, dtype)
    big = 2.0 ** 80
    t = np.arange(m["cache"].shape[1])
    climb = np.where(t // 32 % 5 == 0, 0.0, 14.9 * np.log(2.0))
    q = m["q"].double() * 0.05
    q[..., :DL] /= big
    q[..., DL] = 8.0
    m["cache"][..., :DL] *= big
    m["cache"][:, :, DL] = torch.from_numpy(climb / (8.0 * m["scale"])).to(m["cache"].dtype)
    q = q.to(m["q"].dtype)
    m.update(q=q, ql=q[..., :DL], qr=q[..., DL:], layout="rows")
    check(m, run(m))


@pytest.mark.parametrize("dtype", ["bfloat16", "float32"])
@pytest.mark.parametrize("H, n", [(2, 3), (16, 1), (16, 9)])
def test_heads_in_reverse_storage(H, n, dtype):
    import torch
    DL = 256
    m = make(22, H, DL, [33, 600], [n, 1], 0, dtype, nmax=n)
    base = run(m)
    q = m["q"].to("cuda").flip(2).contiguous()
    cache, out = m["cache"].to("cuda"), torch.full_like(base, 7.0)
    D, elem = DL + L.ROPE, q.element_size()
    kind = ltd.DTYPE_BF16 if dtype == "bfloat16" else ltd.DTYPE_F32
    size = ltd.attn_latent_workspace_size(2, n, H, DL, L.ROPE, 600, kind)
    ws = torch.empty(max(size, 1), dtype=torch.uint8, device="cuda")
    P, par, ns = L.to_dev(m["prefix"]), L.to_dev(m["par"]), L.to_dev(m["n"])
    last = q.data_ptr() + (H - 1) * D * elem
    assert ltd.lib().ltd_tree_verify_attn_latent(
        last, H * D, -D, last + DL * elem, H * D, -D, cache.data_ptr(), None, P.data_ptr(), par.data_ptr(), ns.data_ptr(),
        out.data_ptr(), 2, n, H, DL, L.ROPE, 600, cache.shape[1], 0, 0, m["scale"], kind, ws.data_ptr(), size, 0, None,
        torch.cuda.current_stream().cuda_stream) == ltd.LTD_OK
    torch.cuda.synchronize()
    assert torch.equal(out, base)


@pytest.mark.parametrize("H, n, block", [(16, 1, 16), (4, 4, 0), (40, 1, 0), (16, 3, 8)])
def test_more_sequences_than_shares(H, n, block):
    """1100 short ones, empty ones among them."""
    rng = np.random.default_rng(H + n)
    B = 1100
    prefix = [int(p) for p in rng.choice([0, 1, 15, 31, 32, 70], size=B)]
    sizes = [int(s) for s in rng.integers(0, n + 1, size=B)]
    prefix[-1], sizes[-1], sizes[0] = 400, n, n
    m = make(B + H, H, 256, prefix, sizes, block, nmax=n)
    check(m, run(m))
