"""Rotary positions between parts of one buffer: the same bits as between tensors of their own."""
import numpy as np
import pytest

import latent_util as L
import paper_2603_01639_amd as ltd

pytestmark = pytest.mark.gpu

PARTS = {  # heads of a row's 20 (queries 8, keys 2): queries, their output, keys, theirs
    "outputs behind": (slice(0, 8), slice(10, 18), slice(8, 10), slice(18, 20)),
    "in turn": (slice(0, 16, 2), slice(1, 17, 2), slice(16, 19, 2), slice(17, 20, 2)),
    "queries in place": (slice(0, 8), slice(0, 8), slice(8, 10), slice(10, 12)),
    "both in place": (slice(4, 12), slice(4, 12), slice(12, 14), slice(12, 14)),
    "keys between": (slice(0, 8), slice(12, 20), slice(8, 10), slice(10, 12)),
}


@pytest.mark.parametrize("dtype", ["bfloat16", "float32"])
@pytest.mark.parametrize("inter", [False, True])
@pytest.mark.parametrize("rot, off", [(64, 0), (36, 8), (32, 16)])
@pytest.mark.parametrize("parts", PARTS, ids=lambda s: s.replace(" ", "-"))
def test_parts_of_one_buffer(parts, rot, off, inter, dtype):
    import torch
    rng = np.random.default_rng(rot + off)
    B, N, d = 3, 9, 64
    buf = torch.from_numpy(rng.normal(size=(B, N, 20, d))).to(getattr(torch, dtype)).cuda()
    freq = L.to_dev(L.frequencies(rot))
    prefix, n, dep = L.to_dev(np.array([0, 70, 12345], np.int32)), L.to_dev(np.array([9, 4, 7], np.int32)), \
        L.to_dev(rng.integers(0, 6, (B, N)).astype(np.int32))
    q, q_out, k, k_out = (buf[:, :, p] for p in PARTS[parts])
    want_q, want_k = q_out.clone(), k_out.clone()
    kw = dict(depth=dep, rot_offset=off, interleaved=inter, mscale=1.25)
    ltd.tree_rope(q.clone(), want_q, freq, prefix, n, k=k.clone(), k_out=want_k, **kw)
    before = buf.clone()
    ltd.tree_rope(q, q_out, freq, prefix, n, k=k, k_out=k_out, **kw)
    torch.cuda.synchronize()
    assert torch.equal(q_out, want_q) and torch.equal(k_out, want_k)
    written = torch.zeros(20, dtype=torch.bool)
    written[PARTS[parts][1]] = written[PARTS[parts][3]] = True
    assert torch.equal(buf[:, :, ~written], before[:, :, ~written])
