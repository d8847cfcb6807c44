"""Which layers the binding's compaction of an 8-bit cache lets through, on the CPU (nothing is launched)."""
import pytest

import paper_2603_01639_amd as ltd

B, H, ROWS, D, SR, L = 2, 2, 32, 64, 16, 3
SIZE, SSIZE = B * H * ROWS * D, B * H * ROWS // SR  # a layer's codes and scale bytes
GAP, SGAP = 4096, 64


def _move(offset=0, **kw):
    """Compaction of L layers, GAP codes and SGAP bytes apart, from the views of the first (`offset` layers in)."""
    import torch
    at, sat = offset * (SIZE + GAP), offset * (SSIZE + SGAP)
    codes = [torch.zeros((SIZE + GAP) * L - GAP, dtype=torch.uint8)[at:at + SIZE].view(B, H, ROWS, D) for _ in "kv"]
    scales = [torch.zeros((SSIZE + SGAP) * L - SGAP, dtype=torch.uint8)[sat:sat + SSIZE].view(B, H, ROWS // SR) for _ in "kv"]
    i, path = torch.zeros(B, dtype=torch.int32), torch.zeros((B, 4), dtype=torch.int32)
    args = dict(num_layers=L, layer_stride_elems=SIZE + GAP, scale_stride_elems=SSIZE + SGAP)
    ltd.kv_compact_q8(*codes, *scales, i, i.clone(), path, i, scale_rows=SR, **{**args, **kw})


@pytest.mark.parametrize("kw", [dict(), dict(num_layers=2), dict(num_layers=1, layer_stride_elems=0, scale_stride_elems=0),
                                dict(offset=1, num_layers=2), dict(layer_stride_elems=SIZE, scale_stride_elems=SSIZE)])
def test_layers_inside_the_buffers(kw):
    with pytest.raises(ValueError, match="on a GPU"):  # (every check before the launch has passed)
        _move(**kw)


@pytest.mark.parametrize("kw", [dict(num_layers=4), dict(layer_stride_elems=SIZE + GAP + 16),
                                dict(scale_stride_elems=SSIZE + SGAP + 1), dict(offset=1), dict(offset=2, num_layers=2)])
def test_layers_past_the_buffers(kw):
    """One layer's view of a buffer, with layers or strides that would write past the buffer's end."""
    with pytest.raises(ValueError, match="pass the tensors' end"):
        _move(**kw)
