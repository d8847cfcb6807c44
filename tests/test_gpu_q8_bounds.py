"""Short units over an 8-bit cache under bounds on the prefix far above the call's own lengths, as a captured graph passes:
the splits follow the lengths alone, so the answer is the same bit for bit, and it is right where there are more splits
than workgroups.  (The reference and its tolerance are those of test_gpu_q8_attention.)"""
import numpy as np
import pytest

import paper_2603_01639_amd as ltd
import q8_util as Q
from test_gpu_q8_attention import check, make, run

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("B, prefix, sizes, Hq, Hkv, d, block", [
    (1, [4096], [1], 8, 2, 128, 0), (1, [3000], [4], 8, 8, 64, 16), (3, [0, 5000, 129], [1, 3, 8], 8, 2, 128, 16),
    (16, None, [1] * 16, 16, 8, 128, 16), (16, None, [4] * 16, 16, 4, 64, 0), (70, None, [1] * 70, 8, 4, 128, 32)])
def test_the_bound_changes_no_bit(B, prefix, sizes, Hq, Hkv, d, block):
    import torch
    rng = np.random.default_rng(B)
    prefix = prefix or [int(x) for x in rng.integers(200, 2200 if B < 64 else 700, B)]
    m = make(B + d, B, Hq, Hkv, d, 16, prefix, sizes, block)
    tight = run(m)
    check(m, tight, label="tight")
    for bound in (16384, 40000, 131072, 1 << 20):
        loose = run(m, max_prefix=bound)
        assert torch.equal(loose.view(torch.int16), tight.view(torch.int16)), bound


@pytest.mark.parametrize("paged", [False, True])
@pytest.mark.parametrize("B, H, d, lengths", [(16, 8, 128, [31000, 30999, 64]), (64, 8, 64, [16500, 15400, 17000]), (64, 8, 64, [47000, 46900, 64]),
                                              (1, 100, 64, [39000])])
def test_more_splits_than_workgroups(B, H, d, lengths, paged):
    """Prefixes for which one split a workgroup would be longer than a split may be: each workgroup takes several.  The
    heads hold the same rows and ask the same, so that each answer of a length stands for all of them."""
    import torch
    rng = np.random.default_rng(d + B)
    block, sr, pages = 64, 16, 40
    codes = {w: Q.encode(np.clip(rng.normal(size=(pages, 1, block, d)) * 110, -448, 448)) for w in "kv"}
    codes |= {w + "s": rng.integers(119, 122, (pages, 1, block // sr)).astype(np.uint8) for w in "kv"}
    prefix = np.resize(np.array(lengths, np.int32), B)
    prefix[B // 2:] = lengths[0]
    per = -(-(int(prefix.max()) + 1) // block)
    table = rng.integers(0, pages, per).astype(np.int32)  # (pages are read by many rows and sequences)
    if paged:
        dev = {w: Q.to_dev(x).expand(pages, H, *x.shape[2:]).contiguous() for w, x in codes.items()}
        where = dict(block_table=Q.to_dev(np.tile(table, (B, 1))), num_blocks=pages)
    else:
        flat = {w: np.ascontiguousarray(x[table, 0].reshape(1, 1, -1, *x.shape[3:])) for w, x in codes.items()}
        dev = {w: Q.to_dev(x).expand(B, H, *x.shape[2:]).contiguous() for w, x in flat.items()}
        where = {}
    q = torch.from_numpy(rng.normal(size=d) * 1.5).to(torch.bfloat16).expand(B, 1, H, d).contiguous()
    par, n = np.full((B, 1), -1, np.int32), np.ones(B, np.int32)
    out = torch.full_like(q, 7.0, device="cuda")
    ltd.tree_verify_attn_q8(q.to("cuda"), dev["k"], dev["v"], dev["ks"], dev["vs"], Q.to_dev(prefix), Q.to_dev(par),
                            Q.to_dev(n), out, max_prefix=int(prefix.max()), scale_rows=sr, **where)
    torch.cuda.synchronize()
    got = out.cpu()
    one = dict(c=dict(codes, table=table[None]), sr=sr, q=q[:1, :, :1], n=n[:1], par=par[:1])
    for length in sorted(set(prefix.tolist())):
        rows = got[torch.from_numpy(prefix == length)].view(torch.int16).reshape(-1, d)
        assert (rows == rows[0]).all(), length
        check(dict(one, prefix=np.array([length], np.int32)), rows[0].view(torch.bfloat16).view(1, 1, 1, d),
              label=f"length {length}")


@pytest.mark.parametrize("B, n", [(1, 1), (16, 1), (16, 4)])
def test_a_captured_call_follows_its_lengths(B, n):
    """A graph captured under a bound far above the lengths, whose prefixes then grow and shrink between replays: each
    replay answers as an eager call with tight bounds."""
    import torch
    lengths = [[40] * B, [3000 - 100 * b for b in range(B)], [0] * B, [2500 if b == B // 2 else 7 for b in range(B)]]
    top = [max(x[b] for x in lengths) for b in range(B)]
    m = make(5, B, 8, 2, 128, 16, top, [n] * B, 16)
    dev = Q.dev_cache(m["c"])
    q, par, sizes = m["q"].to("cuda"), Q.to_dev(m["par"]), Q.to_dev(m["n"])
    prefix, out = Q.to_dev(np.array(lengths[0], np.int32)), torch.full_like(q, 7.0)
    ws = torch.empty(ltd.attn_q8_workspace_size(B, n, 8, 2, 128, 131072, ltd.DTYPE_BF16), dtype=torch.uint8, device="cuda")
    call = lambda: ltd.tree_verify_attn_q8(q, dev["k"], dev["v"], dev["ks"], dev["vs"], prefix, par, sizes, out,  # noqa: E731
                                           max_prefix=131072, scale_rows=16, block_table=dev["table"],
                                           num_blocks=m["c"]["pages"], workspace=ws)
    side, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        call()
        side.synchronize()
        with torch.cuda.graph(graph, stream=side):
            call()
    for x in lengths + lengths[:2]:
        prefix.copy_(torch.tensor(x, dtype=torch.int32))
        out.fill_(7.0)
        ws.fill_(0xFF)
        graph.replay()
        torch.cuda.synchronize()
        now = dict(m, prefix=np.array(x, np.int32))
        check(now, out, label=str(x[:3]))
        assert torch.equal(out.view(torch.int16), run(now, dev=dev).view(torch.int16))
