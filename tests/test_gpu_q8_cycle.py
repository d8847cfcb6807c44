"""Decoding cycles over an 8-bit cache, every call on the last one's outputs: a prompt is appended, then per cycle the
draft tree's rows are appended, the tree is verified, the rules applied, drafts accepted, the table of occurrences and the
cache brought up to date.  Eager and as a graph captured once and replayed, against the same cycle in 64 bits."""
import numpy as np
import pytest

import oracle
import paper_2603_01639_amd as ltd
import q8_util as Q
from test_gpu_q8_attention import tolerance

pytestmark = pytest.mark.gpu

B, Hq, Hkv, d, N, VOC, SR, BLOCK, L = 2, 8, 2, 128, 12, 700, 16, 32, 2


class Cycle:
    """The buffers a decoder keeps and one cycle's calls on them."""

    def __init__(self, c, penalties, bias):
        import torch
        self.c, self.dev = c, Q.dev_cache(c)
        i32 = dict(dtype=torch.int32, device="cuda")
        bf = dict(dtype=torch.bfloat16, device="cuda")
        self.prefix, self.new_prefix, self.n = (torch.zeros(B, **i32) for _ in range(3))
        self.parents, self.tokens, self.pred, self.acc, self.toks = (torch.zeros((B, N), **i32) for _ in range(5))
        self.nacc = torch.zeros(B, **i32)
        self.q, self.out = torch.zeros((L, B, N, Hq, d), **bf), torch.zeros((L, B, N, Hq, d), **bf)
        self.kn, self.vn = torch.zeros((L, B, N, Hkv, d), **bf), torch.zeros((L, B, N, Hkv, d), **bf)
        self.logits, self.done = (torch.zeros((B, N, VOC), device="cuda") for _ in range(2))
        self.mask = torch.zeros((B, N, -(-VOC // 32)), **i32)
        self.counts = torch.zeros((B, VOC), **i32)
        self.pen = Q.to_dev(penalties)
        self.bias = [Q.to_dev(x) for x in bias]
        self.ws = torch.empty(max(16, ltd.attn_q8_workspace_size(B, N, Hq, Hkv, d, 200, ltd.DTYPE_BF16)),
                              dtype=torch.uint8, device="cuda")
        self.wa = torch.empty(ltd.accept_workspace_size(B, N, VOC), dtype=torch.uint8, device="cuda")

    def paged(self):
        return dict(scale_rows=SR, block_table=self.dev["table"], num_blocks=self.c["pages"])

    def run(self):
        v = self.dev
        for x in range(L):
            layer = (v["k"][x], v["v"][x], v["ks"][x], v["vs"][x])
            ltd.kv_append_q8(self.kn[x], self.vn[x], *layer, self.prefix, self.n, **self.paged())
            ltd.tree_verify_attn_q8(self.q[x], *layer, self.prefix, self.parents, self.n, self.out[x], max_prefix=200,
                                    workspace=self.ws, **self.paged())
        rules = dict(counts=self.counts, penalties=self.pen, bias_tokens=self.bias[0], bias_values=self.bias[1],
                     n_bias=self.bias[2], mask=self.mask)
        ltd.tree_process_logits(self.logits, self.tokens, self.parents, self.n, self.done, **rules)
        ltd.tree_accept_processed(self.logits, self.tokens, self.parents, self.n, self.pred, self.acc, self.toks, self.nacc,
                                  workspace=self.wa, **rules)
        ltd.token_counts(self.toks, self.nacc, self.counts)
        ltd.kv_compact_q8(v["k"], v["v"], v["ks"], v["vs"], self.prefix, self.new_prefix, self.acc, self.nacc,
                          num_layers=L, **self.paged())
        self.prefix.copy_(self.new_prefix)


def _inputs(rng, step):
    """One cycle's inputs on the host: the same ones for every way of running it."""
    import torch
    sizes = [int(rng.integers(1, N + 1)), N]
    bf = lambda *s: torch.from_numpy(rng.normal(size=s) * (1 + step)).to(torch.bfloat16)  # noqa: E731
    par = Q.trees(rng, sizes)
    tok = rng.integers(0, VOC, (B, N)).astype(np.int32)
    lg = rng.normal(size=(B, N, VOC)).astype(np.float32)
    for b in range(B):
        for i in range(1, sizes[b]):
            if rng.random() < 0.7:
                lg[b, par[b, i], tok[b, i]] += 30
    mask = rng.integers(-(1 << 31), 1 << 31, (B, N, -(-VOC // 32))).astype(np.int32) | np.int32(0x55555555)
    return dict(parents=par, tokens=tok, n=np.array(sizes, np.int32), logits=lg, mask=mask,
                q=bf(L, B, N, Hq, d), kn=bf(L, B, N, Hkv, d), vn=bf(L, B, N, Hkv, d))


@pytest.mark.parametrize("graph", [False, True])
def test_cycles(graph):
    import torch
    rng = np.random.default_rng(41)
    prompt = [37, 64]
    c = Q.cache(rng, B, Hkv, d, SR, [200, 200], BLOCK, layers=L)
    pen = np.array([[1.2, 0.3, 0.1], [1.0, 0.0, 0.0]], np.float32)
    bias = (np.array([[5, 9], [5, 5]], np.int32), np.array([[2.5, -3.0], [1.0, 4.0]], np.float32), np.array([2, 1], np.int32))
    cy = Cycle(c, pen, bias)
    ref = {k: c[k].copy() for k in ("k", "v", "ks", "vs")}
    # the prompt, layer by layer, and its tokens
    n0 = np.array(prompt, np.int32)
    ptok = rng.integers(0, VOC, (B, max(prompt))).astype(np.int32)
    ltd.token_counts(Q.to_dev(ptok), Q.to_dev(n0), cy.counts, prompt=True, reset=True)
    counts = np.zeros((B, VOC), np.int64)
    for b in range(B):
        counts[b, ptok[b, :prompt[b]]] = -(1 << 31)
    zero = torch.zeros(B, dtype=torch.int32, device="cuda")
    for x in range(L):
        new = {w: torch.from_numpy(rng.normal(size=(B, max(prompt), Hkv, d))).to(torch.bfloat16) for w in "kv"}
        ltd.kv_append_q8(new["k"].to("cuda"), new["v"].to("cuda"), *(cy.dev[w][x] for w in ("k", "v", "ks", "vs")), zero,
                         Q.to_dev(n0), **cy.paged())
        for w in "kv":
            Q.append(ref[w][x], ref[w + "s"][x], new[w].double().numpy(), c["table"], [0, 0], prompt, SR)
    cy.prefix.copy_(Q.to_dev(n0))
    prefix = n0.copy()
    g = None
    for step in range(4):
        m = _inputs(rng, step)
        for k, a in m.items():
            t = a if isinstance(a, torch.Tensor) else torch.from_numpy(a)
            getattr(cy, k).copy_(t)
        if graph and g is None:
            keep = {k: t.clone() for k, t in cy.dev.items() if k != "table"}
            kept = {k: getattr(cy, k).clone() for k in ("prefix", "counts")}
            side = torch.cuda.Stream()
            side.wait_stream(torch.cuda.current_stream())
            g = torch.cuda.CUDAGraph()
            with torch.cuda.stream(side):
                cy.run()
                side.synchronize()
                with torch.cuda.graph(g, stream=side):
                    cy.run()
            torch.cuda.current_stream().wait_stream(side)
            for k, t in keep.items():
                cy.dev[k].copy_(t)
            for k, t in kept.items():
                getattr(cy, k).copy_(t)
        g.replay() if graph else cy.run()
        torch.cuda.synchronize()
        # the same cycle in 64 bits
        for x in range(L):
            layer = {k: ref[k][x] for k in ref}
            for w, new in (("k", m["kn"]), ("v", m["vn"])):
                Q.append(layer[w], layer[w + "s"], new[x].double().numpy(), c["table"], prefix, m["n"], SR)
            k, v = (Q.values(layer, w, c["table"], SR) for w in "kv")
            want, A, S = Q.attention(m["q"][x].double().numpy(), k, v, prefix, m["parents"], m["n"], d ** -0.5)
            got = cy.out[x].double().cpu().numpy()
            for b, n in enumerate(m["n"]):
                tol = tolerance(True, want[b, :n], A[b, :n], S[b, :n], int(prefix[b]) + n, d)
                assert (np.abs(got[b, :n] - want[b, :n]) <= tol).all(), (step, x, b)
        done = Q.rules(m["logits"], m["tokens"], m["parents"], m["n"], counts.astype(np.int32), pen, bias, m["mask"])
        for b, n in enumerate(m["n"]):
            np.testing.assert_allclose(cy.done[b, :n].double().cpu().numpy(), done[b, :n], rtol=1e-5, atol=1e-5)
        full = np.nan_to_num(done, nan=0.0, neginf=-3e38).astype(np.float32)
        pred, path, toks, nacc = oracle.tree_accept(full, m["tokens"], m["parents"], m["n"])
        np.testing.assert_array_equal(cy.nacc.cpu().numpy(), nacc)
        for b in range(B):
            k = int(nacc[b])
            np.testing.assert_array_equal(cy.acc[b, :k].cpu().numpy(), path[b, :k])
            np.testing.assert_array_equal(cy.toks[b, :k].cpu().numpy(), toks[b, :k])
            np.add.at(counts[b], toks[b, :k], 1)
        np.testing.assert_array_equal(cy.counts.cpu().numpy(), counts.astype(np.int32))
        for x in range(L):
            for w in "kv":
                Q.compact(ref[w][x], ref[w + "s"][x], c["table"], prefix, path, nacc, SR)
        prefix = prefix + nacc
        np.testing.assert_array_equal(cy.prefix.cpu().numpy(), prefix)
        for w in "kv":
            gk, gs = cy.dev[w].cpu().numpy(), cy.dev[w + "s"].cpu().numpy()
            for x in range(L):
                for b in range(B):
                    rows = np.arange(prefix[b])
                    got = Q.values(dict(c, **{w: gk[x], w + "s": gs[x]}), w, c["table"], SR)(b, rows)
                    want = Q.values({w: ref[w][x], w + "s": ref[w + "s"][x]}, w, c["table"], SR)(b, rows)
                    np.testing.assert_array_equal(got, want)


def test_two_streams_at_once(monkeypatch):
    """Two cycles' reads side by side on streams of their own, given by argument, with workspaces the calls take: each comes
    from its stream's memory, and the results are those of the calls one after the other."""
    import torch
    rng = np.random.default_rng(43)
    P = [1500, 1024]
    c = Q.cache(rng, B, Hkv, d, SR, [p + N for p in P], BLOCK)
    dev = Q.dev_cache(c)
    prefix, sizes = Q.to_dev(np.array(P, np.int32)), [N, 5]
    n, par = Q.to_dev(np.array(sizes, np.int32)), Q.to_dev(Q.trees(rng, sizes))
    tok = Q.to_dev(rng.integers(0, VOC, (B, N)).astype(np.int32))
    i32 = dict(dtype=torch.int32, device="cuda")
    streams = [torch.cuda.Stream() for _ in range(2)]
    q = [torch.from_numpy(rng.normal(size=(B, N, Hq, d))).to(torch.bfloat16).to("cuda") for _ in streams]
    lg = [torch.from_numpy(rng.normal(size=(B, N, VOC)).astype(np.float32)).to("cuda") for _ in streams]
    took = []
    alloc = ltd._alloc_workspace
    monkeypatch.setattr(ltd, "_alloc_workspace", lambda *a: took.append(torch.cuda.current_stream()) or alloc(*a))

    def read(k, stream):
        out = torch.zeros_like(q[k])
        got = [torch.zeros((B, N), **i32) for _ in range(3)] + [torch.zeros(B, **i32)]
        if stream is not None:
            stream.wait_stream(torch.cuda.current_stream())
        ltd.tree_verify_attn_q8(q[k], dev["k"], dev["v"], dev["ks"], dev["vs"], prefix, par, n, out, max_prefix=1500,
                                scale_rows=SR, block_table=dev["table"], num_blocks=c["pages"], stream=stream)
        ltd.tree_accept_processed(lg[k], tok, par, n, *got, stream=stream)
        return [out] + got

    want = [read(k, None) for k in range(2)]
    torch.cuda.synchronize()
    took.clear()
    got = [read(k, streams[k]) for k in range(2)]
    assert took == [streams[0], streams[0], streams[1], streams[1]]
    torch.cuda.synchronize()
    for a, b in zip(want, got):
        for x, y in zip(a, b):
            torch.testing.assert_close(x, y, rtol=0, atol=0)


def test_compaction_of_all_layers_by_default():
    """A cache with a leading dimension of layers, num_layers left out: every layer moves."""
    import torch
    rng = np.random.default_rng(44)
    P, path, nacc = [30, 3], np.tile(np.arange(N, dtype=np.int32), (B, 1)), np.array([3, 2], np.int32)
    path[0, :3], path[1, :2] = [0, 4, 9], [0, 7]
    c = Q.cache(rng, B, Hkv, d, SR, [p + N for p in P], BLOCK, layers=3)
    dev = Q.dev_cache(c)
    prefix = np.array(P, np.int32)
    new = torch.zeros(B, dtype=torch.int32, device="cuda")
    ltd.kv_compact_q8(dev["k"], dev["v"], dev["ks"], dev["vs"], Q.to_dev(prefix), new, Q.to_dev(path), Q.to_dev(nacc),
                      scale_rows=SR, block_table=dev["table"], num_blocks=c["pages"])
    assert new.tolist() == [33, 5]
    for w in "kv":
        gk, gs = dev[w].cpu().numpy(), dev[w + "s"].cpu().numpy()
        for x in range(3):
            ref = {w: c[w][x].copy(), w + "s": c[w + "s"][x].copy()}
            Q.compact(ref[w], ref[w + "s"], c["table"], prefix, path, nacc, SR)
            for b in range(B):
                rows = np.arange(prefix[b] + nacc[b])
                np.testing.assert_array_equal(Q.values({w: gk[x], w + "s": gs[x]}, w, c["table"], SR)(b, rows),
                                              Q.values(ref, w, c["table"], SR)(b, rows))
