"""Verification cycles over a latent cache as a program runs them: the tree's queries get their positions, its rows join the
cache, attention, the accepted path moves next to the prefix; eagerly, captured, and beside other work.

A cycle is checked after every call, against the 64-bit implementation of that call on what the GPU's tensors held before
it, with that call's tolerance (those of the tests of the single calls).
"""
import numpy as np
import pytest

import latent_util as L
import paper_2603_01639_amd as ltd
from test_gpu_latent_attention import tolerance

pytestmark = pytest.mark.gpu

DL, D = 512, 512 + L.ROPE
SCALE = 192 ** -0.5


def f64(t):
    return t.double().cpu().numpy()


def random_tree(rng, n, room):
    """Parents [room], depths, and an accepted path of a tree of n nodes."""
    par, dep = np.full(room, -1, np.int32), np.zeros(room, np.int32)
    for i in range(1, n):
        par[i] = rng.integers(0, i)
        dep[i] = dep[par[i]] + 1
    leaf = int(rng.integers(0, n))
    path = np.zeros(room, np.int32)
    root = L.root_path(par, leaf)[::-1]
    path[:len(root)] = root
    return par, dep, path, len(root)


class Cycle:
    """Static buffers of a batch, and its cycle's calls."""

    def __init__(self, seed, H, N, prefix, block, dtype="bfloat16", layers=2, room=400, workspace=None):
        import torch
        self.rng = np.random.default_rng(seed)
        self.t = getattr(torch, dtype)
        B = len(prefix)
        self.B, self.N, self.H, self.layers = B, N, H, layers
        pages, table = L.make_table(self.rng, [p + room for p in prefix], block)
        self.np_table = table
        self.cache = torch.from_numpy(self.rng.normal(size=(layers, pages, block, D))).to(self.t).cuda()
        self.table = L.to_dev(table)
        self.freq, self.m = ltd.rope_frequencies(L.ROPE, 10000.0, scaling="yarn", factor=4.0, trained_len=4096, device="cuda")
        self.w = torch.from_numpy(1 + 0.2 * self.rng.normal(size=DL)).to(self.t).cuda()
        i = lambda *s: torch.zeros(s, dtype=torch.int32, device="cuda")  # noqa: E731
        self.prefix, self.new, self.n, self.nacc = L.to_dev(np.array(prefix, np.int32)), i(B), i(B), i(B)
        self.par, self.dep, self.path = i(B, N), i(B, N), i(B, N)
        self.q = torch.zeros((layers, B, N, H, D), dtype=self.t, device="cuda")
        self.kv = torch.zeros((layers, B, N, D + 64), dtype=self.t, device="cuda")
        self.out = torch.zeros((layers, B, N, H, DL), dtype=self.t, device="cuda")
        self.most = max(prefix) + room
        size = ltd.attn_latent_workspace_size(B, N, H, DL, L.ROPE, self.most, ltd._dtype_code(self.q))
        self.ws = torch.empty(max(size, 16), dtype=torch.uint8, device="cuda") if workspace is None else workspace

    def draw(self, sizes=None):
        """New trees, queries and rows."""
        import torch
        sizes = self.rng.integers(1, self.N + 1, self.B) if sizes is None else np.array(sizes)
        trees = [random_tree(self.rng, int(n), self.N) for n in sizes]
        for dst, src in ((self.par, 0), (self.dep, 1), (self.path, 2)):
            dst.copy_(torch.from_numpy(np.stack([t[src] for t in trees])))
        self.nacc.copy_(torch.tensor([t[3] for t in trees], dtype=torch.int32))
        self.n.copy_(torch.from_numpy(sizes.astype(np.int32)))
        for x in (self.q, self.kv):
            x.copy_(torch.from_numpy(self.rng.normal(size=x.shape)))

    def rope(self, layer):
        q = self.q[layer]
        ltd.tree_rope(q, q, self.freq, self.prefix, self.n, depth=self.dep, rot_offset=DL, interleaved=True, mscale=self.m)

    def append(self, layer):
        ltd.latent_append(self.kv[layer, :, :, 32:32 + D], self.cache[layer], self.freq, self.prefix, self.n, depth=self.dep,
                          norm_weight=self.w, norm_eps=1e-6, interleaved=True, mscale=self.m, block_table=self.table,
                          num_blocks=self.cache.shape[1])

    def attend(self, layer):
        q = self.q[layer]
        ltd.tree_verify_attn_latent(q[..., :DL], q[..., DL:], self.cache[layer], self.prefix, self.par, self.n, self.out[layer],
                                    max_prefix=self.most, scale=SCALE, block_table=self.table, num_blocks=self.cache.shape[1],
                                    workspace=self.ws)

    def finish(self):
        ltd.latent_compact(self.cache, self.prefix, self.new, self.path, self.nacc, block_table=self.table,
                           num_blocks=self.cache.shape[1])
        self.prefix.copy_(self.new)

    def step(self):
        for layer in range(self.layers):
            self.rope(layer)
            self.append(layer)
            self.attend(layer)
        self.finish()


@pytest.mark.parametrize("dtype", ["bfloat16", "float32"])
@pytest.mark.parametrize("H, N, prefix, block", [(16, 12, [0, 37, 300], 16), (16, 1, [5, 0, 64, 1000], 64), (4, 4, [90, 15], 8),
                                                 (40, 70, [130], 32)])
def test_cycles(H, N, prefix, block, dtype):
    import torch
    c = Cycle(sum(prefix) + H, H, N, prefix, block, dtype)
    h, bf16 = L.half_step(c.t), dtype == "bfloat16"
    freq = f64(c.freq)
    for _ in range(3):
        c.draw()
        P, n, par, dep = (x.cpu().numpy() for x in (c.prefix, c.n, c.par, c.dep))
        live = np.arange(N) < n[:, None]
        pos = P[:, None].astype(np.int64) + dep
        for layer in range(c.layers):
            q0, cache0 = f64(c.q[layer]), f64(c.cache[layer])
            c.rope(layer)
            q1 = f64(c.q[layer])
            part = q0[..., DL:]
            want = L.turn(part, np.repeat(pos[..., None], H, 2), freq, True, c.m)
            pair = np.repeat(np.abs(part).reshape(*part.shape[:-1], -1, 2).max(-1), 2, -1)
            tol = 1.01 * h * np.abs(want) + 12 * 2.0 ** -24 * pair * c.m
            assert (np.abs(q1[..., DL:] - want) <= tol)[live].all()
            assert (q1[..., :DL] == q0[..., :DL]).all() and (q1[~live] == q0[~live]).all()

            c.append(layer)
            cache1, want, tol = f64(c.cache[layer]), cache0.copy(), np.zeros_like(cache0)
            x = f64(c.kv[layer, :, :, 32:32 + D])
            for b in range(c.B):
                for i in range(n[b]):
                    page, r = L.place(c.np_table, b, int(P[b]) + i, block)
                    lat = x[b, i, :DL] / np.sqrt((x[b, i, :DL] ** 2).mean() + 1e-6) * f64(c.w)
                    part = x[b, i, DL:]
                    rot = L.turn(part, np.int64(pos[b, i]), freq, True, c.m)
                    pair = np.repeat(np.abs(part).reshape(-1, 2).max(-1), 2)
                    want[page, r] = np.r_[lat, rot]
                    tol[page, r] = np.r_[1.01 * (h + 15 * 2.0 ** -24) * np.abs(lat),
                                         1.01 * h * np.abs(rot) + 12 * 2.0 ** -24 * pair * c.m]
            assert (np.abs(cache1 - want) <= tol).all()

            before = c.out[layer].clone()
            c.attend(layer)
            got = f64(c.out[layer])
            o, A, S = L.attention(q1[..., :DL], q1[..., DL:], cache1, c.np_table, P, par, n, SCALE)
            for b in range(c.B):
                tol = tolerance(bf16, o[b, :n[b]], A[b, :n[b]], S[b, :n[b]], int(P[b] + n[b]), D)
                assert (np.abs(got[b, :n[b]] - o[b, :n[b]]) <= tol).all()
            assert torch.equal(c.out[layer][torch.from_numpy(~live)], before[torch.from_numpy(~live)])
        path, nacc, was = c.path.cpu().numpy(), c.nacc.cpu().numpy(), c.cache.clone()
        c.finish()
        for b in range(c.B):
            for j in range(nacc[b]):
                sp, sr = L.place(c.np_table, b, int(P[b]) + int(path[b, j]), block)
                dp, dr = L.place(c.np_table, b, int(P[b]) + j, block)
                was[:, dp, dr] = was[:, sp, sr].clone()  # (earlier moves wrote only rows before this one)
        assert torch.equal(c.cache, was)
        assert (c.prefix.cpu().numpy() == P + nacc).all()


def capture(step):
    import torch
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.stream(side):
        step()  # (loads the kernels)
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        step()
    torch.cuda.synchronize()
    return graph


def state(c):
    return [c.cache, c.prefix, c.new, c.q, c.out]


@pytest.mark.parametrize("dtype", ["bfloat16", "float32"])
@pytest.mark.parametrize("H, N, prefix", [(16, 1, [3, 900, 64]), (16, 12, [0, 37, 500])])
def test_captured_cycles(H, N, prefix, dtype):
    """Replays over lengths, trees and tokens that change, with eager cycles of the same inputs between."""
    import torch
    c = Cycle(5, H, N, prefix, 16, dtype)
    c.draw()
    keep = [x.clone() for x in state(c)]
    graph = capture(c.step)
    for x, k in zip(state(c), keep):
        x.copy_(k)
    for r in range(6):
        c.draw(None if r else [1] * c.B)
        keep = [x.clone() for x in state(c)]
        graph.replay()
        torch.cuda.synchronize()
        got = [x.clone() for x in state(c)]
        for x, k in zip(state(c), keep):
            x.copy_(k)
        c.step()
        torch.cuda.synchronize()
        for name, x, g in zip(("cache", "prefix", "new", "q", "out"), state(c), got):
            assert torch.equal(x, g), f"replay {r}: {name}"


def test_two_graphs_share_a_workspace():
    """A graph of single tokens and one of trees with one workspace, replayed in turn, and eager calls with it between."""
    import torch
    tree = Cycle(6, 16, 40, [100, 700, 5], 32, layers=1)
    token = Cycle(7, 16, 1, [2000, 40, 1, 300], 64, layers=1, workspace=tree.ws)
    need = ltd.attn_latent_workspace_size(4, 1, 16, DL, L.ROPE, token.most, ltd.DTYPE_BF16)
    if need > tree.ws.numel():
        tree.ws = token.ws = torch.empty(need, dtype=torch.uint8, device="cuda")
    for c in (tree, token):
        c.draw()
    keep = {c: [x.clone() for x in state(c)] for c in (tree, token)}
    graphs = {c: capture(c.step) for c in (tree, token)}
    for c in (tree, token):
        for x, k in zip(state(c), keep[c]):
            x.copy_(k)
    for r in range(4):
        for c in (token, tree):
            c.draw()
        want = {}
        for c in (tree, token):
            was = [x.clone() for x in state(c)]
            c.step()
            want[c] = [x.clone() for x in state(c)]
            for x, k in zip(state(c), was):
                x.copy_(k)
        for c in (tree, token) if r % 2 else (token, tree):
            graphs[c].replay()
        torch.cuda.synchronize()
        for c in (tree, token):
            for x, k in zip(state(c), want[c]):
                assert torch.equal(x, k), r


def test_cycles_on_two_streams():
    """Two batches' cycles at once, each on a stream and with a workspace of its own."""
    import torch
    a, b = Cycle(8, 16, 20, [500, 3], 16), Cycle(9, 16, 1, [30, 1500, 700], 64)
    for c in (a, b):
        c.draw()
    want = {}
    for c in (a, b):
        was = [x.clone() for x in state(c)]
        c.step()
        want[c] = [x.clone() for x in state(c)]
        for x, k in zip(state(c), was):
            x.copy_(k)
    streams = {a: torch.cuda.Stream(), b: torch.cuda.Stream()}
    torch.cuda.synchronize()
    for c in (a, b):
        with torch.cuda.stream(streams[c]):
            c.step()
    torch.cuda.synchronize()
    for c in (a, b):
        for x, k in zip(state(c), want[c]):
            assert torch.equal(x, k)
