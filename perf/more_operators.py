"""Rotary positions and the latent-attention cycle of a decoder, as cases that can be timed and checked.

A decoder rotates its queries and keys by their positions (`tree_rope`; a draft tree's node stands at its depth
behind the prefix).  A model with latent attention keeps, for every token, one vector that all heads share: a
compressed part of `dl` dims, which serves as key and value, and a rotated part of `dr` dims, which serves as key
alone.  `latent_append` normalises, rotates and writes a prompt's or a draft tree's rows, `tree_verify_attn_latent`
attends in the absorbed form (queries already multiplied into the latent space) under the tree's mask, and
`latent_compact` moves the accepted rows.

With `own` false every operator is computed in its plain form from elementary torch operations, in float32 (the
angles in float64).  All inputs are synthetic and made on the GPU from the seed.
"""
import math

import numpy as np
import torch

own = False

H_8B = dict(Hq=32, Hk=8, d=128)
H_32B = dict(Hq=64, Hk=8, d=128)  # also 70B-shaped
H_13B = dict(Hq=40, Hk=40, d=128)  # no grouped queries
H_D64 = dict(Hq=32, Hk=8, d=64)
H_TINY = dict(Hq=8, Hk=8, d=64)
LATENT = dict(dl=512, dr=64)
LATENT_SMALL = dict(dl=256, dr=64)


def _rope_case(name, heads, B, P, N, tree, r, inter, scaling, dtype="bf16"):
    """Prefixes and row counts spread over P and N (ends included) across the batch; tree: rows are a draft tree's
    nodes, else consecutive tokens; the first r dims rotate, in neighbouring pairs (inter) or halves."""
    c = dict(op="rope", dtype=dtype, B=B, P0=P[0], P1=P[1], N0=N[0], N1=N[1], tree=tree, r=r, inter=inter,
             scaling=scaling, **heads)
    return dict(name=name, **c) if name else c


def _cache_case(name, op, dims, B, P, N, block, dtype="bf16", **more):
    """block = rows per block of a paged cache, 0 for a contiguous one."""
    c = dict(op=op, dtype=dtype, B=B, P0=P[0], P1=P[1], N0=N[0], N1=N[1], block=block, **dims, **more)
    return dict(name=name, **c) if name else c


def listed():
    return [
        # One layer's queries and keys of one user's draft tree, 8B-shaped: the smallest call.
        _rope_case("rope_tree_8b", H_8B, 1, (2041, 2041), (60, 60), True, 128, False, "none"),
        # One layer's of a batch of prompts, 70B-shaped.
        _rope_case("rope_prompts_70b_b8", H_32B, 8, (0, 0), (1024, 8192), False, 128, False, "none"),
        # A serving batch's trees in a model that rotates half of each head, scaled for contexts of a million tokens.
        _rope_case("rope_tree_far_partial_b16", H_32B, 16, (900000, 1040000), (16, 128), True, 64, True, "yarn"),
        # One layer's write of one user's draft tree behind an odd prefix.
        _cache_case("latent_append_tree", "append", LATENT, 1, (2041, 2041), (60, 60), 0, inter=True, norm=True),
        # One layer's write of a batch of prompts into a paged cache.
        _cache_case("latent_append_prompts_b16", "append", LATENT, 16, (0, 0), (1024, 8192), 64, inter=True, norm=True),
        # The correctness setting: float32, a tiny model.
        _cache_case("latent_attn_f32_tiny", "attn", LATENT_SMALL, 1, (128, 128), (16, 16), 0, "f32", Hq=8),
        # Plain decoding of a serving batch, one token a sequence: one GPU's 16 heads of 128 under 8-way tensor
        # parallelism, paged.
        _cache_case("latent_decode_h16_b16", "attn", LATENT, 16, (1024, 8192), (1, 1), 64, Hq=16),
        # The same with all 128 heads on the GPU (data-parallel attention).
        _cache_case("latent_decode_h128_b16", "attn", LATENT, 16, (1024, 8192), (1, 1), 64, Hq=128),
        # One user's tree behind a long prefix.
        _cache_case("latent_attn_h16_p16384_n60", "attn", LATENT, 1, (16384, 16384), (60, 60), 0, Hq=16),
        # Verification of a serving batch with all heads on the GPU: the largest call.
        _cache_case("latent_attn_h128_b8", "attn", LATENT, 8, (1024, 8192), (16, 96), 64, Hq=128),
        # All 60 layers' compaction after one user's cycle.
        _cache_case("latent_compact_60layers", "compact", LATENT, 1, (2041, 2041), (128, 128), 0, layers=60, acc=6),
        # A serving batch's on a pipeline stage of 20 layers.
        _cache_case("latent_compact_b16", "compact", LATENT, 16, (500, 1500), (64, 128), 64, layers=20, acc=8),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    """One more case of the listed ones' ranges."""
    op = rng.choice(["rope", "rope", "append", "attn", "attn", "attn", "attn", "compact"])
    block = rng.choice([0, 0, 16, 64, 64, 1, 48, 128])
    B = rng.choice([1, 1, 2, 3, 5, 8, 13, 16])
    if op == "rope":
        heads = rng.choice([H_8B, H_32B, H_13B, H_D64, H_TINY])
        r = rng.choice([heads["d"], heads["d"], heads["d"] // 2, 32, 36])
        tree = rng.random() < 0.6
        P = _log_int(rng, 1, 1000000)
        N = _log_int(rng, 1, 256) if tree else _log_int(rng, 64, 4096)
        return _rope_case("", heads, B, (P, P + rng.randint(0, P // 8)), (max(1, N // 2), N), tree, r,
                          rng.random() < 0.5, rng.choice(["none", "none", "linear", "yarn"]),
                          rng.choice(["bf16", "bf16", "f32"]))
    dims = rng.choice([LATENT, LATENT, LATENT_SMALL])
    if op == "append":
        if rng.random() < 0.5:  # a tree's rows
            P, N = _log_int(rng, 1, 8192), _log_int(rng, 1, 256)
        else:  # a prompt's, from the start or behind a shared prefix
            P, N = rng.choice([0, _log_int(rng, 1, 2048)]), _log_int(rng, 64, 4096)
        return _cache_case("", op, dims, B, (P, P + rng.randint(0, P)), (max(1, N // 2), N), block,
                           rng.choice(["bf16", "bf16", "f32"]), inter=rng.random() < 0.5, norm=rng.random() < 0.7)
    if op == "attn":
        if rng.random() < 0.15:
            P, N = _log_int(rng, 1, 1024), _log_int(rng, 1, 64)
            return _cache_case("", op, dims, rng.randint(1, 2), (P, P), (N, N), block, "f32", Hq=rng.choice([1, 5, 8]))
        Hq = rng.choice([8, 16, 16, 24, 32, 64, 128])
        P, N = _log_int(rng, 16, 16384 if B == 1 else 4096), rng.choice([1, _log_int(rng, 1, 256)])
        P1 = P if B == 1 else min(8192, 2 * P)
        N = max(1, min(N, 600000000 // (B * Hq * (P1 + 256))))
        return _cache_case("", op, dims, B, (P, P1), (max(1, N // 2), N), block, Hq=Hq)
    P, N, acc = _log_int(rng, 1, 1500), rng.randint(32, 256), rng.randint(1, 12)
    return _cache_case("", op, dims, B, (P, 2 * P), (32, N), block, rng.choice(["bf16", "f32"]),
                       layers=_log_int(rng, 1, 24), acc=acc)


# ------------------------------------------------------------------ inputs

def _beam_tree(r, n):
    """Parents of a draft tree of n nodes, listed level by level: each level's nodes hang from a few of the last's."""
    par, level = [-1], [0]
    while len(par) < n:
        width = min(n - len(par), int(r.integers(4, 17)))
        up = sorted(int(x) for x in r.choice(level, size=width))
        level = list(range(len(par), len(par) + width))
        par += up
    return par


def _ragged(r, lo, hi, B):
    """B sizes spread evenly over [lo, hi], odd ones among them (the same ones for every seed, so that every pass is
    the same work), in the seed's order."""
    return [int(lo + (hi - lo) * (i + 0.5) / B) if B > 1 else hi for i in r.permutation(B)]


def _sizes(case, r):
    return _ragged(r, case["P0"], case["P1"], case["B"]), _ragged(r, case["N0"], case["N1"], case["B"])


def _trees(r, ns):
    """Parents and depths [B][Nmax]."""
    par = np.full((len(ns), max(ns)), -1, np.int32)
    dep = np.zeros((len(ns), max(ns)), np.int32)
    for b, n in enumerate(ns):
        par[b, :n] = _beam_tree(r, n)
        for i in range(1, n):
            dep[b, i] = dep[b, par[b, i]] + 1
    return par, dep


def _frequencies(r, scaling):
    """Angles a position of each of the r / 2 pairs, and what the rotated values are multiplied by."""
    f = 500000.0 ** (-2.0 * np.arange(r // 2) / r)
    if scaling == "none":
        return f, 1.0
    s, trained = 32.0, 32768.0
    if scaling == "linear":
        return f / s, 1.0
    # pairs that turn often within the trained context keep their speed, slow ones are slowed down, a ramp between
    turns = trained * f / (2 * math.pi)
    at = [r * math.log(trained / (t * 2 * math.pi)) / (2 * math.log(500000.0)) for t in (32.0, 1.0)]
    lo, hi = max(math.floor(at[0]), 0), min(math.ceil(at[1]), r - 1)
    slow = np.clip((np.arange(len(turns)) - lo) / max(hi - lo, 1e-3), 0, 1)
    return f * (1 - slow) + f / s * slow, 0.1 * math.log(s) + 1.0


def _gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed * 7919 + 31)
    return g


def _randn(g, shape, dtype=torch.float32, std=1.0):
    return (torch.randn(shape, generator=g, device="cuda", dtype=torch.float32) * std).to(dtype)


def _i32(a):
    return torch.as_tensor(np.asarray(a, np.int32), device="cuda")


def _pages(s, r, block):
    """The block table of a paged cache (as many blocks whichever prefix and tree meet)."""
    per = [-(-(p + n) // block) for p, n in zip(s["P"], s["ns"])]
    s["blocks"] = sum(-(-x // block) for x in s["P"] + s["ns"])
    perm = r.permutation(s["blocks"]).astype(np.int32)
    table = np.zeros((len(per), max(per)), np.int32)
    at = 0
    for b, n in enumerate(per):
        table[b, :n] = perm[at:at + n]
        at += n
    s["table"] = _i32(table)


def prepare(case, seed):
    r, g = np.random.default_rng(seed), _gen(seed)
    B, op = case["B"], case["op"]
    dtype = torch.bfloat16 if case["dtype"] == "bf16" else torch.float32
    P, ns = _sizes(case, r)
    nmax = max(ns)
    s = dict(op=op, B=B, P=P, ns=ns, nmax=nmax, prefix=_i32(P), n=_i32(ns), max_prefix=max(P), table=None, blocks=0,
             depth=None, inter=case.get("inter", False))
    par, dep = _trees(r, ns) if nmax <= 256 else (None, None)
    if op == "rope":
        Hq, Hk, d = case["Hq"], case["Hk"], case["d"]
        if case["tree"]:
            s["depth"] = _i32(dep)
        f, s["m"] = _frequencies(case["r"], case["scaling"])
        s["freq"] = torch.as_tensor(f, device="cuda")
        # queries and keys are views into the fused projection's output
        qkv = _randn(g, (B, nmax, (Hq + 2 * Hk) * d), dtype)
        s["q"] = qkv[:, :, :Hq * d].view(B, nmax, Hq, d)
        s["k"] = qkv[:, :, Hq * d:(Hq + Hk) * d].view(B, nmax, Hk, d)
        s["q_out"] = torch.zeros((B, nmax, Hq, d), dtype=dtype, device="cuda")
        s["k_out"] = torch.zeros((B, nmax, Hk, d), dtype=dtype, device="cuda")
        return s
    dl, dr, bs, L = case["dl"], case["dr"], case["block"], case.get("layers", 1)
    s["dl"], s["layers"] = dl, L
    if bs:
        _pages(s, r, bs)
        shape = (L, s["blocks"], bs, dl + dr)
    else:
        shape = (L, B, -(-(max(P) + nmax) // 64) * 64, dl + dr)
    s["cache"] = torch.empty(shape, dtype=dtype, device="cuda")
    for x in range(L):
        s["cache"][x] = _randn(g, shape[1:])
    # the (sequence, row) pairs of the call, as a host program that knows its lengths lists them
    s["rb"] = torch.as_tensor(np.repeat(np.arange(B), ns), device="cuda")
    s["ri"] = torch.as_tensor(np.concatenate([np.arange(n) for n in ns]), device="cuda")
    if op == "append":
        if nmax <= 256:
            s["depth"] = _i32(dep)
        f, s["m"] = _frequencies(dr, "none")
        s["freq"] = torch.as_tensor(f, device="cuda")
        # the last columns of the fused down projection's output
        down = _randn(g, (B, nmax, 1024 + dl + dr), dtype, 0.7)
        s["new"] = down[:, :, 1024:]
        s["w"] = (1 + 0.1 * _randn(g, (dl,))).to(dtype) if case["norm"] else None
    elif op == "attn":
        s["parents"] = _i32(par)
        # the latent part comes out of a product per head ([heads][tokens][dl]), the rotated part beside it
        s["q"] = _randn(g, (case["Hq"], B, nmax, dl), dtype, 1.5).permute(1, 2, 0, 3)
        s["q_rope"] = _randn(g, (B, nmax, case["Hq"], dr), dtype, 1.5)
        s["out"] = torch.zeros((B, nmax, case["Hq"], dl), dtype=dtype, device="cuda")
        s["scale"] = (128 + dr) ** -0.5
    else:
        # accepted nodes behind the rows that are written, so that a pass can be repeated on its own result
        path, nacc = np.zeros((B, nmax), np.int32), []
        for b, n in enumerate(ns):
            k = max(1, min(case["acc"], n - case["acc"]))
            path[b, 1:k] = np.sort(r.choice(np.arange(case["acc"], n), size=k - 1, replace=False)) if k > 1 else 0
            nacc.append(k)
        s["acc"], s["nacc"] = _i32(path), _i32(nacc)
        s["new_len"] = torch.zeros(B, dtype=torch.int32, device="cuda")
        s["kb"] = torch.as_tensor(np.repeat(np.arange(B), nacc), device="cuda")
        s["kj"] = torch.as_tensor(np.concatenate([np.arange(k) for k in nacc]), device="cuda")
    return s


# ---------------------------------------------------------------- plain forms

def _place(s, b, r):
    """Page and row in the page of logical rows r of sequences b."""
    if s["table"] is None:
        return b, r
    R = s["cache"].shape[2]
    return s["table"][b, r // R].long(), r % R


def _positions(s):
    node = torch.arange(s["nmax"], device="cuda") if s["depth"] is None else s["depth"].long()
    return s["prefix"].long()[:, None] + node


def _turn(x, cos, sin, inter):
    """Pairs of x's last dim turned; cos and sin carry the factor."""
    if inter:
        a, b = x[..., 0::2], x[..., 1::2]
        return torch.stack((a * cos - b * sin, b * cos + a * sin), -1).flatten(-2)
    a, b = x.chunk(2, -1)
    return torch.cat((a * cos - b * sin, b * cos + a * sin), -1)


def _plain_rope(s):
    angle = _positions(s).double()[..., None] * s["freq"]
    cos, sin = (angle.cos() * s["m"]).float()[:, :, None], (angle.sin() * s["m"]).float()[:, :, None]
    r = 2 * s["freq"].numel()
    there = (torch.arange(s["nmax"], device="cuda") < s["n"][:, None])[:, :, None, None]
    out = []
    for k in ("q", "k"):
        x = s[k].float()
        y = torch.cat((_turn(x[..., :r], cos, sin, s["inter"]), x[..., r:]), -1)
        out.append(torch.where(there, y.to(s[k].dtype), s[k + "_out"]))
    return out


def _plain_append(s):
    b, i, dl = s["rb"], s["ri"], s["dl"]
    x = s["new"][b, i].float()
    c = x[:, :dl]
    if s["w"] is not None:
        c = c * torch.rsqrt((c * c).mean(-1, keepdim=True) + 1e-6) * s["w"].float()
    angle = _positions(s).expand(s["B"], s["nmax"])[b, i].double()[:, None] * s["freq"]
    k = _turn(x[:, dl:], (angle.cos() * s["m"]).float(), (angle.sin() * s["m"]).float(), s["inter"])
    page, w = _place(s, b, s["prefix"].long()[b] + i)
    s["cache"][0][page, w] = torch.cat((c, k), -1).to(s["cache"].dtype)
    return s["cache"][0]


def _root_paths(s):
    """[B][Nmax][Nmax]: whether node j is on node i's root path (i among them), by doubling the links."""
    nmax = s["nmax"]
    node = torch.arange(nmax, device="cuda")
    link = (s["parents"].long()[:, :, None] == node) | (node[:, None] == node)
    link = (link & (node < s["n"][:, None])[:, :, None]).float()
    for _ in range(max(1, (nmax - 1).bit_length())):
        link = (torch.matmul(link, link) > 0).float()
    return link > 0


def _plain_attn(s):
    B, nmax, Hq, dl = s["q"].shape
    pre = s["prefix"].long()
    T = s["max_prefix"] + nmax
    last = torch.as_tensor([p + n - 1 for p, n in zip(s["P"], s["ns"])], device="cuda")
    t = torch.arange(T, device="cuda")
    page, w = _place(s, torch.arange(B, device="cuda")[:, None], torch.minimum(t, last[:, None]))
    k = s["cache"][0][page, w].float()  # [B, T, dl + dr]
    rel = t - pre[:, None]
    sees = torch.gather(_root_paths(s), 2, rel.clamp(0, nmax - 1)[:, None, :].expand(B, nmax, T))
    sees = ((rel < 0)[:, None, :] | (sees & (rel < s["n"][:, None])[:, None, :]))
    rows = torch.cat((s["q"].float(), s["q_rope"].float()), -1).reshape(B, nmax * Hq, -1)
    x = torch.matmul(rows, k.transpose(1, 2).contiguous()).view(B, nmax, Hq, T) * s["scale"]
    x = x.masked_fill_(~sees[:, :, None], -math.inf)
    x = torch.exp(x - x.amax(-1, keepdim=True))
    x = x / x.sum(-1, keepdim=True)
    o = torch.matmul(x.view(B, -1, T), k[..., :dl].contiguous()).view(B, nmax, Hq, dl)
    there = (torch.arange(nmax, device="cuda") < s["n"][:, None])[:, :, None, None]
    return torch.where(there, o.to(s["q"].dtype), s["out"])


def _plain_compact(s):
    b, j = s["kb"], s["kj"]
    pre = s["prefix"].long()[b]
    sp, sw = _place(s, b, pre + s["acc"][b, j].long())
    dp, dw = _place(s, b, pre + j)
    s["cache"][:, dp, dw] = s["cache"][:, sp, sw]
    s["new_len"].copy_(s["prefix"] + s["nacc"])
    return [s["cache"], s["new_len"]]


# ---------------------------------------------------------------- the calls

def _own(s):
    import paper_2603_01639_amd as ltd
    op = s["op"]
    if op == "rope":
        ltd.tree_rope(s["q"], s["q_out"], s["freq"], s["prefix"], s["n"], k=s["k"], k_out=s["k_out"], depth=s["depth"],
                      interleaved=s["inter"], mscale=s["m"])
        return [s["q_out"], s["k_out"]]
    paged = dict(block_table=s["table"], num_blocks=s["blocks"])
    if op == "append":
        ltd.latent_append(s["new"], s["cache"][0], s["freq"], s["prefix"], s["n"], depth=s["depth"], norm_weight=s["w"],
                          norm_eps=1e-6, interleaved=s["inter"], mscale=s["m"], **paged)
        return s["cache"][0]
    if op == "attn":
        if "ws" not in s:
            B, nmax, Hq, dl = s["q"].shape
            size = ltd.attn_latent_workspace_size(B, nmax, Hq, dl, s["q_rope"].shape[3], s["max_prefix"],
                                                  ltd.DTYPE_BF16 if s["q"].dtype == torch.bfloat16 else ltd.DTYPE_F32)
            s["ws"] = torch.empty(max(1, size), dtype=torch.uint8, device="cuda")
        return ltd.tree_verify_attn_latent(s["q"], s["q_rope"], s["cache"][0], s["prefix"], s["parents"], s["n"],
                                           s["out"], max_prefix=s["max_prefix"], scale=s["scale"], workspace=s["ws"],
                                           **paged)
    ltd.latent_compact(s["cache"], s["prefix"], s["new_len"], s["acc"], s["nacc"], **paged)
    return [s["cache"], s["new_len"]]


_PLAIN = dict(rope=_plain_rope, append=_plain_append, attn=_plain_attn, compact=_plain_compact)


def run(s):
    return _own(s) if own else _PLAIN[s["op"]](s)


# ---------------------------------------------------------------- the work

def work(case):
    P, ns = _sizes(case, np.random.default_rng(0))
    op, e, B = case["op"], 2 if case["dtype"] == "bf16" else 4, case["B"]
    if op == "rope":
        elems = sum(ns) * (case["Hq"] + case["Hk"])
        return {"bytes": 2 * elems * case["d"] * e + 4 * sum(ns), "flops": 3.0 * elems * case["r"]}
    D = case["dl"] + case["dr"]
    if op == "append":
        return {"bytes": 2 * sum(ns) * D * e, "flops": sum(ns) * (4.0 * case["dl"] + 3 * case["dr"])}
    if op == "compact":
        return {"bytes": case["layers"] * 2 * B * max(1, case["acc"]) * D * e + 16 * B, "flops": 0}
    cache = sum(p + n for p, n in zip(P, ns)) * D * e
    return {"bytes": cache + sum(ns) * case["Hq"] * (D + case["dl"]) * e,
            "flops": sum(2.0 * case["Hq"] * n * p * (D + case["dl"]) for p, n in zip(P, ns))}


# ---------------------------------------------------------------- in 64 bits

def _exact_rows(s, b):
    """The cache rows (pages, rows in them) of sequence b's logical rows."""
    t = np.arange(s["P"][b] + s["ns"][b])
    if s["table"] is None:
        return torch.full((len(t),), b, device="cuda"), torch.as_tensor(t, device="cuda")
    R = s["cache"].shape[2]
    return (torch.as_tensor(s["table"].cpu().numpy()[b, t // R], device="cuda").long(),
            torch.as_tensor(t % R, device="cuda"))


def _exact_turned(s, x, b, r):
    """x [rows, ..., d] of sequence b with its first r dims turned, as products of complex numbers."""
    n = s["ns"][b]
    node = torch.arange(n, device="cuda") if s["depth"] is None else s["depth"][b, :n]
    angle = (node.double() + s["P"][b]).view([n] + [1] * (x.dim() - 1)) * s["freq"]
    first, second = (slice(0, r, 2), slice(1, r, 2)) if s["inter"] else (slice(0, r // 2), slice(r // 2, r))
    z = torch.complex(x[..., first], x[..., second]) * torch.polar(torch.full_like(angle, s["m"]), angle)
    y = x.clone()
    y[..., first], y[..., second] = z.real, z.imag
    return y


def exact(case, seed):
    s = prepare(case, seed)
    op = case["op"]
    if op == "rope":
        out = []
        for k in ("q", "k"):
            y = s[k + "_out"].double()
            for b, n in enumerate(s["ns"]):
                y[b, :n] = _exact_turned(s, s[k][b, :n].double(), b, case["r"])
            out.append(y)
        return out
    if op == "append":
        y = s["cache"][0].double()
        for b, n in enumerate(s["ns"]):
            x = s["new"][b, :n].double()
            c = x[:, :case["dl"]]
            if s["w"] is not None:
                c = c / torch.sqrt(c.pow(2).sum(-1, keepdim=True) / case["dl"] + 1e-6) * s["w"].double()
            page, w = _exact_rows(s, b)
            y[page[-n:], w[-n:]] = torch.cat((c, _exact_turned(s, x[:, case["dl"]:], b, case["dr"])), 1)
        return y
    if op == "compact":
        y = s["cache"].double()
        for b, P in enumerate(s["P"]):
            page, w = _exact_rows(s, b)
            src = P + s["acc"][b, :int(s["nacc"][b])].long()
            y[:, page[P:P + len(src)], w[P:P + len(src)]] = s["cache"][:, page[src], w[src]].double()
        return [y, None]
    out = s["out"].double()
    par = s["parents"].cpu().numpy()
    for b, (P, n) in enumerate(zip(s["P"], s["ns"])):
        page, w = _exact_rows(s, b)
        rows = s["cache"][0][page, w].double()
        c, k = rows[:, :case["dl"]], rows[:, case["dl"]:]
        hide = np.ones((n, P + n), bool)
        hide[:, :P] = False
        for i in range(n):
            j = i
            while j >= 0:
                hide[i, P + j] = False
                j = int(par[b, j])
        hide = torch.as_tensor(hide, device="cuda")
        for h in range(case["Hq"]):
            x = (s["q"][b, :n, h].double() @ c.T + s["q_rope"][b, :n, h].double() @ k.T) * s["scale"]
            out[b, :n, h] = torch.softmax(x.masked_fill(hide, -math.inf), 1) @ c
    return out
