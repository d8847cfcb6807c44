"""The 8-bit KV cache and the logit processing of a decoding cycle, as cases that can be timed and checked.

A decoder that keeps its KV cache in 8 bits writes each layer's new rows (a prompt's, then every cycle's draft
tree) with `kv_append_q8`, verifies the tree with `tree_verify_attn_q8` and moves the accepted rows with
`kv_compact_q8`.  A cache holds e4m3 values and, for every kv head and block of `scale_rows` rows, one power of
two (a biased exponent byte), for K and V apart; a value stands for code * 2^(byte - 127).  Between the target's
logits and acceptance stand the request's sampling rules: penalties for tokens that occurred (`token_counts`
keeps the table), biases and the grammar's mask, per tree node, as each node's own root path counts.
`tree_process_logits` writes the processed logits (what sampling acceptance reads); `tree_accept_processed` takes
the greedy decision on them without writing them.

With `own` false every operator is computed in its plain form from elementary torch operations, in float32.
All inputs are synthetic and made on the GPU from the seed.
"""
import math

import numpy as np
import torch

own = False

H_8B = dict(Hq=32, Hkv=8, d=128)
H_32B = dict(Hq=64, Hkv=8, d=128)  # also 70B-shaped
H_TP8 = dict(Hq=8, Hkv=1, d=128)  # 70B-shaped, one GPU's share under 8-way tensor parallelism
H_14B = dict(Hq=40, Hkv=8, d=128)
H_13B = dict(Hq=40, Hkv=40, d=128)  # no grouped queries
H_D64 = dict(Hq=32, Hkv=8, d=64)
H_TINY = dict(Hq=8, Hkv=8, d=64)
E_MIN, E_MAX = 27, 214  # the exponent bytes that a write chooses from
MIN32 = -(1 << 31)


def _cache_case(name, op, heads, B, P, N, block, sr, dtype="bf16", **more):
    """Prefixes and row counts spread over P and N (ends included) across the batch; block = rows per block of a
    paged cache, 0 for a contiguous one; sr = rows that share a scale."""
    c = dict(op=op, dtype=dtype, B=B, P0=P[0], P1=P[1], N0=N[0], N1=N[1], block=block, sr=sr, **heads, **more)
    return dict(name=name, **c) if name else c


def _logit_case(name, op, B, N, voc, grammar, prompt, gen, bias):
    """Trees of N nodes (both ends), `grammar`: masks at every node, prompts and outputs of up to `prompt` and
    `gen` tokens so far, up to `bias` biased tokens."""
    c = dict(op=op, B=B, N0=N[0], N1=N[1], voc=voc, grammar=grammar, prompt=prompt, gen=gen, bias=bias)
    return dict(name=name, **c) if name else c


def listed():
    return [
        # One layer's write of one user's draft tree: 60 rows behind an odd prefix, the smallest call.
        _cache_case("append_tree_8b", "append", H_8B, 1, (2041, 2041), (60, 60), 0, 64),
        # One layer's write of a batch of prompts into a paged cache, 70B-shaped.
        _cache_case("append_prompts_70b_b16", "append", H_32B, 16, (0, 0), (1024, 8192), 16, 16),
        # The correctness setting: float32 queries of a tiny model.
        _cache_case("attn_f32_tiny", "attn", H_TINY, 1, (128, 128), (16, 16), 0, 32, "f32"),
        # One user of an 8B-shaped model in long reasoning: a 60-node tree over 16384 tokens.
        _cache_case("attn_8b_p16384_n60", "attn", H_8B, 1, (16384, 16384), (60, 60), 0, 64),
        # Plain decoding of a serving batch, one token a sequence, over a paged cache.
        _cache_case("attn_decode_b16_paged", "attn", H_32B, 16, (1024, 8192), (1, 1), 16, 16),
        # Verification of a serving batch over a paged cache, 70B-shaped, ragged prefixes and trees.
        _cache_case("attn_70b_b16_paged", "attn", H_32B, 16, (1024, 8192), (16, 128), 16, 16),
        # All 32 layers' compaction after one user's cycle.
        _cache_case("compact_8b_32layers", "compact", H_8B, 1, (2041, 2041), (128, 128), 0, 64, layers=32, acc=6),
        # A serving batch's on a pipeline stage of 20 layers.
        _cache_case("compact_70b_b16_paged", "compact", H_32B, 16, (500, 1500), (64, 128), 16, 16, layers=20, acc=8),
        # One user with penalties and a few biases, no grammar; every node's processed logits are wanted.
        _logit_case("process_8b", "process", 1, (60, 60), 128256, False, 2048, 500, 20),
        # A serving batch in which every request answers in a grammar.
        _logit_case("process_b16_grammar", "process", 16, (16, 96), 128256, True, 4096, 1000, 300),
        # The greedy decision of one user's cycle under a grammar.
        _logit_case("accept_8b_grammar", "accept", 1, (60, 60), 128256, True, 2048, 500, 20),
        # The greedy decision of a serving batch with penalties alone.
        _logit_case("accept_b16", "accept", 16, (16, 128), 128256, False, 4096, 1000, 20),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    """One more case of the listed ones' ranges."""
    op = rng.choice(["append", "attn", "attn", "attn", "compact", "process", "accept"])
    heads = rng.choice([H_8B, H_32B, H_TP8, H_14B, H_13B, H_D64])
    block = rng.choice([0, 0, 16, 16, 32, 64, 128, 48])
    sr = rng.choice([s for s in (16, 32, 64, 128) if block % s == 0])
    B = rng.choice([1, 1, 2, 3, 5, 8, 13, 16])
    if op == "append":
        if rng.random() < 0.5:  # a tree's rows
            P, N = _log_int(rng, 1, 8192), _log_int(rng, 1, 256)
        else:  # a prompt's, from the start or behind a shared prefix
            P, N = rng.choice([0, _log_int(rng, 1, 2048)]), _log_int(rng, 64, 4096)
        return _cache_case("", op, heads, B, (P, P + rng.randint(0, P)), (max(1, N // 2), N), block, sr,
                           rng.choice(["bf16", "bf16", "f32"]))
    if op == "attn":
        if rng.random() < 0.15:
            P, N = _log_int(rng, 1, 1024), _log_int(rng, 1, 64)
            return _cache_case("", op, rng.choice([H_TINY, dict(Hq=8, Hkv=2, d=128)]), rng.randint(1, 2), (P, P),
                               (N, N), block, sr, "f32")
        P, N = _log_int(rng, 64, 16384 if B == 1 else 4096), _log_int(rng, 1, 256 if B < 8 else 96)
        return _cache_case("", op, heads, B, (P, P if B == 1 else min(8192, 2 * P)), (max(1, N // 2), N), block, sr)
    if op == "compact":
        P, N, acc = _log_int(rng, 1, 1500), rng.randint(160, 256), rng.randint(1, 12)
        return _cache_case("", op, heads, B, (P, 2 * P), (160, N), block, sr, rng.choice(["bf16", "f32"]),
                           layers=_log_int(rng, 1, 16 if heads["Hkv"] < 40 else 4), acc=acc)
    N = _log_int(rng, 1, 256 if B < 8 else 96)
    return _logit_case("", op, B, (max(1, N // 2), N), rng.choice([32000, 128256, 152064, 50257]),
                       rng.random() < 0.5, _log_int(rng, 16, 16384), _log_int(rng, 1, 4096), rng.choice([0, 20, 300]))


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


def _trees(r, ns, voc):
    """Parents [B][Nmax] and tokens with distinct siblings; one token in eight is its parent's again."""
    B, nmax = len(ns), max(ns)
    par = np.full((B, nmax), -1, np.int32)
    tok = r.integers(0, voc, (B, nmax)).astype(np.int32)
    for b, n in enumerate(ns):
        par[b, :n] = _beam_tree(r, n)
        seen = set()
        for i in range(1, n):
            p = int(par[b, i])
            t = int(tok[b, p]) if r.random() < 0.125 else int(tok[b, i])
            while (p, t) in seen:
                t = int(r.integers(0, voc))
            seen.add((p, t))
            tok[b, i] = t
    return par, tok


def _gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed * 7919 + 29)
    return g


def _randn(g, shape, dtype=torch.float32, std=1.0):
    return (torch.randn(shape, generator=g, device="cuda", dtype=torch.float32) * std).to(dtype)


def _i32(a):
    return torch.as_tensor(np.asarray(a, np.int32), device="cuda")


def _zeros(*shape, dtype=torch.int32):
    return torch.zeros(shape, dtype=dtype, device="cuda")


def _prepare_cache(case, seed):
    r, g = np.random.default_rng(seed), _gen(seed)
    B, Hq, Hkv, d, bs, sr = (case[k] for k in ("B", "Hq", "Hkv", "d", "block", "sr"))
    L, op = case.get("layers", 1), case["op"]
    dtype = torch.bfloat16 if case["dtype"] == "bf16" else torch.float32
    P, ns = _sizes(case, r)
    nmax, rows = max(ns), [p + n for p, n in zip(P, ns)]
    s = dict(op=op, B=B, P=P, ns=ns, nmax=nmax, sr=sr, prefix=_i32(P), n=_i32(ns), max_prefix=max(P), table=None,
             blocks=0, layers=L)
    if bs:
        per = [-(-x // bs) for x in rows]
        s["blocks"] = sum(-(-x // bs) for x in P) + sum(-(-x // bs) for x in ns)
        perm = r.permutation(s["blocks"]).astype(np.int32)
        table = np.zeros((B, max(per)), np.int32)
        at = 0
        for b, n in enumerate(per):
            table[b, :n] = perm[at:at + n]
            at += n
        s["table"] = _i32(table)
        shape = (L, s["blocks"], Hkv, bs, d)
    else:
        shape = (L, B, Hkv, -(-max(rows) // 64) * 64, d)
    # codes of values whose largest in a block is near the format's, and exponents that make them about one unit
    for k in ("k", "v"):
        s[k] = torch.empty(shape, dtype=torch.float8_e4m3fn, device="cuda")
        for x in range(L):
            s[k][x] = _randn(g, shape[1:], std=110.0).clamp_(-448, 448).to(torch.float8_e4m3fn)
        s[k + "s"] = torch.randint(119, 122, (L,) + shape[1:3] + (-(-shape[3] // sr),), generator=g, device="cuda",
                                   dtype=torch.uint8)
    # the (sequence, row) pairs of the call, as a host program that knows its lengths lists them
    s["rb"] = torch.as_tensor(np.repeat(np.arange(B), ns), device="cuda")
    s["ri"] = torch.as_tensor(np.concatenate([np.arange(n) for n in ns]), device="cuda")
    if op == "append":
        # the new rows are views into the fused projection's output; rows, heads and dims differ in size
        qkv = _randn(g, (B, nmax, (Hq + 2 * Hkv) * d), dtype) if nmax <= 256 else _randn(g, (B, nmax, 2 * Hkv * d), dtype)
        qkv *= torch.exp(0.5 * _randn(g, (B, nmax, 1))).to(dtype)
        s["k_new"], s["v_new"] = (qkv[:, :, -(2 - x) * Hkv * d:][:, :, :Hkv * d].view(B, nmax, Hkv, d) for x in (0, 1))
    elif op == "attn":
        par, _ = _trees(r, ns, 1000)
        s["parents"] = _i32(par)
        s["q"] = _randn(g, (B, nmax, Hq, d), dtype, 1.5)
        s["out"] = torch.zeros((B, nmax, Hq, d), dtype=dtype, device="cuda")
    else:
        # accepted nodes behind the blocks that are written, so that a pass can be repeated on its own result
        path, nacc = np.zeros((B, nmax), np.int32), []
        for b, n in enumerate(ns):
            lo = case["acc"] + min(sr, 128 if not bs else bs)
            k = max(1, min(case["acc"], n - lo))
            path[b, 1:k] = np.sort(r.choice(np.arange(lo, n), size=k - 1, replace=False)) if k > 1 else 0
            nacc.append(k)
        s["acc"], s["nacc"], s["new_len"] = _i32(path), _i32(nacc), _zeros(B)
        s["kb"] = torch.as_tensor(np.repeat(np.arange(B), nacc), device="cuda")
        s["kj"] = torch.as_tensor(np.concatenate([np.arange(k) for k in nacc]), device="cuda")
    return s


def _prepare_logits(case, seed):
    r, g = np.random.default_rng(seed), _gen(seed)
    B, voc = case["B"], case["voc"]
    ns = _ragged(r, case["N0"], case["N1"], B)
    par, tok = _trees(r, ns, voc)
    nmax, W = par.shape[1], -(-voc // 32)
    s = dict(op=case["op"], B=B, ns=ns, nmax=nmax, voc=voc, parents=_i32(par), tokens=_i32(tok), n=_i32(ns), mask=None,
             bias=(None, None, None))
    lg = _randn(g, (B, nmax, voc), std=3.0)
    pick = r.integers(0, voc, (B, nmax))
    for b, n in enumerate(ns):
        for u in range(n):
            kids = np.nonzero(par[b, :n] == u)[0]
            if len(kids) and r.random() < 0.7:
                pick[b, u] = tok[b, r.choice(kids)]
    at = torch.as_tensor(pick, device="cuda")[:, :, None]
    s["logits"] = lg.scatter_(2, at, lg.amax(2, keepdim=True) + 4)
    # repetition, frequency and presence penalties; the first request has none
    pen = np.stack([r.uniform(1.0, 1.3, B), r.uniform(-0.2, 0.6, B), r.uniform(-0.2, 0.6, B)], 1).astype(np.float32)
    pen[0] = (1.0, 0.0, 0.0) if B > 1 else pen[0]
    s["pen"] = torch.as_tensor(pen, device="cuda")
    # token frequencies fall off as in text
    for k, most in (("prompt", case["prompt"]), ("gen", case["gen"])):
        n = [most if b == 0 else int(r.integers(0, most + 1)) for b in range(B)]
        s[k] = (voc * torch.rand((B, most), generator=g, device="cuda") ** 4).to(torch.int32).clamp_(max=voc - 1)
        s["n_" + k] = _i32(n)
    if case["bias"]:
        t = np.stack([r.choice(voc, size=case["bias"], replace=False) for _ in range(B)]).astype(np.int32)
        s["bias"] = (_i32(t), _randn(g, t.shape, std=4.0), _i32([int(r.integers(0, case["bias"] + 1)) for _ in range(B)]))
    if case["grammar"]:
        # inside a text most tokens are allowed; between fields a third, or a few; a node off the grammar has none
        keep = torch.as_tensor(np.array([_share(i) for i in range(nmax)]), device="cuda", dtype=torch.float32)
        bits = _zeros(B, nmax, 32 * W, dtype=torch.bool)
        bits[:, :, :voc] = torch.rand((B, nmax, voc), generator=g, device="cuda") < keep[None, :, None]
        bits.scatter_(2, at, keep[None, :, None].expand(B, nmax, 1) > 0)
        two = (1 << torch.arange(32, device="cuda", dtype=torch.int64))
        s["mask"] = (bits.view(B, nmax, W, 32) * two).sum(-1).to(torch.int32)
    s["counts"] = _plain_counts(s)
    if case["op"] == "process":
        s["counts_out"], s["out"] = _zeros(B, voc), _zeros(B, nmax, voc, dtype=torch.float32)
    else:
        s["pred"], s["acc"], s["toks"] = (_zeros(B, nmax) for _ in range(3))
        s["nacc"] = _zeros(B)
    return s


def _share(i):
    """The share of the vocabulary that node i's mask allows."""
    return 0.0 if i % 16 == 15 else (0.98, 0.98, 0.3, 0.98, 0.002)[i % 5]


def prepare(case, seed):
    return (_prepare_cache if case["op"] in ("append", "attn", "compact") else _prepare_logits)(case, seed)


# ---------------------------------------------------------------- plain forms

def _place(s, R, b, r):
    """Page, row in the page and scale of logical rows r of sequences b, for pages of R rows."""
    page = b if s["table"] is None else s["table"][b, r // R].long()
    w = r if s["table"] is None else r % R
    return page, w, w // s["sr"]


def _encode(x):
    return x.clamp(-448, 448).to(torch.float8_e4m3fn).view(torch.uint8)


def _decode(codes):
    return codes.view(torch.float8_e4m3fn).float()


def _needed(amax):
    """The smallest exponent byte under which amax fits the format (448 = 0.875 * 2^9)."""
    m, x = torch.frexp(amax)
    return torch.where(amax > 0, x - 9 + (m > 0.875).int() + 127, E_MIN).clamp(E_MIN, E_MAX).int()


def _plain_append(s):
    pre = s["prefix"].long()
    out = []
    for new, c, sc in ((s["k_new"], s["k"][0], s["ks"][0]), (s["v_new"], s["v"][0], s["vs"][0])):
        codes, (NB, H, R, d), G = c.view(torch.uint8), c.shape, sc.shape[2]
        b = s["rb"]
        page, w, gi = _place(s, R, b, pre[b] + s["ri"])
        x = new[b, s["ri"]].float()
        old = sc.permute(0, 2, 1).reshape(NB * G, H).int()
        amax = torch.zeros((NB * G, H), device="cuda").index_reduce_(0, page * G + gi, x.abs().amax(-1), "amax")
        need = _needed(amax)
        touched, keeps = (torch.zeros(NB * G, dtype=torch.bool, device="cuda") for _ in range(2))
        touched[page * G + gi] = True
        # the block that holds row P keeps the rows before it
        seqs = torch.arange(s["B"], device="cuda")
        p0, w0, g0 = _place(s, R, seqs, pre)
        keeps[(p0 * G + g0)[w0 % s["sr"] != 0]] = True
        e = torch.where(touched[:, None], torch.where(keeps[:, None], torch.maximum(old, need), need), old)
        start = (g0 * s["sr"])[:, None]  # (a short block's list repeats its first row)
        back = torch.maximum((w0 - 1)[:, None] - torch.arange(s["sr"] - 1, device="cuda"), start)
        live = (w0[:, None] > start).expand_as(back)
        pg = p0[:, None].expand_as(back)
        gid = (p0 * G + g0)
        was = codes[pg, :, back]
        shifted = torch.ldexp(_decode(was), (old - e)[gid][:, None, :, None])
        codes[pg, :, back] = torch.where(live[:, :, None, None], _encode(shifted), was)
        codes[page, :, w] = _encode(torch.ldexp(x, (127 - e)[page * G + gi][:, :, None]))
        sc.copy_(e.view(NB, G, H).permute(0, 2, 1).to(torch.uint8))
        out += [c, sc]
    return out


def _plain_compact(s):
    pre = s["prefix"].long()
    b, j = s["kb"], s["kj"]
    out = []
    for c, sc in ((s["k"], s["ks"]), (s["v"], s["vs"])):
        codes, (L, NB, H, R, d), G = c.view(torch.uint8), c.shape, sc.shape[3]
        sp, sw, sg = _place(s, R, b, pre[b] + s["acc"][b, j].long())
        dp, dw, dg = _place(s, R, b, pre[b] + j)
        old = sc.permute(1, 3, 0, 2).reshape(NB * G, L, H).int()
        e_src = old[sp * G + sg]
        val = _decode(codes[:, sp, :, sw])  # [moved, L, H, d]
        gid = dp * G + dg
        touched, keeps = (torch.zeros(NB * G, dtype=torch.bool, device="cuda") for _ in range(2))
        touched[gid] = True
        need = torch.zeros((NB * G, L, H), device="cuda").index_reduce_(0, gid, e_src.float(), "amax").int()
        seqs = torch.arange(s["B"], device="cuda")
        p0, w0, g0 = _place(s, R, seqs, pre)
        first = p0 * G + g0
        keeps[first[w0 % s["sr"] != 0]] = True
        e = torch.where(touched[:, None, None],
                        torch.where(keeps[:, None, None], torch.maximum(old, need), need), old)
        start = (g0 * s["sr"])[:, None]
        back = torch.maximum((w0 - 1)[:, None] - torch.arange(s["sr"] - 1, device="cuda"), start)
        live = (w0[:, None] > start)[:, :, None, None, None]
        pg = p0[:, None].expand_as(back)
        was = codes[:, pg, :, back]  # [B, sr - 1, L, H, d]
        shifted = torch.ldexp(_decode(was), (old - e)[first][:, None, :, :, None])
        codes[:, pg, :, back] = torch.where(live, _encode(shifted), was)
        codes[:, dp, :, dw] = _encode(torch.ldexp(val, (e_src - e[gid])[:, :, :, None]))
        sc.copy_(e.view(NB, G, L, H).permute(2, 0, 3, 1).to(torch.uint8))
        out += [c, sc]
    s["new_len"].copy_(s["prefix"] + s["nacc"])
    return out + [s["new_len"]]


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
    q, B, nmax = s["q"], s["B"], s["nmax"]
    Hq, d = q.shape[2:]
    R, H = s["k"].shape[3], s["k"].shape[2]
    pre = s["prefix"].long()
    T = s["max_prefix"] + nmax
    last = torch.as_tensor([p + n - 1 for p, n in zip(s["P"], s["ns"])], device="cuda")
    t = torch.arange(T, device="cuda")
    page, w, gi = _place(s, R, torch.arange(B, device="cuda")[:, None], torch.minimum(t, last[:, None]))
    k, v = (torch.ldexp(_decode(c[0].view(torch.uint8)[page, :, w]), sc[0][page, :, gi][..., None].int() - 127).transpose(1, 2).contiguous()
            for c, sc in ((s["k"], s["ks"]), (s["v"], s["vs"])))  # [B, H, T, d]
    rel = t - pre[:, None]
    sees = torch.gather(_root_paths(s), 2, rel.clamp(0, nmax - 1)[:, None, :].expand(B, nmax, T))
    sees = ((rel < 0)[:, None, :] | (sees & (rel < s["n"][:, None])[:, None, :]))
    rows = q.float().view(B, nmax, H, Hq // H, d).permute(0, 2, 3, 1, 4).reshape(B, H, -1, d)
    x = torch.matmul(rows, k.transpose(2, 3).contiguous()).view(B, H, Hq // H, nmax, T) * d ** -0.5
    x = x.masked_fill_(~sees[:, None, None], -math.inf)
    x = torch.exp(x - x.amax(-1, keepdim=True))
    x = x / x.sum(-1, keepdim=True)
    o = torch.matmul(x.view(B, H, -1, T), v).view(B, H, Hq // H, nmax, d).permute(0, 3, 1, 2, 4).reshape(B, nmax, Hq, d)
    there = (torch.arange(nmax, device="cuda") < s["n"][:, None])[:, :, None, None]
    return torch.where(there, o.to(q.dtype), s["out"])


def _plain_counts(s):
    B, voc = s["B"], s["voc"]
    there = [torch.arange(s[k].shape[1], device="cuda") < s["n_" + k][:, None] for k in ("prompt", "gen")]
    seen = _zeros(B, voc).scatter_add_(1, s["prompt"].long(), there[0].int()) > 0
    made = _zeros(B, voc).scatter_add_(1, s["gen"].long(), there[1].int())
    return torch.where(seen, made | MIN32, made)


def _plain_process(s, counts):
    B, nmax, voc, x = s["B"], s["nmax"], s["voc"], s["logits"]
    on = _root_paths(s)
    on[:, :, 0] = False  # the root is an emitted token: the table has it
    c = (counts & ~MIN32).float()[:, None, :].repeat(1, nmax, 1)
    c.scatter_add_(2, s["tokens"].long()[:, None, :].expand(B, nmax, nmax), on.float())
    rep, freq, pres = (s["pen"][:, k, None, None] for k in range(3))
    x = torch.where((c > 0) | (counts < 0)[:, None, :], torch.where(x > 0, x / rep, x * rep), x)
    x = torch.where(c > 0, (x - freq * c) - pres, x)
    if s["bias"][0] is not None:
        t, val, n = s["bias"]
        use = torch.arange(t.shape[1], device="cuda") < n[:, None]
        x = x + torch.zeros((B, voc), device="cuda").scatter_add_(1, t.long(), torch.where(use, val, 0.0))[:, None]
    if s["mask"] is not None:
        bits = (s["mask"][..., None] >> torch.arange(32, device="cuda", dtype=torch.int32)) & 1
        x = torch.where(bits.view(B, nmax, -1)[:, :, :voc] > 0, x, -math.inf)
    return x


def _plain_accept(s, x):
    """Greedy acceptance of the processed logits x; entries past the tree or the path stay as they were."""
    B, nmax = s["B"], s["nmax"]
    node = torch.arange(nmax, device="cuda")
    pred = x.argmax(-1)
    up = s["parents"].long().clamp(min=0)
    good = (s["tokens"].long() == torch.gather(pred, 1, up)) | (node == 0)
    on = _root_paths(s)
    there = node < s["n"][:, None]
    ok = (~on | good[:, None, :]).all(-1) & there
    depth = on.sum(-1)
    leaf = torch.where(ok, depth * nmax - node, -1 << 40).argmax(-1)
    seqs = torch.arange(B, device="cuda")
    length = depth[seqs, leaf]
    path = torch.where(on[seqs, leaf], node, nmax).sort(-1).values.clamp(max=nmax - 1)
    toks = torch.gather(s["tokens"], 1, path).roll(-1, 1)
    toks = torch.where(node == (length - 1)[:, None], pred[seqs, leaf][:, None].int(), toks)
    inside = node < length[:, None]
    s["pred"].copy_(torch.where(there, pred.int(), s["pred"]))
    s["acc"].copy_(torch.where(inside, path.int(), s["acc"]))
    s["toks"].copy_(torch.where(inside, toks, s["toks"]))
    s["nacc"].copy_(length)


def _plain(s):
    op = s["op"]
    if op == "append":
        return _plain_append(s)
    if op == "attn":
        return _plain_attn(s)
    if op == "compact":
        return _plain_compact(s)
    if op == "process":
        counts = _plain_counts(s)
        there = (torch.arange(s["nmax"], device="cuda") < s["n"][:, None])[:, :, None]
        return [counts, torch.where(there, _plain_process(s, counts), s["out"])]
    _plain_accept(s, _plain_process(s, s["counts"]))
    return [s[k] for k in ("pred", "acc", "toks", "nacc")]


# ---------------------------------------------------------------- the calls

def _own(s):
    import paper_2603_01639_amd as ltd
    op = s["op"]
    if op in ("append", "attn", "compact"):
        paged = dict(block_table=s["table"], num_blocks=s["blocks"], scale_rows=s["sr"])
    if op == "append":
        ltd.kv_append_q8(s["k_new"], s["v_new"], s["k"][0], s["v"][0], s["ks"][0], s["vs"][0], s["prefix"], s["n"],
                         **paged)
        return [s["k"][0], s["ks"][0], s["v"][0], s["vs"][0]]
    if op == "attn":
        if "ws" not in s:
            B, nmax, Hq, d = s["q"].shape
            size = ltd.attn_q8_workspace_size(B, nmax, Hq, s["k"].shape[2], d, s["max_prefix"],
                                              ltd.DTYPE_BF16 if s["q"].dtype == torch.bfloat16 else ltd.DTYPE_F32)
            s["ws"] = torch.empty(max(1, size), dtype=torch.uint8, device="cuda")
        ltd.tree_verify_attn_q8(s["q"], s["k"][0], s["v"][0], s["ks"][0], s["vs"][0], s["prefix"], s["parents"], s["n"],
                                s["out"], max_prefix=s["max_prefix"], workspace=s["ws"], **paged)
        return s["out"]
    if op == "compact":
        ltd.kv_compact_q8(s["k"], s["v"], s["ks"], s["vs"], s["prefix"], s["new_len"], s["acc"], s["nacc"],
                          num_layers=s["layers"], layer_stride_elems=s["k"][0].numel(),
                          scale_stride_elems=s["ks"][0].numel(), **paged)
        return [s["k"], s["ks"], s["v"], s["vs"], s["new_len"]]
    t, val, n = s["bias"]
    rules = dict(penalties=s["pen"], bias_tokens=t, bias_values=val, n_bias=n, mask=s["mask"])
    if op == "process":
        ltd.token_counts(s["prompt"], s["n_prompt"], s["counts_out"], prompt=True, reset=True)
        ltd.token_counts(s["gen"], s["n_gen"], s["counts_out"])
        ltd.tree_process_logits(s["logits"], s["tokens"], s["parents"], s["n"], s["out"], counts=s["counts_out"], **rules)
        return [s["counts_out"], s["out"]]
    if "ws" not in s:
        s["ws"] = torch.empty(ltd.accept_workspace_size(s["B"], s["nmax"], s["voc"]), dtype=torch.uint8, device="cuda")
    ltd.tree_accept_processed(s["logits"], s["tokens"], s["parents"], s["n"], s["pred"], s["acc"], s["toks"], s["nacc"],
                              counts=s["counts"], workspace=s["ws"], **rules)
    return [s[k] for k in ("pred", "acc", "toks", "nacc")]


def run(s):
    return _own(s) if own else _plain(s)


# ---------------------------------------------------------------- the work

def work(case):
    r = np.random.default_rng(0)
    op, B = case["op"], case["B"]
    if op in ("process", "accept"):
        ns, voc = _ragged(r, case["N0"], case["N1"], B), case["voc"]
        need = 0.0  # logits that have to be read: the 64-byte lines with an allowed token
        for n in ns:
            for i in range(n):
                need += voc * (1 - (1 - _share(i)) ** 16) if case["grammar"] else voc
        nbytes = 4 * need + 4 * B * voc + 12 * B + sum(ns) * (8 + (voc / 8 if case["grammar"] else 0)) + 8 * B * case["bias"]
        if op == "process":
            nbytes += 4 * voc * sum(ns) + 4 * B * (case["prompt"] + case["gen"])
        return {"bytes": nbytes, "flops": 0}
    P, ns = _sizes(case, r)
    Hq, Hkv, d, sr, e = case["Hq"], case["Hkv"], case["d"], case["sr"], 2 if case["dtype"] == "bf16" else 4
    if op == "append":
        return {"bytes": sum(ns) * Hkv * d * 2 * (e + 1) + 2 * Hkv * sum(-(-n // sr) for n in ns), "flops": 0}
    if op == "compact":
        moved = B * max(1, case["acc"])
        return {"bytes": case["layers"] * Hkv * 2 * (2 * moved * d + 2 * moved) + 16 * B, "flops": 0}
    cache = sum(p + n for p, n in zip(P, ns)) * Hkv * 2 * (d + 1 / sr)
    return {"bytes": cache + 2 * sum(ns) * Hq * d * e, "flops": sum(4.0 * Hq * n * p * d for p, n in zip(P, ns))}


# ---------------------------------------------------------------- in 64 bits

def _round_e4m3(x):
    """The nearest e4m3 values (3 fraction bits, exponents from -6, largest 448), ties to even, in float64."""
    step = torch.exp2(torch.floor(torch.log2(x.abs().clamp(min=2.0 ** -6))).clamp(min=-6) - 3)
    return (torch.round(x / step) * step).clamp(-448, 448)


def _exact_rows(table, b, r, R):
    return (b, r) if table is None else (int(table[b, r // R]), r % R)


def exact(case, seed):
    s = prepare(case, seed)
    op = case["op"]
    if op in ("append", "compact"):
        if op == "append" and sum(s["ns"]) * case["Hkv"] > 40000:
            return None
        return _exact_cache(s)
    if op == "attn":
        return _exact_attn(s)
    if op == "process":
        return [None, _exact_process(s)]
    return None


def _exact_cache(s):
    """The cache's codes after the write or the move, block by block."""
    table = None if s["table"] is None else s["table"].cpu().numpy()
    out = []
    for k in ("k", "v"):
        codes, exps = s[k].double(), s[k + "s"].double() - 127
        R, sr = codes.shape[3], s["sr"]
        for b, P in enumerate(s["P"]):
            if s["op"] == "append":
                new = {P + i: s[k + "_new"][b, i].double()[None] for i in range(s["ns"][b])}  # row -> [L, H, d]
            else:
                path = s["acc"][b, :int(s["nacc"][b])].tolist()
                new, e_src = {}, {}
                for j, node in enumerate(path):
                    p, w = _exact_rows(table, b, P + node, R)
                    e_src[P + j] = exps[:, p, :, w // sr]
                    new[P + j] = codes[:, p, :, w] * torch.exp2(e_src[P + j])[..., None]
            blocks = {}
            for r in new:
                p, w = _exact_rows(table, b, r, R)
                blocks.setdefault((p, w // sr), []).append(r)
            for (p, gi), rows in blocks.items():
                first = _exact_rows(table, b, rows[0], R)[1] - gi * sr  # rows of the block that stay
                vals = torch.stack([new[r] for r in rows], 2)  # [L, H, rows, d]
                if s["op"] == "append":
                    top = vals.abs().amax((2, 3))
                    e = torch.ceil(torch.log2((top / 448).clamp(min=2.0 ** -300)))
                    e = e.clamp(E_MIN - 127, E_MAX - 127)
                else:
                    e = torch.stack([e_src[r] for r in rows]).amax(0)
                if first > 0:
                    was = exps[:, p, :, gi].clone()
                    e = torch.maximum(e, was)
                    old = codes[:, p, :, gi * sr:gi * sr + first]
                    codes[:, p, :, gi * sr:gi * sr + first] = _round_e4m3(old * torch.exp2(was - e)[..., None, None])
                exps[:, p, :, gi] = e
                at = [_exact_rows(table, b, r, R)[1] for r in rows]
                codes[:, p, :, at] = _round_e4m3(vals * torch.exp2(-e)[..., None, None])
        out += [codes[0] if s["op"] == "append" else codes, None]
    return out + ([] if s["op"] == "append" else [None])


def _exact_attn(s):
    q = s["q"].double()
    B, nmax, Hq, d = q.shape
    out = torch.zeros_like(q)
    par = s["parents"].cpu().numpy()
    R, H, sr = s["k"].shape[3], s["k"].shape[2], s["sr"]
    for b, (P, n) in enumerate(zip(s["P"], s["ns"])):
        rows = np.arange(P + n)
        pages = torch.as_tensor(np.full(P + n, b) if s["table"] is None else s["table"].cpu().numpy()[b, rows // R], device="cuda").long()
        w = torch.as_tensor(rows if s["table"] is None else rows % R, device="cuda")
        k, v = (c[0][pages, :, w].double() * torch.exp2(e[0][pages, :, w // sr].double() - 127)[..., None]
                for c, e in ((s["k"], s["ks"]), (s["v"], s["vs"])))  # [T, H, d]
        hide = np.ones((n, P + n), bool)
        hide[:, :P] = False
        for i in range(n):
            j = i
            while j >= 0:
                hide[i, P + j] = False
                j = int(par[b, j])
        hide = torch.as_tensor(hide, device="cuda")
        for h in range(Hq):
            g = h // (Hq // H)
            x = (q[b, :n, h] @ k[:, g].T) / math.sqrt(d)
            out[b, :n, h] = torch.softmax(x.masked_fill(hide, -math.inf), 1) @ v[:, g]
    return out


def _exact_process(s):
    B, nmax, voc = s["B"], s["nmax"], s["voc"]
    out = torch.zeros((B, nmax, voc), dtype=torch.float64, device="cuda")
    par, tok, pen = s["parents"].cpu().numpy(), s["tokens"].cpu().numpy(), s["pen"].double()
    for b in range(B):
        seen = torch.zeros(voc, dtype=torch.bool, device="cuda")
        seen[s["prompt"][b, :int(s["n_prompt"][b])].long()] = True
        made = torch.bincount(s["gen"][b, :int(s["n_gen"][b])].long(), minlength=voc).double()
        add = torch.zeros(voc, dtype=torch.float64, device="cuda")
        if s["bias"][0] is not None:
            n = int(s["bias"][2][b])
            add[s["bias"][0][b, :n].long()] += s["bias"][1][b, :n].double()
        for i in range(s["ns"][b]):
            c, j = made.clone(), i
            while j > 0:
                c[int(tok[b, j])] += 1
                j = int(par[b, j])
            x = s["logits"][b, i].double()
            x = torch.where(seen | (c > 0), torch.where(x > 0, x / pen[b, 0], x * pen[b, 0]), x)
            x = x - pen[b, 1] * c - pen[b, 2] * (c > 0) + add
            if s["mask"] is not None:
                at = torch.arange(voc, device="cuda")
                x = torch.where((s["mask"][b, i][at // 32] >> (at % 32).int()) & 1 > 0, x, -math.inf)
            out[b, i] = x
    return out
