"""Penalties, biases and masks on the logits of tree nodes, the table of occurrences, and greedy acceptance on processed
logits, on the GPU against their definitions in 64 bits.

A processed logit takes at most five float32 roundings (the penalty, the product f * c, two subtractions, the
bias), and a biased token's sum one per further entry: each off by at most 2^-24 of its result, all of which are
bounded by |x| * max(r, 1/r) + |f| * c + |p| + sum|bias|.  Five times that, times 2^-24, bounds the error.  Where the
definition leaves a logit alone its bits are kept."""
import numpy as np
import pytest

import oracle
import paper_2603_01639_amd as ltd
import q8_util as Q

pytestmark = pytest.mark.gpu


def make(seed, sizes, voc, *, prompt=40, gen=30, bias=0, grammar=None, kind="random", std=3.0, dup=True, counts=True,
         pen=True, nmax=None):
    rng = np.random.default_rng(seed)
    B = len(sizes)
    par = Q.trees(rng, sizes, kind)
    if nmax:
        par = np.pad(par, ((0, 0), (0, nmax - par.shape[1])), constant_values=99999)
    N = par.shape[1]
    tok = rng.integers(0, min(voc, 50) if dup else voc, (B, N)).astype(np.int32)
    m = dict(logits=(rng.normal(size=(B, N, voc)) * std).astype(np.float32), tokens=tok, parents=par,
             n=np.array(sizes, np.int32), counts=None, pen=None, bias=None, mask=None, voc=voc)
    m["logits"][:, :, rng.integers(0, voc, 3)] = 0.0
    if counts:
        c = np.zeros((B, voc), np.int64)
        for b in range(B):
            np.add.at(c[b], rng.integers(0, voc, gen) % max(1, voc // 2), 1)
            c[b, rng.integers(0, voc, prompt)] |= -(1 << 31)
        m["counts"] = c.astype(np.int32)
    if pen:
        m["pen"] = np.stack([rng.uniform(0.7, 1.5, B), rng.uniform(-0.5, 0.9, B), rng.uniform(-0.5, 0.9, B)], 1).astype(np.float32)
    if bias:
        t = rng.integers(0, voc, (B, bias)).astype(np.int32)
        t[:, ::5] = t[:, :1]  # the same token again and again
        n = rng.integers(0, bias + 1, B).astype(np.int32)
        n[0] = bias
        m["bias"] = (t, (rng.normal(size=t.shape) * 5).astype(np.float32), n)
    if grammar is not None:
        words = -(-voc // 32)
        keep = rng.random((B, N, words * 32)) < np.asarray(grammar)[np.arange(N) % len(grammar)][None, :, None]
        keep[..., voc:] = True  # bits past the vocabulary mean nothing
        m["mask"] = np.packbits(keep.reshape(B, N, words, 32), axis=-1, bitorder="little").view(np.int32)[..., 0]
    return m


def rules(m):
    t, x, n = m["bias"] if m["bias"] is not None else (None, None, None)
    return {k: Q.to_dev(v) for k, v in dict(counts=m["counts"], penalties=m["pen"], bias_tokens=t, bias_values=x, n_bias=n,
                                            mask=m["mask"]).items()}


def process(m, in_place=False, fill=123.0, **more):
    import torch
    lg = Q.to_dev(m["logits"])
    out = lg if in_place else torch.full_like(lg, fill)
    ltd.tree_process_logits(lg, Q.to_dev(m["tokens"]), Q.to_dev(m["parents"]), Q.to_dev(m["n"]), out, **rules(m), **more)
    torch.cuda.synchronize()
    return out.cpu().numpy()


def wanted(m):
    return Q.rules(m["logits"], m["tokens"], m["parents"], m["n"], m["counts"], m["pen"], m["bias"], m["mask"])


def bound(m):
    """Per logit: five float32 half steps of the largest value on its way."""
    lg = np.abs(m["logits"].astype(np.float64))
    B, N, voc = lg.shape
    top = lg.copy()
    if m["pen"] is not None:
        r, f, p = (np.abs(m["pen"].astype(np.float64))[:, k][:, None, None] for k in range(3))
        c = np.zeros((B, voc)) if m["counts"] is None else (m["counts"].astype(np.int64) & 0x7FFFFFFF).astype(np.float64)
        top = lg * np.maximum(r, 1 / r) + f * (c[:, None] + N) + p
    steps = 5
    if m["bias"] is not None:
        t, x, n = m["bias"]
        add = np.zeros((B, voc))
        for b in range(B):
            use = slice(0, int(n[b]))
            ok = (t[b, use] >= 0) & (t[b, use] < voc)
            np.add.at(add[b], t[b, use][ok], np.abs(x[b, use][ok].astype(np.float64)))
        top, steps = top + add[:, None], 5 + t.shape[1]
    return steps * 2.0 ** -24 * top + 1e-40


def check(m, got, fill, label=""):
    want, tol = wanted(m), bound(m)
    for b, n in enumerate(m["n"]):
        w, g = want[b, :n], got[b, :n]
        low = np.isneginf(w)
        assert np.array_equal(np.isneginf(g), low), f"{label} sequence {b}: masked tokens"
        err = np.abs(np.where(low, 0.0, g) - np.where(low, 0.0, w))
        assert (err <= np.where(low, 0.0, tol[b, :n])).all(), f"{label} sequence {b}: {float((err - tol[b, :n]).max())}"
        same = np.where(low, True, w == m["logits"][b, :n].astype(np.float64))
        np.testing.assert_array_equal(g[same & ~low], m["logits"][b, :n][same & ~low].astype(np.float32) + 0.0)
        rest = m["logits"][b, n:] if fill is None else np.full_like(m["logits"][b, n:], fill)
        np.testing.assert_array_equal(got[b, n:], rest)


CASES = [
    dict(sizes=[1], voc=1),
    dict(sizes=[1], voc=7, bias=3),
    dict(sizes=[5], voc=31, grammar=[0.5, 0.0]),
    dict(sizes=[9, 1], voc=33, bias=9, grammar=[0.9]),
    dict(sizes=[17, 4, 30], voc=4096, bias=20),
    dict(sizes=[12], voc=4097, grammar=[0.98, 0.001, 0.0, 0.3], bias=300),
    dict(sizes=[3, 8], voc=50257, grammar=[0.98, 0.01], bias=5),
    dict(sizes=[6], voc=16384 + 5, bias=1000, dup=False),
    dict(sizes=[6, 2], voc=32000, pen=False, grammar=[0.4]),
    dict(sizes=[6, 2], voc=32000, counts=False),
    dict(sizes=[6, 2], voc=32000, counts=False, pen=False, bias=40),
    dict(sizes=[60], voc=128256, bias=20),
    dict(sizes=[20, 7], voc=2000, nmax=64, grammar=[0.5]),
]


@pytest.mark.parametrize("in_place", [False, True])
@pytest.mark.parametrize("case", CASES, ids=lambda c: "-".join(f"{k}={v}" for k, v in c.items()).replace(" ", ""))
def test_process(case, in_place):
    m = make(sum(case["sizes"]) + case["voc"], **case)
    check(m, process(m, in_place), None if in_place else 123.0)


@pytest.mark.parametrize("kind", ["chain", "star"])
def test_trees_of_one_token(kind):
    """256 nodes that all carry the same token: a chain counts it up to 255 times."""
    m = make(2, [256, 200], 600, kind=kind)
    m["tokens"][:] = 77
    check(m, process(m), 123.0, kind)


def test_infinite_logits_and_tokens_outside_the_vocabulary():
    m = make(12, [8, 5], 1000, bias=12)
    m["logits"][:, :, 3] = -np.inf
    m["logits"][:, :, 900] = np.inf
    m["logits"][:, :, 901] = -0.0
    m["tokens"][:, 2] = 1000
    m["tokens"][:, 3] = -5
    m["bias"][0][:, 1] = 1000
    m["bias"][0][:, 2] = -1
    got, want = process(m), wanted(m)
    for b, n in enumerate(m["n"]):
        inf = np.isinf(want[b, :n])
        np.testing.assert_array_equal(got[b, :n][inf], want[b, :n][inf].astype(np.float32))
        m["logits"][b, :n][inf] = 0.0
        assert (np.abs(np.where(inf, 0, got[b, :n]) - np.where(inf, 0, want[b, :n])) <= bound(m)[b, :n]).all()


def test_token_counts():
    import torch
    rng = np.random.default_rng(1)
    B, T, voc = 5, 700, 301
    tok = rng.integers(-3, voc + 3, (B, T)).astype(np.int32)
    tok[2] = 17
    n = np.array([T, 0, T, 1, T + 50], np.int32)
    counts = torch.full((B, voc), 12345, dtype=torch.int32, device="cuda")
    ltd.token_counts(Q.to_dev(tok), Q.to_dev(n), counts, prompt=True, reset=True)
    more = rng.integers(0, voc, (B, 9)).astype(np.int32)
    n2 = np.array([9, 3, 0, -2, 5], np.int32)
    for _ in range(3):
        ltd.token_counts(Q.to_dev(more), Q.to_dev(n2), counts)
    torch.cuda.synchronize()
    want = np.zeros((B, voc), np.int64)
    for b in range(B):
        t = tok[b, :min(n[b], T)]
        want[b, t[(t >= 0) & (t < voc)]] |= -(1 << 31)
        np.add.at(want[b], more[b, :max(n2[b], 0)], 3)
    np.testing.assert_array_equal(counts.cpu().numpy(), want.astype(np.int32))


def accept(m, **more):
    import torch
    B, N = m["tokens"].shape
    outs = [torch.full((B, N), -1, dtype=torch.int32, device="cuda") for _ in range(3)]
    nacc = torch.zeros(B, dtype=torch.int32, device="cuda")
    ltd.tree_accept_processed(Q.to_dev(m["logits"]), Q.to_dev(m["tokens"]), Q.to_dev(m["parents"]), Q.to_dev(m["n"]), *outs,
                              nacc, **rules(m), **more)
    torch.cuda.synchronize()
    return [t.cpu().numpy() for t in outs] + [nacc.cpu().numpy()]


@pytest.mark.parametrize("case", CASES, ids=lambda c: "-".join(f"{k}={v}" for k, v in c.items()).replace(" ", ""))
def test_accept_processed(case):
    """The decision equals acceptance on the processed logits that were written, which the test above pins: prediction
    by prediction, path by path."""
    m = make(sum(case["sizes"]) + case["voc"] + 1, **case)
    rng = np.random.default_rng(4)
    for b, n in enumerate(m["n"]):  # let some drafts be right
        for i in range(1, int(n)):
            if rng.random() < 0.6:
                m["logits"][b, m["parents"][b, i], m["tokens"][b, i]] += 40
    written = np.nan_to_num(process(m), neginf=-3.0e38)
    par = np.where(np.arange(m["parents"].shape[1]) < m["n"][:, None], m["parents"], 0).astype(np.int32)
    par[:, 0] = -1
    want = oracle.tree_accept(written, m["tokens"], par, m["n"])
    got = accept(m)
    np.testing.assert_array_equal(got[3], want[3])
    for b, n in enumerate(m["n"]):
        k = int(want[3][b])
        np.testing.assert_array_equal(got[0][b, :n], want[0][b, :n])
        np.testing.assert_array_equal(got[1][b, :k], want[1][b, :k])
        np.testing.assert_array_equal(got[2][b, :k], want[2][b, :k])
        assert (got[0][b, n:] == -1).all() and (got[1][b, k:] == -1).all() and (got[2][b, k:] == -1).all()


def test_empty_masks_predict_token_zero():
    m = make(9, [4], 40000, grammar=[0.0])
    assert (accept(m)[0][0] == 0).all()
    assert np.isneginf(process(m)[0]).all()


@pytest.mark.parametrize("what, code", [("n", ltd.STATUS_BAD_NNODES), ("parent", ltd.STATUS_BAD_PARENT),
                                        ("repetition", ltd.STATUS_BAD_RULE), ("nan", ltd.STATUS_BAD_RULE),
                                        ("bias", ltd.STATUS_BAD_RULE), ("none", 0)])
def test_validation(what, code):
    import torch
    m = make(8, [5, 6], 500, bias=4)
    if what == "n":
        m["n"][1] = 7
    elif what == "parent":
        m["parents"][1, 2] = 3
    elif what == "repetition":
        m["pen"][1, 0] = 0.0
    elif what == "nan":
        m["pen"][0, 2] = np.nan
    elif what == "bias":
        m["bias"][2][1] = 5
    status = torch.full((1,), 55, dtype=torch.int32, device="cuda")
    got = process(m, validate=True, status=status)
    assert int(status.cpu()[0]) == code
    assert (got == 123.0).all() == (code != 0)
    status.fill_(55)
    acc = accept(m, validate=True, status=status)
    assert int(status.cpu()[0]) == code
    assert (acc[0] == -1).all() == (code != 0)


@pytest.mark.parametrize("temperature", [0.7, 1.0])
def test_sampling_on_processed_logits(temperature):
    """Acceptance by sampling takes the written logits, minus infinities and a node without an allowed token among
    them, as the oracle does."""
    import torch
    rng = np.random.default_rng(33)
    m = make(5, [24, 9, 17], 3000, bias=30, grammar=[0.6, 0.05, 0.9, 0.0], dup=False)
    B, N = m["tokens"].shape
    m["mask"][:, 0] = -1  # the root is on the grammar
    draft = np.zeros((B, N, 3000), np.float32)
    for b, n in enumerate(m["n"]):
        for u in range(int(n)):
            kids = np.nonzero(m["parents"][b, :n] == u)[0]
            p = np.exp(m["logits"][b, u].astype(np.float64) + rng.normal(size=3000))
            draft[b, u] = p / p.sum()
            if len(kids):
                m["tokens"][b, kids] = rng.choice(3000, size=len(kids), replace=False, p=p / p.sum())
    uni = rng.random((B, N, 2)).astype(np.float32) * np.float32(1 - 2.0 ** -20)
    done = process(m, fill=0.0)
    outs = [torch.full((B, N), -1, dtype=torch.int32, device="cuda") for _ in range(2)]
    nacc = torch.zeros(B, dtype=torch.int32, device="cuda")
    par = np.where(np.arange(N) < m["n"][:, None], m["parents"], 0).astype(np.int32)
    par[:, 0] = -1
    ltd.tree_accept_sampling(Q.to_dev(done), Q.to_dev(draft), Q.to_dev(m["tokens"]), Q.to_dev(par), Q.to_dev(m["n"]),
                             Q.to_dev(uni), *outs, nacc, temperature=temperature)
    torch.cuda.synchronize()
    path, toks, want = oracle.tree_accept_sampling(done, draft, m["tokens"], par, m["n"], uni, temperature=temperature)[:3]
    np.testing.assert_array_equal(nacc.cpu().numpy(), want)
    for b in range(B):
        k = int(want[b])
        np.testing.assert_array_equal(outs[0][b, :k].cpu().numpy(), path[b, :k])
        np.testing.assert_array_equal(outs[1][b, :k].cpu().numpy(), toks[b, :k])
        for j in range(k):  # (a node that allows nothing has no token to go on with)
            row = done[b, path[b, j]]
            assert np.isfinite(row[toks[b, j]]) or np.isneginf(row).all()


@pytest.mark.parametrize("voc", [100, 5003])
def test_masked_logits_and_banned_tokens(voc):
    """NaN and infinities where the mask forbids a token, rules or not, change nothing; a bias of -infinity bans its token."""
    m = make(voc, [9, 20], voc, bias=30, grammar=[0.6, 0.02], nmax=24)
    m["bias"][1][:, 1::7] = -np.inf
    keep = np.unpackbits(m["mask"].view(np.uint8), axis=-1, bitorder="little").reshape(2, 24, -1)[..., :voc].astype(bool)
    dirty = dict(m, logits=np.where(keep, m["logits"], np.resize(np.array([np.nan, np.inf, -np.inf], np.float32),
                                                                 m["logits"].shape)))
    for in_place in (False, True):
        for b, n in enumerate(m["n"]):
            np.testing.assert_array_equal(process(dirty, in_place)[b, :n], process(m, in_place)[b, :n])
    got = process(dirty)
    assert all((got[b, i][~keep[b, i]] == -np.inf).all() for b, n in enumerate(m["n"]) for i in range(n))
    banned = [m["bias"][0][b, 1] for b in range(2)]
    assert all((got[b, :n, banned[b]] == -np.inf).all() for b, n in enumerate(m["n"]) if m["bias"][2][b] > 1)
    for x, y in zip(accept(dirty), accept(m)):
        np.testing.assert_array_equal(x, y)


@pytest.mark.parametrize("rep, freq, pres", [(1.3, 0.4, 0.2), (0.6, 0.0, 0.0), (1.0, -0.7, 0.1), (1.2, -0.3, -0.5), (1.0, 0.0, 0.0),
                                             (1.0, 2.0, 1.0)])
def test_accept_where_penalised_tokens_compete(rep, freq, pres):
    """Vocabularies of mostly counted tokens with logits close together, equal ones among them: the best token is now a
    penalised one, now a plain one, and often tied."""
    rng = np.random.default_rng(int(rep * 100 + freq * 10 + 50))
    sizes, voc = [24, 7, 40], 20000
    m = make(3, sizes, voc, prompt=9000, gen=12000, bias=12, std=0.0)
    m["pen"] = np.tile(np.array([rep, freq, pres], np.float32), (3, 1))
    m["logits"] = (rng.integers(-3, 4, m["logits"].shape) / 4).astype(np.float32)
    m["logits"][0] += 2
    m["logits"][1] -= 2
    got = accept(m)
    written = np.nan_to_num(process(m), neginf=-3.0e38)
    for b, n in enumerate(m["n"]):
        np.testing.assert_array_equal(got[0][b, :n], written[b, :n].argmax(-1))
