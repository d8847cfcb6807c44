"""The sampling rules with 3 to 8 nodes a workgroup, as serving batches give: nodes of one group with masks, draft tokens,
paths and biases of their own, ragged trees whose last group is a part of one, written, in place and as the argmax.
(Definitions and tolerances are those of test_gpu_logit_rules; each case first makes sure of its group size.)"""
import numpy as np
import pytest

import oracle
import rules_plan as R
from test_gpu_logit_rules import accept, check, make, process

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def exe(tmp_path_factory):
    return R.build(tmp_path_factory.mktemp("rules"))


def _cus():
    import torch
    return torch.cuda.get_device_properties(0).multi_processor_count


def _sizes(B, nmax, seed):
    """Trees of every size up to nmax: whole groups, remainders and single nodes."""
    n = np.random.default_rng(seed).integers(1, nmax + 1, B)
    n[:4] = [nmax, nmax - 1, 1, 5][:B]
    return [int(x) for x in n]


GRAMMAR = [0.9, 0.3, 0.0, 0.99, 0.01, 0.6, 1.0]  # (7 shares: no group of up to 8 nodes repeats with them)


@pytest.mark.parametrize("in_place", [False, True])
@pytest.mark.parametrize("nodes, B, nmax, voc", [(3, 16, 160, 4096), (4, 16, 250, 4091), (3, 10, 150, 4101), (4, 30, 35, 16390)])
@pytest.mark.parametrize("mask, bias", [(True, 200), (False, 7)])
def test_written_groups(exe, nodes, B, nmax, voc, mask, bias, in_place):
    assert R.nodes(exe, B, nmax, voc, False, _cus()) == nodes
    m = make(nodes + voc, _sizes(B, nmax, voc), voc, bias=bias, grammar=GRAMMAR if mask else None, gen=200, prompt=300)
    check(m, process(m, in_place), None if in_place else 123.0, f"{nodes} nodes")


@pytest.mark.parametrize("nodes, B, nmax, voc", [(3, 6, 110, 5003), (4, 8, 120, 700), (5, 10, 121, 4000), (6, 6, 119, 20001),
                                                 (7, 40, 110, 3001), (8, 16, 128, 5000), (8, 16, 63, 20001)])
@pytest.mark.parametrize("mask, bias", [(True, 200), (False, 7)])
def test_argmax_groups(exe, nodes, B, nmax, voc, mask, bias):
    """Every prediction is the written row's first largest token, and the decision the oracle's on the written rows."""
    assert R.nodes(exe, B, nmax, voc, True, _cus()) == nodes
    m = make(nodes + voc, _sizes(B, nmax, voc), voc, bias=bias, grammar=GRAMMAR if mask else None, gen=200, prompt=300)
    rng = np.random.default_rng(nodes)
    for b, n in enumerate(m["n"]):  # let some drafts be right
        for i in range(1, int(n)):
            if rng.random() < 0.6:
                m["logits"][b, m["parents"][b, i], m["tokens"][b, i]] += 40
    written = process(m)
    check(m, written, 123.0, f"{nodes} nodes")
    got = accept(m)
    written = np.nan_to_num(written, neginf=-3.0e38)
    par = np.where(np.arange(nmax) < m["n"][:, None], m["parents"], 0).astype(np.int32)
    par[:, 0] = -1
    want = oracle.tree_accept(written, m["tokens"], par, m["n"])
    np.testing.assert_array_equal(got[3], want[3])
    for b, n in enumerate(m["n"]):
        k = int(want[3][b])
        np.testing.assert_array_equal(got[0][b, :n], written[b, :n].argmax(-1))
        np.testing.assert_array_equal(got[1][b, :k], want[1][b, :k])
        np.testing.assert_array_equal(got[2][b, :k], want[2][b, :k])
