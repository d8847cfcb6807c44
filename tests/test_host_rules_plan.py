"""The sampling rules' node groups (csrc/rules_plan.hpp) on the host: they follow the device's compute units."""
import numpy as np
import pytest

import rules_plan as R


@pytest.fixture(scope="module")
def exe(tmp_path_factory):
    return R.build(tmp_path_factory.mktemp("rules"))


@pytest.mark.parametrize("argmax", [False, True])
def test_groups_fill_one_round_of_the_card(exe, argmax):
    rng = np.random.default_rng(1)
    most = 8 if argmax else 4
    for _ in range(200):
        B, N, voc = (int(2 ** rng.uniform(0, x)) for x in (6, 8, 17))
        cus = int(rng.choice([32, 64, 128, 256]))
        chunks = -(-voc // R.CHUNK[argmax])
        card = cus * (1024 // R.THREADS[argmax])
        got = R.nodes(exe, B, N, voc, argmax, cus)
        assert 1 <= got <= most
        if got < most - 1:  # as few nodes as leave one round
            assert B * N * chunks <= got * card
        if got > 1:
            assert B * N * chunks > (got - 1) * card


def test_a_smaller_card_takes_larger_groups(exe):
    for argmax in (False, True):
        by_cus = [R.nodes(exe, 1, 60, 128256, argmax, cus) for cus in (256, 128, 64)]
        assert by_cus == sorted(by_cus) and by_cus[0] < by_cus[-1]


def test_the_groups_of_known_calls(exe):
    assert [R.nodes(exe, 1, 60, 128256, a) for a in (False, True)] == [2, 2]
    assert [R.nodes(exe, 16, 96, 128256, a) for a in (False, True)] == [4, 7]
    assert R.nodes(exe, 16, 60, 32000, True) == 8
