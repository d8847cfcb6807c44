"""Rotary frequencies and their scalings for long contexts, against their definitions written out pair by pair."""
import math

import pytest

import paper_2603_01639_amd as ltd


def plain(rot, base):
    return [base ** (-2 * j / rot) for j in range(rot // 2)]


def check(got, want):
    f, m = got
    assert f.dtype.is_floating_point and f.element_size() == 8
    assert f.tolist() == pytest.approx(want, rel=1e-14)
    return m


@pytest.mark.parametrize("rot, base", [(2, 10000.0), (64, 10000.0), (128, 500000.0), (36, 1e6)])
def test_plain_and_linear(rot, base):
    assert check(ltd.rope_frequencies(rot, base), plain(rot, base)) == 1.0
    assert check(ltd.rope_frequencies(rot, base, scaling="linear", factor=8.0), [x / 8 for x in plain(rot, base)]) == 1.0


def test_ntk_keeps_the_fastest_and_divides_the_slowest():
    f, m = ltd.rope_frequencies(128, 10000.0, scaling="ntk", factor=4.0)
    p = plain(128, 10000.0)
    assert m == 1.0 and f[0] == 1.0
    assert float(f[-1]) == pytest.approx(p[-1] / 4, rel=1e-13)
    ratio = [float(a) / b for a, b in zip(f, p)]
    assert all(x > y for x, y in zip(ratio, ratio[1:]))


def test_yarn():
    rot, base, s, trained = 64, 10000.0, 40.0, 4096
    f, m = ltd.rope_frequencies(rot, base, scaling="yarn", factor=s, trained_len=trained)
    assert m == pytest.approx(0.1 * math.log(40.0) + 1)
    # the pair (a real number) that turns t times within the trained length
    at = lambda t: rot / 2 * math.log(trained / (2 * math.pi * t), base)  # noqa: E731
    lo, hi = math.floor(at(32)), math.ceil(at(1))
    assert (lo, hi) == (10, 23)
    for j, (x, p) in enumerate(zip(f.tolist(), plain(rot, base))):
        w = min(max((j - lo) / (hi - lo), 0.0), 1.0)
        assert x == pytest.approx(p * (1 - w) + p / s * w, rel=1e-13)
        if trained * p / (2 * math.pi) < 1:
            assert x == pytest.approx(p / s)
    assert ltd.rope_frequencies(rot, base, scaling="yarn", factor=1.0, trained_len=trained)[1] == 1.0


def test_bands():
    rot, base, s, trained = 128, 500000.0, 8.0, 8192
    f, m = ltd.rope_frequencies(rot, base, scaling="bands", factor=s, trained_len=trained, low_factor=1.0, high_factor=4.0)
    assert m == 1.0
    kinds = set()
    for x, p in zip(f.tolist(), plain(rot, base)):
        wave = 2 * math.pi / p
        if wave < trained / 4:
            kinds.add("kept")
            assert x == pytest.approx(p, rel=1e-14)
        elif wave > trained:
            kinds.add("slowed")
            assert x == pytest.approx(p / s, rel=1e-14)
        else:
            kinds.add("blended")
            k = (trained / wave - 1) / 3
            assert x == pytest.approx((1 - k) * p / s + k * p, rel=1e-13)
    assert kinds == {"kept", "slowed", "blended"}


@pytest.mark.parametrize("kw", [dict(rot_dim=3), dict(rot_dim=0), dict(rot_dim=64, base=1.0), dict(rot_dim=64, factor=0.0),
                                dict(rot_dim=64, scaling="other"), dict(rot_dim=64, scaling="yarn", factor=2.0),
                                dict(rot_dim=64, scaling="bands", factor=2.0), dict(rot_dim=2, scaling="ntk", factor=2.0),
                                dict(rot_dim=64, scaling="bands", factor=2.0, trained_len=8, low_factor=4.0, high_factor=1.0)])
def test_refusals(kw):
    with pytest.raises(ValueError):
        ltd.rope_frequencies(**kw)
