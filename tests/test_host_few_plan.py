"""How attention over an 8-bit cache cuts its short units (csrc/few_plan.hpp), built for the host with g++ and checked on
random batches: whatever bound on the prefixes a launch is sized for, the call's splits have the same length, fit the
launch's slots, the merge's table and the block-id table, and need more rounds than one only where a split would be
longer than that table allows."""
import os
import subprocess

import numpy as np
import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2603_01639_amd", "csrc")
MIN, MAX, TILE, MOST = 128, 7680, 64, 1024

DRIVER = r"""
#include <cstdio>
#include <vector>
#include "few_plan.hpp"
using namespace ltd::few;
// stdin: "B Hkv cus max_prefix" and B prefixes; stdout: target, width, slots, workgroups, keys, rounds
int main() {
  int B, H, cus, mp;
  while (std::scanf("%d %d %d %d", &B, &H, &cus, &mp) == 4) {
    std::vector<int> P(B);
    int64_t T = 0;
    for (int& p : P) {
      if (std::scanf("%d", &p) != 1) return 2;
      T += p;
    }
    const int resident = 2 * cus;
    const int64_t units = int64_t(B) * H, t = target(units, resident), width = round_width(units, resident);
    const Length len = B == 1 ? one_length(P[0], H, int(t), int(width), mp)
                              : batch_length(T, H, int(units), int(t), int(width), mp, [&](int keys) {
                                  int n = 0;
                                  for (int p : P) n += p > 0 ? (p + keys - 1) / keys : 1;
                                  return n * H;
                                });
    std::printf("%lld %lld %lld %lld %d %d\n", (long long)t, (long long)width, (long long)most_splits(units, mp, resident),
                (long long)workgroups(units, mp, resident), len.keys, len.rounds);
  }
  return 0;
}
"""


@pytest.fixture(scope="module")
def plan(tmp_path_factory):
    d = tmp_path_factory.mktemp("few")
    (d / "few.cpp").write_text(DRIVER)
    subprocess.run(["g++", "-std=c++17", "-O1", "-I", CSRC, str(d / "few.cpp"), "-o", str(d / "few")], check=True)

    def run(cases):
        """cases: (Hkv, cus, max_prefix, prefixes)."""
        text = "\n".join(f"{len(P)} {H} {cus} {mp} " + " ".join(map(str, P)) for H, cus, mp, P in cases)
        r = subprocess.run([str(d / "few")], input=text, capture_output=True, text=True, timeout=60)
        assert r.returncode == 0
        return [tuple(map(int, line.split())) for line in r.stdout.splitlines()]
    return run


def _splits(P, H, keys):
    return sum(max(-(-p // keys), 1) for p in P) * H


def _check(case, got):
    H, _, mp, P = case
    target, width, slots, wgs, keys, rounds = got
    units, n, few = len(P) * H, _splits(P, H, keys), _splits(P, H, MAX)
    top = MAX // 2 if width > target and len(P) > 1 else MAX
    assert keys % TILE == 0 and MIN <= keys <= MAX
    assert max(-(-p // keys) for p in P) <= MOST
    assert n <= rounds * wgs and n <= slots  # (every split has a workgroup and a slot)
    assert units <= n and wgs <= max(target, width)
    if _splits(P, H, top) <= target:  # the splits run side by side, or are dealt out once
        assert rounds == 1 and n <= target and keys <= top
    else:
        assert keys >= MAX // 2 and (rounds - 1) * width < few <= rounds * width


def _random(rng):
    B = int(rng.choice([1, 2, 3, 16, 64, 65, 200, 300]))
    H = int(rng.choice([1, 2, 4, 8, 40]))
    top = int(2 ** rng.uniform(0, 19 if B < 64 else 16))
    kind = rng.integers(0, 4)
    if kind == 0:
        P = [top] * B
    elif kind == 1:
        P = [int(x) for x in rng.integers(0, top + 1, B)]
    elif kind == 2:  # one long sequence among empty ones
        P = [0] * B
        P[int(rng.integers(0, B))] = top
    else:
        P = [int(x) for x in top / MIN * rng.integers(0, 3, B)]
    return H, int(rng.choice([256, 256, 128, 32])), max(P), P


def test_random_batches(plan):
    rng = np.random.default_rng(5)
    cases = [_random(rng) for _ in range(3000)]
    for case, got in zip(cases, plan(cases)):
        _check(case, got)


def test_the_bound_on_the_prefixes_does_not_move_the_splits(plan):
    rng = np.random.default_rng(6)
    cases = [_random(rng) for _ in range(500)]
    cases.append((8, 256, 8192, [int(x) for x in np.linspace(1024, 8192, 16)]))
    tight = plan(cases)
    for mp in (8192, 32768, 131072, 1 << 20, 3_900_000):
        loose = [(H, cus, max(mp, m), P) for H, cus, m, P in cases]
        for a, b, got in zip(loose, tight, plan(loose)):
            _check(a, got)
            assert got[4:] == b[4:], (a, b, got)


def test_the_shortest_length_that_fits_side_by_side(plan):
    rng = np.random.default_rng(7)
    cases = [c for c in (_random(rng) for _ in range(2000)) if 1 < len(c[3]) and 4 * len(c[3]) * c[0] <= 512 and c[1] == 256]
    assert len(cases) > 300
    for (H, _, _, P), (target, width, _, _, keys, rounds) in zip(cases, plan(cases)):
        least, room = (MIN, target) if _splits(P, H, MAX) <= target else (MAX // 2, rounds * width)
        assert keys == least or _splits(P, H, keys - TILE) > room


@pytest.mark.parametrize("B, H", [(1, 1), (1, 8), (129, 1), (200, 1), (2, 1)])
def test_the_longest_prefixes(plan, B, H):
    """Prefixes up to what the matrix kernel plans for, alone and among empty ones."""
    top = MAX * MOST
    cases = [(H, 256, top, [p] + [0] * (B - 1)) for p in (top, top - 1, top // 2, 3_932_160, 1_000_000, 7681 * 64)]
    for case, got in zip(cases, plan(cases)):
        _check(case, got)
