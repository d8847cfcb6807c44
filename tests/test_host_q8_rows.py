"""The blocks that an append to an 8-bit cache touches (csrc/q8_rows.hpp), built for the host with g++: every row lies in
exactly one unit's block, and units past the rows have none, up to the longest lengths the call takes."""
import os
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2603_01639_amd", "csrc")
TOP = 1 << 30  # rows and prefixes end here

DRIVER = r"""
#include <cstdio>
#include "q8_rows.hpp"
// stdin: "u rows sr" or "b P n unit sr", one a line; stdout: the answers
int main() {
  char what;
  while (std::scanf(" %c", &what) == 1) {
    int a, b, c, d;
    if (what == 'u') {
      if (std::scanf("%d %d", &a, &b) != 2) return 2;
      std::printf("%d\n", ltd::append_units(a, b));
    } else {
      if (std::scanf("%d %d %d %d", &a, &b, &c, &d) != 4) return 2;
      std::printf("%d\n", ltd::append_block(a, b, c, d));
    }
  }
  return 0;
}
"""


@pytest.fixture(scope="module")
def ask(tmp_path_factory):
    d = tmp_path_factory.mktemp("rows")
    (d / "rows.cpp").write_text(DRIVER)
    subprocess.run(["g++", "-std=c++17", "-O1", "-I", CSRC, str(d / "rows.cpp"), "-o", str(d / "rows")], check=True)

    def run(lines):
        r = subprocess.run([str(d / "rows")], input="\n".join(lines), capture_output=True, text=True, timeout=20)
        assert r.returncode == 0
        return [int(x) for x in r.stdout.split()]
    return run


@pytest.mark.parametrize("sr", [16, 32, 64, 128])
def test_every_row_has_one_block(ask, sr):
    starts = [0, 1, sr - 1, sr, 5 * sr + 3, TOP - 2 * sr, TOP - sr - 1]
    for n in (1, 2, sr - 1, sr, sr + 1, 3 * sr + 2):
        units, = ask([f"u {n} {sr}"])
        for P in starts:
            if P + n > TOP:
                continue
            got = ask([f"b {P} {n} {u} {sr}" for u in range(units + 4)])
            want = list(range(P // sr * sr, P + n, sr))
            assert len(want) <= units
            assert got == want + [-1] * (units + 4 - len(want))


@pytest.mark.parametrize("sr", [16, 32, 64, 128])
def test_units_past_the_rows_of_the_longest_call(ask, sr):
    """Few rows near the end of a cache in a launch for the most rows: the last units' first rows pass 2^31."""
    units, = ask([f"u {TOP} {sr}"])
    assert units == TOP // sr + 1
    for P, n in ((TOP - 1, 1), (TOP - sr, 3), (TOP - 2 * sr, sr), (TOP, 0)):
        last = [units - 3, units - 2, units - 1, units, units + 1, units + 2]
        assert ask([f"b {P} {n} {u} {sr}" for u in last]) == [-1] * 6
    assert ask([f"b 0 {TOP} {TOP // sr - 1} {sr}"]) == [TOP - sr]
    assert ask([f"b 0 {TOP} {TOP // sr} {sr}"]) == [-1]
