"""Whether two strided tensors share bytes (csrc/runs.hpp, built for the host with g++; and the binding's form of it),
against sets of bytes."""
import os
import random
import subprocess

import pytest

import paper_2603_01639_amd as ltd

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2603_01639_amd", "csrc")

DRIVER = r"""
#include <cstdio>
#include "runs.hpp"
// stdin: at rows row heads head run, twice a line; 1 or 0 a line
int main() {
  long long t[12];
  while (true) {
    for (int i = 0; i < 12; ++i)
      if (std::scanf("%lld", t + i) != 1) return i ? 2 : 0;
    const ltd::Runs x{static_cast<uint64_t>(t[0]), t[1], t[2], t[3], t[4], t[5]}, y{static_cast<uint64_t>(t[6]), t[7], t[8], t[9], t[10], t[11]};
    std::printf("%d\n", ltd::runs_meet(x, y) ? 1 : 0);
  }
}
"""


@pytest.fixture(scope="module")
def meet(tmp_path_factory):
    d = tmp_path_factory.mktemp("runs")
    (d / "driver.cpp").write_text(DRIVER)
    subprocess.run(["g++", "-O2", "-std=c++17", "-I", CSRC, "-o", str(d / "driver"), str(d / "driver.cpp")], check=True)

    def ask(pairs):
        text = "\n".join(" ".join(map(str, x + y)) for x, y in pairs)
        out = subprocess.run([str(d / "driver")], input=text, capture_output=True, text=True, check=True).stdout.split()
        assert len(out) == len(pairs)
        return [o == "1" for o in out]
    return ask


def covered(t):
    at, rows, row, heads, head, run = t
    return {at + r * row + h * head + i for r in range(rows) for h in range(heads) for i in range(run)}


def drawn(rng, same):
    """Two tensors near each other; same: "both" strides, the "rows"' or "none"."""
    rows, row, head = rng.randint(1, 5), rng.choice([-24, 0, 3, 16, 24, 25]), rng.choice([-4, 0, 1, 4, 5, 50])
    x = (1000, rows, row, rng.randint(1, 4), head, rng.randint(1, 5))
    y = (1000 + rng.randint(-130, 130), rng.choice([rows, rng.randint(1, 5)]), row if same != "none" else rng.choice([0, 7, 24]),
         rng.randint(1, 4), head if same == "both" else rng.choice([0, 2, 6]), rng.randint(1, 5))
    return x, y


@pytest.mark.parametrize("same", ["both", "rows", "none"])
def test_against_sets(meet, same):
    rng = random.Random(same)
    pairs = [drawn(rng, same) for _ in range(6000)]
    wrong = loose = 0
    for (x, y), said in zip(pairs, meet(pairs)):
        true = bool(covered(x) & covered(y))
        assert said or not true, (x, y)  # never apart where they share a byte
        loose += said and not true
        if same == "both":
            assert said == true, (x, y)
    assert loose < len(pairs) / 2


@pytest.mark.parametrize("x, y, want", [
    ((0, 8, 1152, 8, 128, 128), (1024, 8, 1152, 1, 128, 128), False),   # a key head behind eight query heads in each row
    ((0, 8, 1152, 8, 128, 128), (1023, 8, 1152, 1, 128, 128), True),
    ((0, 8, 2048, 8, 256, 128), (128, 8, 2048, 8, 256, 128), False),    # heads in turn
    ((0, 8, 2048, 8, 256, 128), (127, 8, 2048, 8, 256, 128), True),
    ((0, 8, 2048, 8, 256, 128), (128 + 16384, 8, 2048, 8, 256, 128), False),
    ((0, 8, 4160, 8, 256, 128), (2048, 8, 4160, 8, 128, 128), False),   # different head strides, rows' parts apart
    ((0, 8, 4160, 8, 256, 128), (1919, 8, 4160, 8, 128, 128), True),
    ((1 << 62, 2**31 - 2, 1 << 60, 4, 64, 64), (128 + (1 << 62), 2**31 - 2, 1 << 60, 4, 64, 64), True),
    ((1 << 62, 2**31 - 2, 1 << 60, 4, 64, 64), (256 + (1 << 62), 2**31 - 2, 1 << 60, 4, 64, 64), False)])
def test_layouts(meet, x, y, want):
    assert meet([(x, y), (y, x)]) == [want, want]


@pytest.mark.parametrize("same", ["both", "rows", "none"])
def test_the_bindings_form(same):
    rng = random.Random(same + "b")
    for _ in range(4000):
        x, y = drawn(rng, same)
        rows, heads, run = x[1], x[3], x[5]
        y = (y[0], rows, y[2], heads, y[4], run)
        if x[2] < 0 or x[4] < 0 or y[4] < 0:  # (torch has no such strides)
            continue
        true = bool(covered(x) & covered(y))
        said = ltd._heads_meet(y[0] - x[0], rows, x[2], y[2], heads, x[4], y[4], run)
        assert said or not true, (x, y)
        if same == "both" and x[2] > 0:
            assert said == true, (x, y)
