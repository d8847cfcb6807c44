"""How latent attention's work is cut (csrc/latent_plan.hpp), built for the host with g++: the shares cover every tile of
every unit once, divisions are exact, and the count of workgroups is bounded for every size a call takes."""
import os
import random
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2603_01639_amd", "csrc")
TOP = 1 << 30

DRIVER = r"""
#include <cstdio>
#include "latent_plan.hpp"
using namespace ltd::latent;
// stdin: "q x y", "d kv_rows row", "w B Nmax heads max_prefix cus", or "c W Nmax heads B n P n P ..."; one answer a line (for
// c one "sequence unit tile0 tile1" a piece, and a line with -1)
int main() {
  char what;
  while (std::scanf(" %c", &what) == 1) {
    long long x, y;
    int a, b, c, d, e;
    if (what == 'q') {
      if (std::scanf("%lld %lld", &x, &y) != 2) return 2;
      std::printf("%lld\n", static_cast<long long>(quotient(x, y)));
    } else if (what == 'd') {
      if (std::scanf("%d %d", &a, &b) != 2) return 2;
      const RowDivisor r = row_divisor(a);
      const uint32_t top = static_cast<uint32_t>((static_cast<uint64_t>(2u * static_cast<uint32_t>(b)) * r.magic) >> 32);
      std::printf("%u\n", top >> r.shift);
    } else if (what == 'w') {
      if (std::scanf("%d %d %d %d %d", &a, &b, &c, &d, &e) != 5) return 2;
      std::printf("%d\n", workgroups(a, b, c, d, e));
    } else {
      static int n[512], P[512];
      if (std::scanf("%d %d %d %d", &a, &b, &c, &d) != 4) return 2;
      const Cut cut = cut_of(b, c);
      int64_t total = 0;
      for (int i = 0; i < d; ++i) {
        if (std::scanf("%d %d", &n[i], &P[i]) != 2) return 2;
        total += n[i] > 0 ? length_of(P[i], n[i], c, cut) : 0;
      }
      const int64_t share = share_of(total, a, cut);
      for (int w = 0; w < a; ++w) {
        int64_t pos = w * share, before = 0;
        const int64_t end = pos + share < total ? pos + share : total;
        for (int i = 0; i < d && pos < end; ++i) {
          if (n[i] <= 0) continue;
          const int64_t length = cut.cost + tiles_of(P[i], n[i]);
          for (int64_t u = 0; u < units_of(n[i], c, cut) && pos < end; ++u, before += length) {
            if (pos >= before + length) continue;
            const int64_t stop = before + length < end ? before + length : end;
            std::printf("%d %lld %lld %lld\n", i, static_cast<long long>(u), static_cast<long long>(tile_at(pos - before, cut)),
                        static_cast<long long>(tile_at(stop - before, cut)));
            pos = stop;
          }
        }
      }
      std::printf("-1\n");
    }
  }
  return 0;
}
"""


@pytest.fixture(scope="module")
def ask(tmp_path_factory):
    d = tmp_path_factory.mktemp("plan")
    (d / "plan.cpp").write_text(DRIVER)
    subprocess.run(["g++", "-std=c++17", "-O1", "-I", CSRC, str(d / "plan.cpp"), "-o", str(d / "plan")], check=True)

    def run(lines):
        r = subprocess.run([str(d / "plan")], input="\n".join(lines), capture_output=True, text=True, timeout=60)
        assert r.returncode == 0
        return r.stdout.splitlines()
    return run


def test_quotients(ask):
    rng = random.Random(1)
    pairs = [(0, 1), (1, 1), (2**52 - 1, 1), (2**52 - 1, 2**52 - 1), (2**52 - 2, 2**52 - 1)]
    for _ in range(20000):
        y = rng.randrange(1, 1 << rng.randrange(1, 40))
        k = rng.randrange(0, max((2**52 - 2) // y, 1))
        pairs += [(k * y, y), (k * y + y - 1, y), (k * y + rng.randrange(y), y)]
    pairs = [(x, y) for x, y in pairs if x < 2**52]
    got = ask([f"q {x} {y}" for x, y in pairs])
    assert [int(g) for g in got] == [x // y for x, y in pairs]


def test_blocks_of_rows(ask):
    rng = random.Random(2)
    pairs = []
    for R in [1, 2, 3, 5, 7, 16, 24, 48, 63, 64, 65, 127, 1000, 4096, 99991, 2**20 + 1, TOP - 1, TOP, 2**31 - 1] + [
            rng.randrange(1, 2**31) for _ in range(300)]:
        for k in [0, 1, 2, (2**31 - 1) // R, rng.randrange(0, (2**31 - 1) // R + 1)]:
            pairs += [(R, r) for r in (k * R - 1, k * R, k * R + 1, k * R + R - 1) if 0 <= r < 2**31]
        pairs += [(R, 2**31 - 1), (R, rng.randrange(2**31))]
    got = ask([f"d {R} {r}" for R, r in pairs])
    assert [int(g) for g in got] == [r // R for R, r in pairs]


def test_shares_cover_every_tile_once(ask):
    rng = random.Random(3)
    for _ in range(300):
        few = rng.random() < 0.4
        heads, most = rng.choice([(16, 1), (1, 16), (4, 4), (5, 3)] if few else [(16, 60), (128, 1), (128, 5), (17, 1), (3, 256)])
        B = rng.choice([1, 2, 3, 16, 70])
        seqs = [(rng.randrange(0, most + 1), rng.choice([0, 1, 31, 32, 33, 500, 5000])) for _ in range(B)]
        W = rng.choice([1, 2, 7, 8, 100, 256])
        rows = 16 if few else 128
        got = ask([f"c {W} {most} {heads} {B} " + " ".join(f"{n} {P}" for n, P in seqs)])
        assert got.pop() == "-1"
        at = {}
        for line in got:
            b, u, t0, t1 = map(int, line.split())
            assert t0 == at.get((b, u), 0) and t1 >= t0  # in order, without a gap
            at[b, u] = t1
        want = {(b, u): -(-(P + n) // 32) for b, (n, P) in enumerate(seqs) for u in range(-(-n * heads // rows))}
        assert at == want


def test_workgroups(ask):
    cases = [(1, 1, 1, 0, 256), (1, 1, 1, TOP, 256), (1, 256, 65536, TOP, 256), (2**31 - 1, 256, 65536, TOP, 256),
             (2**31 - 1, 1, 1, 0, 256), (2560, 256, 65536, TOP, 256), (2049, 1, 16, TOP, 256), (16, 60, 16, 8192, 256)]
    got = [int(g) for g in ask([f"w {' '.join(map(str, c))}" for c in cases])]
    assert all(1 <= g <= 256 for g in got)
    assert got[0] == 1 and got[1:] == [256] * (len(cases) - 1)
