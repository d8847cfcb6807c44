"""The node groups that a launch of the sampling rules makes (csrc/rules_plan.hpp, built for the host with g++)."""
import os
import subprocess

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2603_01639_amd", "csrc")
CHUNK = {True: 16384, False: 4096}  # tokens of a workgroup: argmax, written rows
THREADS = {True: 1024, False: 256}

DRIVER = r"""
#include <cstdio>
#include "rules_plan.hpp"
int main() {
  int B, N, chunks, argmax, threads, cus;
  while (std::scanf("%d %d %d %d %d %d", &B, &N, &chunks, &argmax, &threads, &cus) == 6)
    std::printf("%d\n", ltd::rules::nodes(B, N, chunks, argmax != 0, threads, cus));
  return 0;
}
"""


def build(folder):
    """The program's path, built in `folder` (a pathlib path)."""
    (folder / "rules.cpp").write_text(DRIVER)
    exe = folder / "rules"
    subprocess.run(["g++", "-std=c++17", "-O1", "-I", CSRC, str(folder / "rules.cpp"), "-o", str(exe)], check=True)
    return str(exe)


def nodes(exe, B, N, voc, argmax, cus=256):
    """Nodes of a workgroup for B trees of up to N nodes and voc tokens."""
    text = f"{B} {N} {-(-voc // CHUNK[argmax])} {int(argmax)} {THREADS[argmax]} {cus}"
    r = subprocess.run([exe], input=text, capture_output=True, text=True, timeout=20, check=True)
    return int(r.stdout)
