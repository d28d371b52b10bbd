"""The arithmetic that cuts a call's visible rows into units, compiled for the host and compared with whole numbers of any
size: a unit is at least one step, covers its share of the rows, and no sequence is left without units."""

import os
import random
import shutil
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2409_03856_amd", "csrc")
STEP, MOST = 128, (1 << 20) + 32

PROGRAM = """
#include <cstdio>
#include "paged_plan.h"
int main() {
  long rows;
  int span;
  while (std::scanf("%ld %d", &rows, &span) == 2) {
    const int every = sirius::whole_steps(rows);
    std::printf("%d %d\\n", every, every > 0 ? sirius::units_of(span, every) : -1);
  }
}
"""


@pytest.mark.skipif(shutil.which("g++") is None, reason="no g++")
def test_units_of_any_total(tmp_path):
    src, exe = tmp_path / "plan.cpp", tmp_path / "plan"
    src.write_text(PROGRAM)
    subprocess.run(["g++", "-std=c++17", "-Wall", "-Werror", "-I", CSRC, str(src), "-o", str(exe)], check=True, timeout=120)
    rng = random.Random(1)
    totals = [0, 1, 127, 128, 129, MOST - 1, MOST, MOST + 1, 2 ** 31 - 128, 2 ** 31 - 1, 2 ** 31, 2 ** 32 - 1, 2 ** 32, 2 ** 32 + 1,
              65535 * 2 ** 20 // 2, 65535 * 2 ** 20] + [int(2 ** rng.uniform(0, 36)) for _ in range(3000)]
    spans = [rng.choice((0, 1, MOST, rng.randint(1, MOST))) for _ in totals]
    lines = "\n".join(f"{t} {s}" for t, s in zip(totals, spans))
    out = subprocess.run([str(exe)], input=lines, capture_output=True, text=True, check=True, timeout=60).stdout.split("\n")
    for t, s, line in zip(totals, spans, out):
        every, units = map(int, line.split())
        assert every % STEP == 0 and every >= min(max(t, 1), MOST) and every < min(max(t, 1), MOST) + STEP, (t, every)
        assert units == -(-s // every), (t, s)
