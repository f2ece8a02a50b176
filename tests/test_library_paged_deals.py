"""How tiles of 128 rows are cut into parts (csrc/paged_cut.h, compiled here as plain C++): no more parts than there are records for, whatever the lengths."""
import os
import random
import shutil
import subprocess

import pytest

import paged_deals as deals
from paper_2605_18753_amd import binding as B

pytestmark = pytest.mark.skipif(not shutil.which("g++"), reason="no host compiler")

PROGRAM = r"""
#include <cstdio>
#include <vector>
#include "paged_cut.h"
using namespace dash;
// lines: four wgs slots gain, sequences, (tiles cost) of each -> size, whole, parts
int main() {
  int four, wgs, slots, n;
  float gain;
  while (std::scanf("%d %d %d %f %d", &four, &wgs, &slots, &gain, &n) == 5) {
    std::vector<int> tiles(n), cost(n);
    int items = 0;
    float sum = 0.f, most = 0.f, rest = 0.f;
    for (int i = 0; i < n; i++) {
      if (std::scanf("%d %d", &tiles[i], &cost[i]) != 2) return 1;
      for (int k = 0; k < tiles[i]; k++)
        if (items + k >= slots / 2) rest += (float)cost[i];
      items += tiles[i];
      sum += (float)tiles[i] * (float)cost[i];
      if (tiles[i] && (float)cost[i] > most) most = (float)cost[i];
    }
    const PagedCut c = four ? paged_cut<true>(wgs, slots, gain, items, sum, most, rest) : paged_cut<false>(wgs, slots, gain, items, sum, most, rest);
    long parts = 0;
    int before = 0;
    for (int i = 0; i < n; i++)
      for (int k = 0; k < tiles[i]; k++, before++) parts += before < c.whole ? 1 : (cost[i] + c.size - 1) / c.size;
    std::printf("%d %d %ld\n", c.size, c.whole, parts);
  }
}
"""


@pytest.fixture(scope="module")
def cut(tmp_path_factory):
    at = tmp_path_factory.mktemp("cut")
    (at / "cut.cpp").write_text(PROGRAM)
    subprocess.run(["g++", "-std=c++17", "-O1", "-ffp-contract=off", "-I", os.path.join(os.path.dirname(B.__file__), "csrc"), str(at / "cut.cpp"), "-o", str(at / "cut")], check=True, timeout=120)

    def run(calls):
        text = "\n".join(f"{int(four)} {wgs} {slots} {gain} {len(seqs)} " + " ".join(f"{t} {c}" for t, c in seqs) for four, wgs, slots, gain, seqs in calls)
        out = subprocess.run([str(at / "cut")], input=text, capture_output=True, text=True, timeout=100, check=True).stdout
        return [tuple(int(x) for x in line.split()) for line in out.splitlines()]
    return run


def test_the_calls_of_the_gpu_tests_are_cut_in_every_way(cut):
    calls = [(True, *deals.room(*deal[:5])) for deal in deals.DEALS]
    assert all(wgs > 0 for _, wgs, *_ in calls)
    got = [deals.way(four, wgs, slots, c, seqs) for (four, wgs, slots, _, seqs), c in zip(calls, cut(calls))]
    assert got == [deal[5] for deal in deals.DEALS]


def test_parts_never_outnumber_their_records(cut):
    rng = random.Random(1)
    calls = []
    for t in range(30000):
        four, slots = rng.random() < 0.6, max(rng.choice([256, 512, 768]) // rng.randint(1, 128), 1)
        n = rng.choice([1, 1, 1, 2, 3, rng.randint(1, 70)])
        same = rng.randint(1, 1 << rng.randint(1, 18))
        seqs = [(rng.choice([1, rng.randint(0, 2 * slots)]) if n < 4 else rng.randint(0, 3), same if rng.random() < 0.5 else rng.randint(1, 1 << rng.randint(1, 18))) for _ in range(n)]
        items = sum(x for x, _ in seqs)
        most = items + rng.randint(0, n)                         # what the host takes for them: no fewer
        if most >= 2 * slots:
            continue
        calls.append((four, most + slots * 3 // 2 if most * 4 >= slots else slots, slots, rng.choice([0.65, 0.9]), seqs))
    ways = {}
    for (four, wgs, slots, gain, seqs), c in zip(calls, cut(calls)):
        items = sum(x for x, _ in seqs)
        assert c[2] <= wgs or c[2] == items, (four, wgs, slots, gain, seqs, c)   # what is not cut needs no record
        key = (four, deals.way(four, wgs, slots, c, seqs))
        ways[key] = ways.get(key, 0) + 1
    assert all(ways.get((True, w), 0) > 50 for w in ("once", "twice", "whole", "fine", "even", "none")), ways
    assert all(ways.get((False, w), 0) > 50 for w in ("whole", "fine", "even", "none")), ways
