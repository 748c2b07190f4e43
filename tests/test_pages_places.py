"""The integers of paged attention (csrc/places.h), built for the host: chunks of all units' tiles,
against the same sums without a width."""
import os
import random
import shutil
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
MAIN = r"""
#include <stdio.h>
#include <string.h>
#include "places.h"
using namespace certkv;
int main() {
  char what[16];
  while (scanf("%15s", what) == 1) {
    if (!strcmp(what, "cut")) {
      unsigned copies, tiles, parts, most;
      scanf("%u %u %u %u", &copies, &tiles, &parts, &most);
      const PgCut c = pg_cut(copies, tiles, parts, most);
      printf("%u %u %d\n", c.tiles, c.total, (int)c.fits);
    } else if (!strcmp(what, "tiles")) {
      long long rows;
      unsigned lists;
      int gap;
      scanf("%lld %u %d", &rows, &lists, &gap);
      printf("%u\n", pg_tiles(rows, lists, gap));
    } else {
      unsigned x, y;
      scanf("%u %u", &x, &y);
      printf("%u\n", pg_add(x, y));
    }
  }
}
"""
MOST = 2 ** 31 - 1  # tiles of all units are fewer


@pytest.fixture(scope="module")
def ask(tmp_path_factory):
    if not shutil.which("g++"):
        pytest.skip("g++ not available")
    d = tmp_path_factory.mktemp("places")
    (d / "main.cc").write_text(MAIN)
    subprocess.run(["g++", "-O1", "-Wall", "-fsanitize=undefined", "-fno-sanitize-recover=all",
                    "-D__host__=", "-D__device__=", "-D__forceinline__=inline", "-I",
                    os.path.join(ROOT, "paper_2608_21541_amd", "csrc"), "-o", str(d / "main"),
                    str(d / "main.cc")], check=True)

    def run(lines):
        r = subprocess.run([str(d / "main")], input="\n".join(lines), capture_output=True, text=True,
                           check=True)
        return [tuple(int(x) for x in line.split()) for line in r.stdout.splitlines()]
    return run


def sizes(rng, top):
    return rng.choice([rng.randint(1, 40), int(2 ** rng.uniform(0, top)), 2 ** top - 1])


def test_chunks(ask):
    rng = random.Random(1)
    cases = [(640, 2048 * (105000 // 32 + 9), 512, 10000),  # (lists that share pages)
             (1, MOST - 1, 512, 1), (1, MOST, 512, 1), (2, 2 ** 30 - 1, 512, 7), (2, 2 ** 30, 512, 7)]
    cases += [(sizes(rng, 22), sizes(rng, 31), sizes(rng, 11), sizes(rng, 20)) for _ in range(4000)]
    some = 0
    for (copies, tiles, parts, most), (k, total, fits) in zip(cases, ask(
            ["cut %d %d %d %d" % c for c in cases])):
        want = copies * tiles
        assert fits == (want < MOST) and total == (want if fits else 0)
        assert k >= 4 and k % 4 == 0
        # partials have room for the chunks, all begin and end within 32 bits, and they are no
        # shorter than the parts make them
        n = -(-total // k)
        assert n <= most and n * k < 2 ** 32
        if fits and most >= parts:
            assert n <= max(parts, -(-total // 512))
            some += 1
    assert some > 500


def test_tiles_of_the_lists(ask):
    rng = random.Random(2)
    cases = [(rng.choice([-1, 1, 1, 1]) * int(2 ** rng.uniform(0, 62.9)), sizes(rng, 30),
              rng.choice([8, 16])) for _ in range(3000)]
    cases += [(2 ** 63 - 1, 1, 8), (-2 ** 63, 1, 8), (0, 1, 8), (-1, 1, 8)]
    for (rows, lists, gap), (got,) in zip(cases, ask(["tiles %d %d %d" % c for c in cases])):
        assert got == (min(MOST, -(-rows // 32) + lists * gap) if rows >= 0 else MOST)


def test_sums_that_stop(ask):
    cases = [(x, y) for x in (0, 1, 77, 2 ** 30, MOST - 1, MOST) for y in (0, 1, 2 ** 30, MOST - 1, MOST)]
    for (x, y), (got,) in zip(cases, ask(["add %d %d" % c for c in cases])):
        assert got == min(MOST, x + y)
