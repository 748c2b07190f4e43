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
    } else if (!strcmp(what, "lists")) {
      // the pieces of every list's copies, as the join takes them
      int lists, gap;
      unsigned copies, cover, parts, most;
      scanf("%d %u %u %d %u %u", &lists, &copies, &cover, &gap, &parts, &most);
      long long off[64];
      for (int r = 0; r <= lists; ++r) scanf("%lld", off + r);
      const long long base = off[0], rows = off[lists] - base;
      const PgCut c = pg_cut(copies, pg_tiles(rows, lists, gap), parts, most);
      printf("%u", c.tiles);
      for (int r = 0; r < lists; ++r) {
        const long long p0 = off[r] - base, p1 = off[r + 1] - base;
        const bool held = c.fits && pg_held(p0, p1, rows) && p1 > p0;
        const uint32_t n = held ? pg_up(p1 - p0 < cover ? p1 - p0 : cover) : 0;
        const uint32_t span = held ? pg_place(p1, r + 1, gap) - pg_place(p0, r, gap) : 0;
        for (unsigned x = 0; x < copies; ++x) {
          PgPieces y = {0, 0};
          if (held) y = pg_pieces(copies * pg_place(p0, r, gap) + x * span, n, c.tiles);
          printf(" %u %u", y.first, y.n);
        }
      }
      printf("\n");
    } else if (!strcmp(what, "list")) {
      long long p0, p1, rows;
      scanf("%lld %lld %lld", &p0, &p1, &rows);
      printf("%u\n", pg_list_tiles(p0, p1, rows));
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


def test_tiles_of_a_list(ask):
    # from its first row to the next one's, where 32 bits do not hold them either
    rng = random.Random(3)
    far = lambda: rng.choice([0, int(2 ** rng.uniform(0, 62.9)), 2 ** rng.randint(30, 62)])  # noqa: E731
    cases = [(0, 2 ** 37, 2 ** 37 + 70), (0, 2 ** 37 + 70, 2 ** 37 + 70), (2 ** 37, 2 ** 37 + 50, 2 ** 38),
             (-1, 5, 5), (6, 5, 9), (0, 6, 5), (0, 2 ** 63 - 1, 2 ** 63 - 1), (0, 2 ** 36 - 1, 2 ** 36)]
    for _ in range(3000):
        p0 = rng.choice([1, 1, 1, -1]) * far()
        p1 = p0 + rng.choice([1, 1, 1, -1]) * rng.choice([far(), rng.randint(0, 99)])
        cases.append((p0, p1, rng.choice([p1, p1 + 5, p1 - 1, far()])))
    cases = [c for c in cases if all(-2 ** 63 <= x < 2 ** 63 for x in c)]
    for (p0, p1, rows), (got,) in zip(cases, ask(["list %d %d %d" % c for c in cases])):
        held = 0 <= p0 <= p1 <= rows
        assert got == (min(MOST, -(-p1 // 32) - -(-p0 // 32)) if held else 0)


def pieces(off, copies, cover, gap, chunk):
    """(first chunk, chunks) of every list's copies, their places counted without a width."""
    up, out = lambda n: -(-n // 32), []  # noqa: E731
    base, end = off[0], off[-1] - off[0]
    place = lambda rows, r: up(rows) + r * gap  # noqa: E731
    fits = end >= 0 and copies * place(end, len(off) - 1) < MOST
    for r in range(len(off) - 1):
        p0, p1 = off[r] - base, off[r + 1] - base
        for x in range(copies):
            if not fits or not 0 <= p0 < p1 <= end:
                out.append((0, 0))
                continue
            at = copies * place(p0, r) + x * (place(p1, r + 1) - place(p0, r))
            first = at // chunk
            out.append((first, (at + up(min(p1 - p0, cover)) - 1) // chunk - first + 1))
    return out


@pytest.mark.parametrize("kind", ["fall", "rise"])
def test_pieces_of_lists(ask, kind):
    # lists below the first offset, behind the last, that fall, and that are as they should be: no
    # partial outside the workspace, and none that two units share
    rng = random.Random(kind)
    cases = [([1000, 488, 1088, 1088, 1088], 1, 2000, 8, 512, 71)] if kind == "fall" else []
    for _ in range(3000):
        n = rng.randint(1, 8)
        step = lambda: int(2 ** rng.uniform(0, rng.choice([4, 12, 40])))  # noqa: E731
        off = [rng.choice([0, step()])]
        for _ in range(n):
            off.append(off[-1] + (rng.choice([1, 1, 1, -1]) if kind == "fall" else 1) * step() * rng.randint(0, 1))
        cases.append((off, rng.choice([1, 2, 16]), rng.choice([64, 2000, 2 ** 31 - 1024]), rng.choice([8, 16]),
                      rng.choice([1, 512, 1024]), rng.choice([1, 71, 5000])))
    lines = ["lists %d %d %d %d %d %d %s" % (len(o) - 1, c, cover, gap, parts, most, " ".join(map(str, o)))
             for o, c, cover, gap, parts, most in cases]
    some = 0
    for (off, copies, cover, gap, parts, most), got in zip(cases, ask(lines)):
        chunk, got = got[0], list(zip(got[1::2], got[2::2]))
        assert got == pieces(off, copies, cover, gap, chunk)
        # partial (chunk + unit): within chunks + units
        kept = [first + u + i for u, (first, n) in enumerate(got) for i in range(min(n, 10 ** 4))]
        assert all(first + n <= most for first, n in got)
        some += len(kept)
        if kind == "rise":
            assert len(set(kept)) == len(kept)
    assert some > 1000


def test_sums_that_stop(ask):
    cases = [(x, y) for x in (0, 1, 77, 2 ** 30, MOST - 1, MOST) for y in (0, 1, 2 ** 30, MOST - 1, MOST)]
    for (x, y), (got,) in zip(cases, ask(["add %d %d" % c for c in cases])):
        assert got == min(MOST, x + y)
