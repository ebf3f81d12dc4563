"""The ring of tiles of the chunk attention's copying warps, on the CPU: whatever copies are under way when a block is ended
early are among those that the block then waits for.  The rule is the header that the kernel includes, compiled for the host."""
import os
import random
import subprocess

import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2606_03077_b200", "csrc")
MAIN = r"""
#include <cstdio>
#include "chunk_ring.hpp"
int main() {
  int next, n;
  std::printf("%d\n", libra::kChunkLoaders);
  while (std::scanf("%d %d", &next, &n) == 2) {
    for (int t = libra::ring_newest(next); libra::ring_may_fly(t, next, n); t = libra::ring_before(t)) std::printf("%d ", t);
    std::printf("\n");
  }
}
"""


@pytest.fixture(scope="module")
def rule(tmp_path_factory):
    """{(next tile of a warp, stages): the tiles that are waited for}, and the number of copying warps."""
    d = tmp_path_factory.mktemp("ring")
    (d / "main.cpp").write_text(MAIN)
    subprocess.run(["g++", "-std=c++17", "-Wall", "-Werror", "-I", CSRC, str(d / "main.cpp"), "-o", str(d / "main")], check=True)
    keys = [(i, n) for i in range(60) for n in range(3, 10)]
    r = subprocess.run([str(d / "main")], input="".join(f"{i} {n}\n" for i, n in keys), capture_output=True, text=True, check=True)
    lines = r.stdout.split("\n")
    return {k: [int(x) for x in line.split()] for k, line in zip(keys, lines[1:])}, int(lines[0])


def test_everything_under_way_is_waited_for(rule):
    waited, warps = rule
    rng = random.Random(1)
    older = 0   # states with a copy further back than one ring from the warp's next tile
    for _ in range(4000):
        n, tiles = rng.randint(3, 9), rng.randint(1, 40)
        following, landed, used = list(range(warps)), set(), 0
        weights = [rng.random() ** 3 + 1e-3 for _ in range(3)]
        for _ in range(rng.randint(0, 4 * tiles)):
            step = rng.choices(("ask", "land", "use"), weights)[0]
            flying = [t for w in range(warps) for t in range(w, following[w], warps) if t not in landed]
            if step == "ask":
                w = rng.randrange(warps)
                if following[w] < tiles and following[w] - n < used:   # the place's tile before has been used
                    following[w] += warps
            elif step == "land" and flying:
                landed.add(rng.choice(flying))
            elif step == "use" and used in landed:                     # in order
                used += 1
        for w in range(warps):
            flying = [t for t in range(w, following[w], warps) if t not in landed]
            got = waited[(following[w], n)] if following[w] >= warps else []
            assert set(flying) <= set(got), (n, following, used, flying, got)
            assert all(0 <= t < following[w] and t % warps == w for t in got)
            older += any(t < following[w] - n for t in flying)
    assert older > 0


def test_no_tile_is_waited_for_twice_at_one_place(rule):
    waited, warps = rule
    for (following, n), tiles in waited.items():
        assert len({t % n for t in tiles}) == len(tiles) and tiles == sorted(tiles, reverse=True)
