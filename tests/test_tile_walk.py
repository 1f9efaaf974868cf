"""The walk over a batch's tiles (csrc/tile_walk.cuh), compiled for the host: every tile once, whatever the number of entries, and an end."""
import os
import shutil
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CODE = r"""
#include <cstdio>
#include <cstdlib>
#include "tile_walk.cuh"
// the walker `first` of `step` over entries * per tiles, from its last `keep` tiles on: prints what it visits and where it ends
int main(int argc, char **argv)
{
    const long long first = atoll(argv[1]), step = atoll(argv[2]), entries = atoll(argv[3]), keep = atoll(argv[5]);
    const int per = atoi(argv[4]);
    const long long tiles = entries * per, mine = first < tiles ? (tiles - first + step - 1) / step : 0, skip = mine > keep ? mine - keep : 0;
    hn::TileWalk w(first + skip * step, step, per);
    w.step_b = hn::TileWalk(first, step, per).step_b; w.step_r = hn::TileWalk(first, step, per).step_r;
    long long n = 0;
    for (; w.inside((int)entries) && n <= keep + 4; w.next(), ++n) printf("%u %d\n", w.b, w.r);
    hn::TileWalk ahead = w;
    ahead.next();                                            // what is fetched for the tile behind the last
    printf("end %d %d\n", (int)w.inside((int)entries), (int)ahead.inside((int)entries));
}
"""


@pytest.fixture(scope="module")
def walk(tmp_path_factory):
    if not shutil.which("g++"):
        pytest.skip("no host compiler")
    d = tmp_path_factory.mktemp("walk")
    (d / "walk.cpp").write_text(CODE)
    subprocess.run(["g++", "-O2", "-std=c++17", "-fsanitize=undefined", "-fno-sanitize-recover", "-I", os.path.join(ROOT, "paper_2607_19378_b200", "csrc"),
                    str(d / "walk.cpp"), "-o", str(d / "walk")], check=True)
    return lambda *a: subprocess.run([str(d / "walk")] + [str(x) for x in a], capture_output=True, text=True, check=True).stdout.splitlines()


@pytest.mark.parametrize("entries,per,step", [(1, 1, 1), (3, 7, 4), (5, 1, 592), (70, 3, 148), (1000, 2, 592), (2, 5000, 592), (2 ** 31 - 1, 1, 592),
                                              (2 ** 31 - 1, 1, 1), (2 ** 31 - 1, 3, 592), (2 ** 31 - 1183, 1, 591), (2 ** 31 - 1, 2, 65)])
def test_every_tile_once(walk, entries, per, step):
    tiles, keep = entries * per, 20
    for first in sorted({0, 1, min(step, tiles) // 2, min(step, tiles) - 1}):
        if not 0 <= first < min(step, tiles):
            continue
        mine = range(first, tiles, step)
        want = ["%d %d" % divmod(t, per) for t in mine[max(0, len(mine) - keep):]]
        assert walk(first, step, entries, per, keep) == want + ["end 0 0"]
