"""How the uniform cache's many-row attention counts its work: a 128-row block's units follow the tiles that it goes over, with
windows, first tokens and both.  Read from the built source, compiled for the host (CPU only).

Units of a block are its tiles + 4, counted along a line between two ends.  Each end and each block's own count are off by at most
one tile at either of their borders, the line's integer division by one: 4 altogether.  Where 128 is no multiple of G,
blocks are taken as ceil(128 / G) tokens long, which makes the line's slope ceil(128 / G) G / 128 times what it is.
"""
import math
import os
import shutil
import subprocess

import pytest

from paper_2412_03131_amd import build

PROGRAM = r"""
#include <cstdio>
#include <cstring>
#include "block_units.hpp"
int main()
{
    int G, window, sinks, n, L;
    while (scanf("%d %d %d %d %d", &G, &window, &sinks, &n, &L) == 5) {
        dkv::BlockAttnArgs a;
        memset(&a, 0, sizeof(a));
        a.G = G;
        a.window = window;
        a.sinks = sinks;
        const dkv::TileUnits u = dkv::tile_units(a, n, L);
        printf("%d", u.blocks);
        for (int i = 0; i < u.blocks; ++i) printf(" %lld", u.upto(i + 1) - u.upto(i));
        printf("\n");
    }
}
"""
NONE = 2 ** 31 - 1
CASES = [(4, NONE, 0, 2048, 0), (8, NONE, 0, 2048, 8192), (1, NONE, 0, 5000, 77), (4, 64, 2048, 2048, 0), (4, 33, 128, 512, 0),
         (4, 4096, 128, 2000, 3000), (8, 512, 500, 3000, 100), (1, 1000, 3000, 9000, 500), (4, 64, 2048, 2048, 1900),
         (4, 64, 2048, 1024, 5000), (2, 256, 200, 4000, 300), (7, 300, 1000, 3000, 0), (33, 100, 64, 800, 10),
         (48, 90, 300, 600, 0), (64, 1, 1, 300, 0), (4, 1, NONE, 1000, 10), (4, 10 ** 9, 10 ** 9, 1000, 0), (5, 45, 5, 30, 3)]


def tiles(G, window, sinks, n, L, block):
    """Tiles with a key that some row of the block sees, from the definition (whole tiles of first tokens count)."""
    first, last = L + block * 128 // G, L + (min(n * G, (block + 1) * 128) - 1) // G
    near = set(range(max(0, first + 1 - window) // 32, last // 32 + 1))
    return len(near | set(range(min(-(-sinks // 32), last // 32 + 1))))


@pytest.mark.skipif(not shutil.which(build.HIPCC), reason="no hipcc")
def test_units_follow_tiles(tmp_path):
    src, exe = str(tmp_path / "units.cpp"), str(tmp_path / "units")
    with open(src, "w") as f:
        f.write(PROGRAM)
    subprocess.run([build.HIPCC, "-x", "hip", "--offload-host-only", "-std=c++17", "-O1", "-I", build.CSRC, "-I",
                    os.path.join(os.path.dirname(build.HERE), "include"), src, "-o", exe], check=True, capture_output=True)
    out = subprocess.run([exe], input="\n".join(" ".join(map(str, c)) for c in CASES), text=True, check=True,
                         capture_output=True).stdout.splitlines()
    assert len(out) == len(CASES)
    for case, line in zip(CASES, out):
        G, window, sinks, n, L = case
        blocks, *units = map(int, line.split())
        assert blocks == len(units) == -(-n * G // 128)
        want = [tiles(*case, i) for i in range(blocks)]
        steeper = math.ceil(128 / G) * G / 128 - 1
        slack = 4 + steeper * (max(want) - min(want))
        off = [u - 4 - w for u, w in zip(units, want)]
        assert max(map(abs, off)) <= slack, (case, off)
