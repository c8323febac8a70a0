"""The tile rule of the 8-bit product (csrc/linear_fp8_tiles.h), compiled on its
own: no GPU.  The GPU tests of every tile rely on the tiles checked here."""
import subprocess

import pytest

from paper_2607_01817_amd import build
from tests import fp8_shapes as fs

DRIVER = r"""
#include <cstdio>
#include "linear_fp8_tiles.h"
using namespace hcms;
template <int C> void tell(const Fp8TileCost (&t)[C], long long M, long long N, long long K, long long n_cu) {
    const Fp8TileCost &c = t[fp8_tile(t, M, N, K, n_cu)];
    std::printf("%d %d %d %d %d\n", c.bm, c.bn, c.groups, c.per_cu, M <= kFp8Rows ? 1 + fp8_rows_wide(N, n_cu) : 0);
}
int main() {
    long long M, N, K, n_cu;
    int wide;
    while (std::scanf("%lld %lld %lld %d %lld", &M, &N, &K, &wide, &n_cu) == 5)
        if (wide) tell(kFp8WideTiles, M, N, K, n_cu);
        else tell(kFp8Tiles, M, N, K, n_cu);
}
"""


@pytest.fixture(scope="module")
def tiles(tmp_path_factory):
    d = tmp_path_factory.mktemp("fp8tiles")
    (d / "driver.cpp").write_text(DRIVER)
    subprocess.run(["g++", "-std=c++17", "-Wall", "-Werror", "-I", build.CSRC, str(d / "driver.cpp"),
                    "-o", str(d / "driver")], check=True)

    def ask(cases):
        text = "".join(" ".join(map(str, c)) + "\n" for c in cases)
        out = subprocess.run([str(d / "driver")], input=text, text=True, capture_output=True, check=True).stdout
        return [tuple(map(int, ln.split())) for ln in out.splitlines()]

    return ask


def test_shapes_take_every_tile(tiles):
    got = tiles([(M, N, K, int(t == "fp32"), 256) for t, _, _, M, N, K in fs.SHAPES])
    for (t, i, more, M, N, K), (bm, bn, groups, per_cu, few) in zip(fs.SHAPES, got):
        assert (bm, bn, groups) == fs.TILES[t][i] and few == 0, (M, N, K)
        assert (-(-M // bm) * -(-N // bn) > 256 * per_cu) == more, (M, N, K)
    # groups of waves pay for one round mostly
    assert {r[:3] for r in fs.SHAPES} >= {(t, i, m) for t in fs.TILES for i, tile in enumerate(fs.TILES[t])
                                         for m in ((False, True) if tile[2] == 1 else (False,))}


def test_few_rows_take_their_kernel(tiles):
    rows = [(1, 8), (16, 4096), (17, 4096), (64, 4104), (65, 8)]
    got = [t[4] for t in tiles([(M, N, 640, 0, 256) for M, N in rows])]
    assert got == [1, 1, 1, 2, 0]


def test_small_devices_get_a_tile(tiles):
    for bm, bn, groups, per_cu, _ in tiles([(M, N, 64, w, n) for M in (1, 5000) for N in (8, 8000) for w in (0, 1)
                                    for n in (1, 304)]):
        assert (bm, bn, groups) in fs.TILES["bf16"] + fs.TILES["fp32"] and per_cu in (1, 2)
