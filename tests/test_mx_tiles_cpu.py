"""The tile that a product of two 4-bit matrices takes, compiled from the header that the library's launch uses (no GPU)."""
import os
import shutil
import subprocess

import mx_gemm_sizes

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

SOURCE = r"""
#include "mx_tiles.h"
#include <cstdio>

int main()
{
    long long tokens, n_out, k_in;
    while (std::scanf("%lld %lld %lld", &tokens, &n_out, &k_in) == 3) {
        const llvq::MxTile& t = llvq::kMxTiles[llvq::mx_tile_of(n_out, tokens, (uint32_t)((k_in + 255) / 256), 148)];
        std::printf("%d %d\n", t.rows, t.tokens);
    }
}
"""


def test_the_sizes_that_are_tested_reach_every_tile(tmp_path):
    src, exe = tmp_path / "t.cpp", tmp_path / "t"
    src.write_text(SOURCE)
    subprocess.check_call([shutil.which("g++") or "c++", "-O1", "-std=c++17", "-I", os.path.join(ROOT, "paper_2603_11021_b200", "csrc"), str(src), "-o", str(exe)])
    cases = [(tile, size) for tile, sizes in mx_gemm_sizes.TILES.items() for size in sizes]
    out = subprocess.run([str(exe)], input="".join("%d %d %d\n" % size for _, size in cases), capture_output=True, text=True, timeout=60, check=True).stdout
    assert [tuple(map(int, line.split())) for line in out.splitlines()] == [tile for tile, _ in cases]
    for (rows, tokens), sizes in mx_gemm_sizes.TILES.items():
        tiles = [-(-n // rows) * -(-t // tokens) for t, n, _ in sizes]
        assert min(tiles) <= 148 < max(tiles)             # one round of tiles and several
        assert any(t % tokens > tokens // 2 for t, _, _ in sizes) and any(0 < t % tokens <= tokens // 2 for t, _, _ in sizes)
        assert any(n % rows for _, n, _ in sizes) and any(k % 256 for _, _, k in sizes)
