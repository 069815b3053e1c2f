"""How long tc_attn_chunk's warps wait for one another, without a GPU."""
import os
import subprocess

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

WAITS_CHECK = r"""
#include <stdio.h>
#include <initializer_list>
#include "attn_chunk_split.h"
using namespace tc;
int main() {
    // 7.1 us a tile of 128 keys and 3.1 of 64 are the slowest measured; clocks may be a half of those, and memory slower than the L2 they were read from
    for (int32_t len = 1; len <= 1 << 24; len += len / 7 + 1)
        for (int window : {1, 1000, 1 << 22, 1 << 30})
            for (int keys : {64, 128}) {
                const ChunkShape s = chunk_shape(4, keys == 64 ? 128 : 256, keys, window, 0, 8);
                const int32_t tiles = chunk_tiles(s, len);
                const double slow = tiles * (keys == 64 ? 3.1e-6 : 7.1e-6);
                if (chunk_patience(tiles) < 4 * slow) return printf("%d tiles: %d seconds for %f s\n", tiles, chunk_patience(tiles), slow), 1;
            }
    // what a serving program meets is still given up after a second
    if (chunk_patience(16383) != 1) return printf("short items\n"), 1;
    printf("ok\n");
    return 0;
}
"""


def test_a_warp_waits_long_enough_for_the_longest_item(tmp_path):
    src, exe = tmp_path / "waits.cpp", tmp_path / "waits"
    src.write_text(WAITS_CHECK)
    subprocess.check_call(["g++", "-std=c++17", "-O1", "-Wall", "-Wextra", "-I", os.path.join(ROOT, "paper_2608_06007_b200", "csrc"), str(src), "-o", str(exe)])
    assert subprocess.check_output([str(exe)], text=True) == "ok\n"
