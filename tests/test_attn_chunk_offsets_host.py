"""tc_attn_chunk's workspace without a GPU: offsets that decrease, so that requests share tokens, write no further than it reaches."""
import os
import subprocess

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

ROOM_CHECK = r"""
#include <stdio.h>
#include <vector>
#include "attn_chunk_split.h"
using namespace tc;
static uint32_t seed = 1;
static int pick(int lo, int hi) { seed = seed * 1664525u + 1013904223u; return lo + (int)((seed >> 8) % (uint32_t)(hi - lo + 1)); }
#define FAIL(...) return printf(__VA_ARGS__), printf("\n"), 1
int main() {
    long past = 0;
    for (int round = 0; round < 4000; round++) {
        const bool shared = round & 1;  // requests lie over one another: offsets 0, n, 0, n, ..
        const int heads = pick(1, 4), group = pick(1, 16);
        const ChunkShape s = chunk_shape(group, 256, 128, 1 << 30, 0, heads);
        // requests of `from` tokens or more have their tiles made fp16, of which a call plans no more than n_tokens / from
        const int from = 512 / group + 1, each = from + pick(0, 200), live = pick(1, 60);
        const int64_t n_tokens = shared ? each + pick(0, each) : (int64_t)each * live, R = shared ? 2 * live : live, len = each + pick(0, 5000);
        const int64_t planned = R < n_tokens / from ? R : n_tokens / from;
        ChunkPlan plan;
        plan_chunk(s, planned, n_tokens, each, len, 128, &plan);
        if (!plan.part_rows) continue;
        // the cut, as the kernel finds it
        int32_t share = 1 << 30;
        const int64_t uncut = (int64_t)live * chunk_blocks(s, each) * heads;
        const int32_t tiles = chunk_tiles(s, (int32_t)len);
        if (uncut < kChunkEnough && tiles > kChunkLeastShare) {
            float best = 3e38f;
            for (int c = 0; c < kChunkCuts; c++) {
                ChunkCost sum;
                const int32_t sh = chunk_share(tiles, c);
                for (int r = 0; r < live; r++) sum.add(chunk_blocks(s, each) * heads, tiles, sh, chunk_parts(tiles, sh));
                const float cost = chunk_cost(sum);
                if (cost < best) best = cost, share = sh;
            }
        }
        const int32_t parts = tiles > share ? chunk_parts(tiles, share) : 1;
        if (parts == 1) continue;
        const int64_t rows = (int64_t)each * group * heads * parts * live;
        if (chunk_has_room(plan.part_rows, rows) != (rows <= plan.part_rows)) FAIL("room");
        if (rows <= plan.part_rows) continue;
        if (!shared) FAIL("no room for %lld rows though offsets do not decrease", (long long)rows);
        past++;
    }
    if (!past) FAIL("no batch that shares tokens is larger than its plan");
    printf("ok\n");
    return 0;
}
"""


def test_requests_that_share_tokens_write_within_the_workspace(tmp_path):
    src, exe = tmp_path / "room.cpp", tmp_path / "room"
    src.write_text(ROOM_CHECK)
    subprocess.check_call(["g++", "-std=c++17", "-O1", "-Wall", "-Wextra", "-fsanitize=undefined,address", "-fno-sanitize-recover", "-I", os.path.join(ROOT, "paper_2608_06007_b200", "csrc"), str(src), "-o", str(exe)])
    assert subprocess.check_output([str(exe)], text=True) == "ok\n"
