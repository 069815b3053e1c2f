"""tc_attn_chunk without a GPU: how it cuts its work, what it refuses, its workspace."""
import os
import subprocess

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

SPLIT_CHECK = r"""
#include <stdio.h>
#include <stdlib.h>
#include <vector>
#include "attn_chunk_split.h"
using namespace tc;
static uint32_t seed = 1;
static int pick(int lo, int hi) { seed = seed * 1664525u + 1013904223u; return lo + (int)((seed >> 8) % (uint32_t)(hi - lo + 1)); }
#define FAIL(...) return printf(__VA_ARGS__), printf("\n"), 1
int main() {
    for (int round = 0; round < 3000; round++) {
        const int wide = pick(0, 3) == 0, group = pick(1, 20), window = pick(0, 1) ? pick(1, round % 2 ? 3000 : 100) : 1 << 30, sinks = window < (1 << 30) && pick(0, 1) ? pick(0, 400) : 0;
        const ChunkShape s = chunk_shape(group, wide ? 128 : 256, wide ? 64 : 128, window, sinks, pick(1, 8));
        for (int i = 0; i < 100; i++) {
            const int v = i < 50 ? i : pick(0, 2147483647 >> 1);
            if (chunk_by_group(s, v) != v / group) FAIL("%d / %d", v, group);
        }
        const int R = pick(1, round % 50 == 0 ? 300 : 6), longest = round % 7 == 0 ? 300000 : round % 3 ? 3000 : 300;
        std::vector<int> len(R), n(R);
        int64_t n_tokens = 0, max_new = 1, max_len = 1;
        for (int r = 0; r < R; r++) {
            len[r] = pick(0, longest), n[r] = pick(0, len[r] < 400 ? len[r] : 400);
            n_tokens += n[r];
            if (n[r] > max_new) max_new = n[r];
            if (len[r] > max_len) max_len = len[r];
        }
        if (!n_tokens) continue;
        ChunkPlan plan;
        plan_chunk(s, R, n_tokens, max_new, max_len, 128, &plan);
        // the cut, as the kernel finds it
        int32_t share = 1 << 30, most = 0;
        int64_t uncut = 0;
        for (int r = 0; r < R; r++) if (n[r]) uncut += (int64_t)chunk_blocks(s, n[r]) * s.heads, most = chunk_high(most, chunk_tiles(s, len[r]));
        if (plan.part_rows && uncut < kChunkEnough && most > kChunkLeastShare) {
            float best = 3e38f;
            for (int c = 0; c < kChunkCuts; c++) {
                ChunkCost sum;
                const int32_t sh = chunk_share(most, c);
                const float inverse = 1.f / sh;
                for (int r = 0; r < R; r++) if (n[r]) {
                    const int tiles = chunk_tiles(s, len[r]);
                    const int parts = (int)(((float)(tiles + sh - 1) + 0.5f) * inverse);
                    if (parts != chunk_parts(tiles, sh)) FAIL("parts");
                    sum.add(chunk_blocks(s, n[r]) * s.heads, tiles, sh, parts);
                }
                const float cost = chunk_cost(sum);
                if (cost < best) best = cost, share = sh;
            }
            if (best > 1e38f) FAIL("no cut at all");
        }
        int64_t items = 0, rows = 0;
        for (int r = 0; r < R; r++) {
            if (!n[r]) continue;
            const int tiles = chunk_tiles(s, len[r]), parts = chunk_parts(tiles, share), blocks = chunk_blocks(s, n[r]);
            if (parts > kChunkMostParts) FAIL("%d parts", parts);
            items += (int64_t)blocks * parts * s.heads;
            if (parts > 1) rows += (int64_t)n[r] * s.group * s.heads * parts;
            const int pos0 = len[r] - n[r];
            int covered = 0;
            for (int b = 0; b < blocks; b++) {
                const int row0 = b * s.rows, here = chunk_low(n[r] * s.group - row0, s.rows);
                if (here < 1) FAIL("an empty block");
                covered += here;
                const ChunkList l = chunk_list(s, pos0, row0, here, 128);
                if (l.count > tiles || l.count < 1 || (int64_t)parts * share < l.count) FAIL("%d tiles of %d", l.count, tiles);
                if (l.firsts < 0 || l.skip < 0 || l.key_end > len[r] || l.key_low < 0) FAIL("list");
                // what each row sees lies in tiles that its slot takes, and a tile is taken by some slot
                for (int i = 0; i < l.count; i++) {
                    const bool s0 = i < l.end0, s1 = here > 128 && (i < l.firsts || i >= l.begin1);
                    if (!s0 && !s1) FAIL("a tile for nobody");
                }
                for (int row = row0; row < row0 + here; row += pick(1, 40)) {
                    const int p = pos0 + row / s.group, slot = row - row0 >= 128;
                    if (p < 0 || p >= len[r]) FAIL("position");
                    for (int j : {0, s.sinks - 1, s.sinks, p - s.window, p - s.window + 1, p, p / 2, p - 1, p + 1}) {
                        const bool seen = j >= 0 && j <= p && (j > p - s.window || j < s.sinks);
                        if (!seen) continue;
                        if (j >= l.key_end || (j < l.key_low && j >= s.sinks)) FAIL("a key is not read");
                        const int tile = j / s.keys, i = tile < l.firsts ? tile : tile - l.skip;
                        if (i < 0 || i >= l.count || (i >= l.firsts) != (tile >= l.firsts)) FAIL("a tile is not listed");
                        const bool taken = slot ? (i < l.firsts || i >= l.begin1) : i < l.end0;
                        if (!taken) FAIL("a tile is not taken: row %d of %d, key %d", row, here, j);
                    }
                }
            }
            if (covered != n[r] * s.group) FAIL("rows");
        }
        if (items > plan.grid) FAIL("%lld items for a grid of %lld", (long long)items, (long long)plan.grid);
        if (rows > plan.part_rows) FAIL("%lld rows of parts, room for %lld", (long long)rows, (long long)plan.part_rows);
    }
    printf("ok\n");
    return 0;
}
"""


def test_the_cut_covers_every_key_of_every_row_and_fits_its_grid_and_workspace(tmp_path):
    src, exe = tmp_path / "split.cpp", tmp_path / "split"
    src.write_text(SPLIT_CHECK)
    subprocess.check_call(["g++", "-std=c++17", "-O1", "-Wall", "-Wextra", "-fsanitize=undefined,address", "-fno-sanitize-recover", "-I", os.path.join(ROOT, "paper_2608_06007_b200", "csrc"), str(src), "-o", str(exe)])
    assert subprocess.check_output([str(exe)], text=True) == "ok\n"
