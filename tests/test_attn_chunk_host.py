"""tc_attn_chunk without a GPU: how it cuts its work, what it refuses, its workspace."""
import ctypes as C
import os
import subprocess

import pytest
import torch

import paper_2608_06007_b200 as tc
from paper_2608_06007_b200 import binding as b
from test_operators_host import BASE, BOUNDS, INVALID, LAYERS, OVERLAP, SHAPE, TOO_LARGE, call, decode_args, layer

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
        ChunkShape s = chunk_shape(group, wide ? 128 : 256, wide ? 64 : 128, window, sinks, pick(1, 8));
        s.turns = !wide && pick(0, 1);
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
            if (parts > 1) rows += (int64_t)n[r] * s.group * s.heads * parts * (chunk_turns(s, n[r], parts) ? 2 : 1);
            if (chunk_turns(s, n[r], parts) && (blocks > 1 || 2 * parts > kChunkMostParts)) FAIL("turns");
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


# ------------------------------------------------------------------------------------- refusals

def chunk_args(R=3, n=40, Hq=32, D=128, **changes):
    row = D * 2
    a = b.tc_attn_chunk_t(C.sizeof(b.tc_attn_chunk_t), tc.TC_BF16, R, n, Hq, 3 * BASE, 4 * BASE, (C.c_int64 * 2)(Hq * row, row), (C.c_int64 * 2)(Hq * row, row), 5 * BASE, 0.0, 0, 0, 0,
                          6 * BASE, 400, 1600, 7 * BASE, 8 * BASE, 20, 6000, 10 * BASE, 1 << 40)
    for name, value in changes.items():
        setattr(a, name, (C.c_int64 * 2)(*value) if isinstance(value, tuple) else value)
    return a


def window_call(made, args, window, sinks):
    lib = tc.load_library()
    return lib.tc_attn_decode_window(made.ref if made is not None else None, C.byref(args) if args is not None else None, window, sinks, None), lib.tc_last_error().decode()


def test_a_layer_that_makes_no_sense_is_refused():
    plain = decode_args(max_prefix=0)
    for changes, status in LAYERS:
        for rc, why in (call("tc_attn_chunk", layer(**changes), chunk_args()), window_call(layer(**changes), plain, 5, 0)):
            assert rc == status and why, (changes, rc, why)
    assert call("tc_attn_chunk", None, chunk_args())[0] == call("tc_attn_chunk", layer(), None)[0] == INVALID
    assert window_call(None, plain, 5, 0)[0] == window_call(layer(), None, 5, 0)[0] == INVALID
    for D in (8, 72, 272):
        assert call("tc_attn_chunk", layer(D=D), chunk_args(D=D))[0] == window_call(layer(D=D), decode_args(D=D, max_prefix=0), 5, 0)[0] == SHAPE
    assert call("tc_attn_chunk", layer(base=BASE + 8), chunk_args())[0] == INVALID
    assert call("tc_attn_chunk", layer(block_stride=16 * 8 * 128 * 2 + 8), chunk_args())[0] == INVALID


@pytest.mark.parametrize("changes,status", [
    (dict(struct_size=8), INVALID), (dict(dtype=tc.TC_FP32), INVALID), (dict(dtype=tc.TC_FP16), INVALID), (dict(R=-1), SHAPE), (dict(R=1 << 25), SHAPE), (dict(n_tokens=-1), SHAPE), (dict(n_tokens=1 << 31), SHAPE),
    (dict(Hq=12), SHAPE), (dict(Hq=0), SHAPE), (dict(max_len=-1), SHAPE), (dict(max_len=(1 << 24) + 1), SHAPE), (dict(max_new=-1), SHAPE), (dict(max_new=6001), SHAPE), (dict(window=-1), SHAPE),
    (dict(window=5, sinks=-1), SHAPE), (dict(sinks=4), INVALID), (dict(reserved=1), INVALID), (dict(scale=float("nan")), INVALID), (dict(scale=float("inf")), INVALID), (dict(scale=-2e30), INVALID),
    (dict(q=None), INVALID), (dict(out=None), INVALID), (dict(out=3 * BASE), OVERLAP), (dict(q=3 * BASE + 8), INVALID), (dict(out_stride=(8192, 128)), OVERLAP), (dict(out_stride=(0, 256)), OVERLAP),
    (dict(q_stride=(-8192, 256)), SHAPE), (dict(q_stride=(8192, 264)), INVALID), (dict(lse=BASE + 2), INVALID), (dict(lens=None), INVALID), (dict(lens=BASE + 2), INVALID), (dict(offsets=None), INVALID),
    (dict(offsets=BASE + 4), INVALID), (dict(tables=None), INVALID), (dict(tables=BASE + 2), INVALID), (dict(table_stride=2), INVALID), (dict(table_stride=-4), INVALID), (dict(table_width=374), BOUNDS),
    (dict(workspace=None), INVALID), (dict(workspace=BASE + 8), INVALID), (dict(workspace_bytes=100), BOUNDS),
    (dict(R=1 << 24, n_tokens=1 << 24, max_new=1 << 23, max_len=1 << 24, table_width=1 << 20), TOO_LARGE), (dict(R=1 << 24, n_tokens=1 << 24, max_new=1, max_len=1 << 24, table_width=1 << 20), TOO_LARGE),
])
def test_chunk_refuses(changes, status):
    rc, why = call("tc_attn_chunk", layer(), chunk_args(**changes))
    assert rc == status and why, (rc, why)


@pytest.mark.parametrize("window,sinks,changes,status", [
    (0, 0, {}, SHAPE), (-1, 0, {}, SHAPE), (5, -1, {}, SHAPE), (5, 0, dict(max_prefix=100), INVALID), (5, 0, dict(struct_size=8), INVALID), (5, 0, dict(R=-1), SHAPE), (5, 0, dict(Hq=12), SHAPE),
    (5, 0, dict(out=3 * BASE), OVERLAP), (5, 0, dict(lens=None), INVALID), (5, 0, dict(table_width=3), BOUNDS), (5, 0, dict(workspace=None), INVALID), (5, 0, dict(workspace_bytes=100), BOUNDS),
    (5, 0, dict(reserved=3), INVALID), (5, 0, dict(scale=float("nan")), INVALID),
])
def test_window_refuses(window, sinks, changes, status):
    rc, why = window_call(layer(), decode_args(**(dict(max_prefix=0) | changes)), window, sinks)
    assert rc == status and why, (rc, why)


def test_a_call_for_nothing_returns_before_it_needs_a_device():
    for changes in (dict(R=0), dict(n_tokens=0, q=None, out=None), dict(max_new=0)):
        assert call("tc_attn_chunk", layer(), chunk_args(**changes))[0] == 0
    assert window_call(layer(), decode_args(R=0, max_prefix=0), 5, 0)[0] == 0


@pytest.mark.skipif(torch.cuda.is_available(), reason="asks for the error without a device")
def test_without_a_device_a_good_call_says_so():
    assert call("tc_attn_chunk", layer(), chunk_args())[0] == window_call(layer(), decode_args(max_prefix=0), 5, 0)[0] == b.TC_ERR_CUDA


def test_the_workspace_is_the_same_for_the_same_sizes_and_stays_small():
    lib, out = tc.load_library(), C.c_int64()
    for dtype in (tc.TC_BF16, tc.TC_E4M3):
        for R, n, Hq, H, max_new, max_len, window in ((1, 1, 8, 8, 1, 1, 0), (1, 2048, 32, 8, 2048, 8192, 0), (1, 33, 28, 4, 33, 1 << 24, 0), (512, 1000, 32, 8, 400, 131072, 0), (64, 65536, 64, 8, 8192, 131072, 1024)):
            a = chunk_args(R=R, n=n, Hq=Hq, max_new=max_new, max_len=max_len, window=window)
            assert lib.tc_attn_chunk_workspace(layer(H=H, dtype=dtype).ref, C.byref(a), C.byref(out)) == 0
            first = out.value
            # parts of the items that are cut, those of the single tokens and, of codes, tiles made fp16
            assert 0 <= first <= (4 * 148 * 256 * 129 * 4) + (64 << 20) + R * Hq * 129 * 4 + R * 8 + 4096 + (1 << 30 if dtype == tc.TC_E4M3 else 0)
            assert lib.tc_attn_chunk_workspace(layer(H=H, dtype=dtype).ref, C.byref(a), C.byref(out)) == 0 and out.value == first
    assert lib.tc_attn_chunk_workspace(layer().ref, C.byref(chunk_args(max_new=7000)), C.byref(out)) == SHAPE and out.value == 0
    assert lib.tc_attn_chunk_workspace(layer().ref, C.byref(chunk_args()), None) == INVALID


def test_binding_checks_what_the_library_cannot_see():
    made = layer()
    q, lens, ws, offsets, tables = torch.zeros(5, 16, 128, dtype=torch.bfloat16), torch.zeros(2, dtype=torch.int32), torch.zeros(64, dtype=torch.uint8), torch.zeros(3, dtype=torch.int64), torch.zeros(2, 3, dtype=torch.int32)
    good = dict(q=q, out=q.clone(), tables=tables, offsets=offsets, lens=lens, max_new=3, max_len=16, workspace=ws)
    for bad in (dict(out=q.half()), dict(out=q[:1]), dict(lens=lens.long()), dict(lens=lens[:1]), dict(offsets=offsets.int()), dict(tables=tables[:1]), dict(tables=tables.long()), dict(lse=torch.zeros(5, 8)), dict(q=q.float()),
                dict(q=q[..., :64], out=q[..., :64])):
        with pytest.raises(ValueError):
            tc.tc_attn_chunk(made, **(good | bad))
    good = dict(q=q[:2], out=q[:2].clone(), tables=tables, lens=lens, window=4, max_len=16, workspace=ws)
    for bad in (dict(out=q[:2].half()), dict(lens=lens.long()), dict(tables=tables.long()), dict(lse=torch.zeros(2, 8)), dict(q=q[:2].float())):
        with pytest.raises(ValueError):
            tc.tc_attn_decode_window(made, **(good | bad))


def test_a_window_needs_no_more_workspace_than_the_whole_length():
    """tc_attn_workspace's bytes for the same arguments are enough for every window: nothing but the missing device is found wrong."""
    lib, out = tc.load_library(), C.c_int64()
    for R, max_len in ((1, 100), (3, 131072), (512, 8192)):
        for dtype in (tc.TC_BF16, tc.TC_INT8):
            made, a = layer(dtype=dtype), decode_args(R=R, max_prefix=0, max_len=max_len, table_width=8192)
            assert lib.tc_attn_workspace(made.ref, C.byref(a), C.byref(out)) == 0
            for window in (1, 16, 1000, 100000, 1 << 50):
                a.workspace_bytes = out.value
                rc, why = window_call(made, a, window, window // 3)
                assert "workspace" not in why, why
