"""tc_attn_chunk and tc_attn_decode_window where they can go wrong: numbers that are not finite in places that are not seen, scales far apart, indexes
out of range, pages far apart, streams and captured calls."""
import os
import subprocess
import sys

import numpy as np
import pytest
import torch

import paper_2608_06007_b200 as tc
from attn_chunk import TOP, batch, check_chunk, check_window, run_chunk, run_window, set_rows, set_scales, window_batch
from test_operators_gpu import append_case, dev, np64, status_is

pytestmark = pytest.mark.gpu

TYPES = [("bf16", "bf16"), ("fp16", "fp16"), ("bf16", "e4m3"), ("fp16", "int8")]
# new tokens, cached ones, D: cut into parts; one block; blocks of several items; tiles of codes made fp16 before
SHAPES = {"parts": ([9], [3000], 128), "one block": ([40], [200], 128), "many blocks": ([333], [150], 128), "d 64": ([150], [300], 64), "d 256": ([70], [333], 256)}


def shaped(name, kind, x, **more):
    new, cached, D = SHAPES[name]
    return batch(kind, x, [n + c for n, c in zip(new, cached)], new, Hq=8, D=D, **more)


@pytest.mark.parametrize("shape", SHAPES)
@pytest.mark.parametrize("x,kind", TYPES)
@pytest.mark.parametrize("bad", [float("inf"), float("nan")])
@pytest.mark.parametrize("window,sinks", [(0, 0), (100, 3)])
def test_what_a_row_does_not_see_may_be_anything(shape, x, kind, bad, window, sinks):
    new, cached, _ = SHAPES[shape]
    n, c = new[0], cached[0]
    s = shaped(shape, kind, x, window=window, sinks=sinks, poison=False)
    # V of a new token in the middle and of the last; K of one near the end: the rows before them are as if they were not there
    set_rows(s, 1, 0, [c + n // 2, c + n - 1], bad)
    set_rows(s, 0, 0, [c + 3 * n // 4], float("nan"))
    if window:  # tokens that have left the first rows' windows, or all
        set_rows(s, 1, 0, [c - 99, c - 98, 10], bad)
        set_rows(s, 0, 0, [c - 97], float("nan"))
    run_chunk(s)
    check_chunk(s)
    out = np64(s["out"])
    assert np.isfinite(out[: n // 2]).all() or window
    assert not np.isfinite(out[n - 1]).any()
    status_is(0)


@pytest.mark.parametrize("shape", SHAPES)
@pytest.mark.parametrize("x,kind", [("bf16", "e4m3"), ("fp16", "int8")])
@pytest.mark.parametrize("scales", ["falling", "rising", "apart", "two sizes", "zero"])
def test_scales_of_v_far_apart(shape, x, kind, scales):
    s = shaped(shape, kind, x, poison=False)
    rng = np.random.default_rng(7)
    total = s["lens"][0]
    make = {"falling": lambda t, shape: 2.0 ** (6 - 90 * t / total)[:, None] * np.ones(shape), "rising": lambda t, shape: 2.0 ** (-84 + 90 * t / total)[:, None] * np.ones(shape),
            "apart": lambda t, shape: 2.0 ** rng.integers(-60, 10, shape), "two sizes": lambda t, shape: np.where(rng.random(shape) < 0.02, 1.0, 2.0 ** -24), "zero": lambda t, shape: np.where(rng.random(shape) < 0.5, 0.0, 0.01)}[scales]
    set_scales(s, 1, make)
    run_chunk(s)
    check_chunk(s, far=True)
    status_is(0)


@pytest.mark.parametrize("x,kind", TYPES)
def test_scales_and_spreads(x, kind):
    for shape in ("parts", "one block", "many blocks"):
        for scale, spread in ((-0.05, 1.0), (0.3, 2.0), (1e-3, 3.0)):
            s = shaped(shape, kind, x, scale=scale, spread=spread)
            run_chunk(s)
            check_chunk(s)
    status_is(0)


@pytest.mark.parametrize("shape", ["parts", "one block", "many blocks"])
def test_values_next_to_the_largest_number(shape):
    s = shaped(shape, "bf16", "bf16", poison=False)
    pool = s["pool"]
    v = (torch.randint(0, 2, (pool.blocks, pool.B, pool.H, pool.D)) * 2 - 1).bfloat16() * 3.0e38
    pool.codes(1).copy_(v.view(torch.uint8))
    s["values"][1] = np64(v)
    run_chunk(s)
    check_chunk(s)
    status_is(0)


@pytest.mark.parametrize("x,kind", TYPES)
def test_blocks_out_of_range_are_left_out(x, kind):
    for shape in SHAPES:
        for window, sinks in ((0, 0), (60, 5)):
            s = shaped(shape, kind, x, window=window, sinks=sinks, poison=False)
            n, total = s["new"][0], s["lens"][0]
            B = s["pool"].B
            lost = [total // B - 1, 0, (total - n) // B]
            for i, entry in enumerate(lost):
                s["d"]["tables"][0, entry] = (-1, s["pool"].blocks, 1 << 30)[i]
            run_chunk(s)
            there = ~np.isin(np.arange(total) // B, lost)
            check_chunk(s, there={0: there})
            status_is(tc.TC_DEVICE_BAD_INDEX)
    s = window_batch(kind, x, [300, 90], Hq=8, window=50, sinks=20, poison=False)
    s["d"]["tables"][0, 17], s["d"]["tables"][0, 0] = -5, s["pool"].blocks
    s["d"]["tables"][0, 5] = -1  # of tokens that are not seen: never looked at
    run_window(s)
    check_window(s, there={0: ~np.isin(np.arange(300) // 16, [17, 0])})
    status_is(tc.TC_DEVICE_BAD_INDEX)
    status_is(0)


@pytest.mark.parametrize("x,kind", [("bf16", "bf16"), ("fp16", "int8")])
def test_requests_whose_lengths_make_no_sense_are_left_out(x, kind):
    for others in (0, 8):  # with eight more, requests with one token have their own kernels
        lens, new = [50, 60, 70, 80, 40] + [30] * others, [20, 1, 30, 5, 9] + [1] * others
        s = batch(kind, x, lens, new, Hq=8, front=3, behind=4, poison=False)
        base = s["d"]["offsets"].clone()
        for change, out in ((("lens", 0, 19), [0]), (("lens", 1, 0), [1]), (("lens", 2, 100000), [2]), (("lens", 1, 100000), [1]), (("offsets", 0, -2), [0]), (("offsets", 2, 24 + 40), [1, 2])):
            name, i, value = change
            t = s["d"][name].clone()
            t[i] = value
            s["out"].fill_(9.0), s["lse"].fill_(9.0)
            run_chunk(s, **{name: t})
            check_chunk(s, left_out=out)
            status_is(tc.TC_DEVICE_BAD_INDEX)
        t = base.clone()
        t[-1] = len(s["q"]) + 1
        s["out"].fill_(9.0), s["lse"].fill_(9.0)
        run_chunk(s, offsets=t)
        check_chunk(s, left_out=[len(lens) - 1])
        status_is(tc.TC_DEVICE_BAD_INDEX)
        # more new tokens than were announced
        s["out"].fill_(9.0), s["lse"].fill_(9.0)
        run_chunk(s, max_new=20)
        check_chunk(s, left_out=[2])
        status_is(tc.TC_DEVICE_BAD_INDEX)
    status_is(0)


@pytest.mark.parametrize("x,kind", TYPES)
def test_bounds_wider_than_the_batch(x, kind):
    s = batch(kind, x, [400, 33, 90], [100, 33, 1], Hq=8, extra_len=3000, extra_new=500, front=5)
    run_chunk(s)
    check_chunk(s)
    status_is(0)


@pytest.mark.parametrize("kind", ["bf16", "e4m3"])
def test_pages_past_32_bits_of_bytes(kind):
    s = batch(kind, "bf16", [9000, 300], [40, 200], Hq=4, H=1, gap=8 << 20, poison=False)
    assert s["pool"].raw.numel() > 1 << 33
    run_chunk(s)
    check_chunk(s)
    w = window_batch(kind, "bf16", [9000, 300], Hq=4, H=1, gap=8 << 20, poison=False, window=5000, sinks=30)
    run_window(w)
    check_window(w)
    status_is(0)


@pytest.mark.parametrize("x,kind", TYPES)
def test_more_items_than_multiprocessors(x, kind):
    rng = np.random.default_rng(3)
    new = rng.integers(0, 150, 60).tolist()
    lens = [n + int(c) for n, c in zip(new, rng.integers(0, 400, 60))]
    s = batch(kind, x, lens, new, Hq=16, H=8, D=64, window=0)
    run_chunk(s)
    check_chunk(s, only=set(range(0, 60, 7)) | {59})
    first = s["out"].clone(), s["lse"].clone()
    for _ in range(3):  # and the same bits again
        s["out"].fill_(9.0), s["lse"].fill_(9.0)
        run_chunk(s)
        assert torch.equal(s["out"].view(torch.int16), first[0].view(torch.int16)) and torch.equal(s["lse"], first[1])
    status_is(0)


def test_other_streams_and_replays_with_new_lengths():
    """Captured calls on their own streams and workspaces, replayed together and with other lengths and offsets."""
    cases, torch_streams = [], []
    for kind, x, D in (("bf16", "bf16", 128), ("e4m3", "bf16", 128), ("fp16", "fp16", 64), ("int8", "fp16", 256)):
        s = batch(kind, x, [500, 90, 1300], [120, 90, 5], Hq=8, D=D, behind=30, poison=False)
        w = window_batch(kind, x, [500, 90, 1300], Hq=8, D=D, window=70, sinks=8, poison=False)
        spaces = [torch.empty(tc.tc_attn_chunk_workspace_bytes(s["pool"].handle, s["dq"], 3, max_new=120, max_len=1300), dtype=torch.uint8, device="cuda"),
                  torch.empty(tc.tc_attn_workspace_bytes(w["pool"].handle, w["dq"], max_len=1300), dtype=torch.uint8, device="cuda")]
        cases.append((s, w, spaces, torch.cuda.Stream()))
    torch.cuda.synchronize()
    graphs = []
    for s, w, spaces, stream in cases:
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=stream):
            run_chunk(s, spaces[0], max_new=120, max_len=1300, stream=torch.cuda.current_stream())
            run_window(w, spaces[1], max_len=1300, stream=torch.cuda.current_stream())
        graphs.append(graph)
    for lens, new in (([500, 90, 1300], [120, 90, 5]), ([300, 1, 1000], [1, 1, 100]), ([-1, 60, 1300], [40, 0, 120]), ([1, 2, 3], [1, 1, 1])):
        offsets = np.concatenate([[0], np.cumsum(new)]).astype(np.int64)
        for s, w, spaces, stream in cases:
            for b in (s, w):
                b["lens"] = list(lens)
                b["d"]["lens"].copy_(dev(np.array(lens, dtype=np.int32)))
                b["out"].fill_(9.0), b["lse"].fill_(9.0)
            s["new"], s["offsets"] = list(new), offsets
            s["d"]["offsets"].copy_(dev(offsets))
        torch.cuda.synchronize()
        for _ in range(3):
            for (s, w, spaces, stream), graph in zip(cases, graphs):
                with torch.cuda.stream(stream):
                    graph.replay()
        torch.cuda.synchronize()
        for s, w, spaces, stream in cases:
            check_chunk(s)
            check_window(w)
    status_is(0)


def test_two_calls_at_once_have_their_own_workspaces():
    cases = [(batch(kind, "bf16", [3000, 400], [7, 300], Hq=8), torch.cuda.Stream()) for kind in ("bf16", "e4m3", "bf16")]
    spaces = [torch.empty(tc.tc_attn_chunk_workspace_bytes(s["pool"].handle, s["dq"], 2, max_new=300, max_len=3000), dtype=torch.uint8, device="cuda") for s, _ in cases]
    torch.cuda.synchronize()
    for _ in range(10):
        for (s, stream), space in zip(cases, spaces):
            run_chunk(s, space, stream=stream)
    torch.cuda.synchronize()
    for s, _ in cases:
        check_chunk(s)
    status_is(0)


@pytest.mark.parametrize("kind", ["bf16", "e4m3", "int8"])
def test_a_prompt_written_and_answered_piece_by_piece(kind):
    """append -> chunk, three times over one request in two layers' worth of windows; then a decode step: the answers are those of the whole."""
    from oracle import operators as orc
    from attn_chunk import rows_off
    from test_operators_gpu import Pool, expect_append, tables_for, tokens_of
    rng = np.random.default_rng(11)
    H, D, Hq, B, total, pieces = 2, 128, 8, 16, 261, [100, 33, 127, 1]
    for window, sinks in ((0, 0), (64, 4)):
        pool = Pool(kind, blocks=30, B=B, H=H, D=D)
        table = tables_for([total], pool, rng)
        app = append_case(pool, total, Hq, "bf16", D, False, rng, positions=512)
        app["slots"] = np.array([table[0, t // B] * B + t % B for t in range(total)], dtype=np.int64)
        app["pos"] = np.arange(total)
        cos, sin = dev(app["cos"]), dev(app["sin"])
        out, lse = torch.full((total, Hq, D), 9.0, dtype=torch.bfloat16, device="cuda"), torch.full((total, Hq), 9.0, device="cuda")
        at = 0
        for n in pieces:
            part = slice(at, at + n)
            tc.tc_kv_append(pool.handle, app["k"][part], app["v"][part], dev(app["slots"][part]), q=app["q"][part], q_out=app["q_out"][part], positions=dev(app["pos"][part]), cos=cos, sin=sin)
            if n > 1:
                ws = torch.empty(tc.tc_attn_chunk_workspace_bytes(pool.handle, out[part], 1, max_new=n, max_len=total, window=window, sinks=sinks), dtype=torch.uint8, device="cuda")
                tc.tc_attn_chunk(pool.handle, app["q_out"][part], out[part], dev(table), dev(np.array([0, n])), dev(np.array([at + n], dtype=np.int32)), max_new=n, max_len=total, window=window, sinks=sinks,
                                 lse=lse[part], workspace=ws)
            else:
                ws = torch.empty(tc.tc_attn_workspace_bytes(pool.handle, out[part], max_len=total), dtype=torch.uint8, device="cuda")
                tc.tc_attn_decode_window(pool.handle, app["q_out"][part], out[part], dev(table), dev(np.array([at + n], dtype=np.int32)), window=window or total, sinks=sinks, max_len=total, lse=lse[part], workspace=ws)
            at += n
        q, rows = expect_append(pool, app)
        values = []
        for stored, scale in rows:
            x = orc.values(stored.numpy().view(np.uint8 if kind == "e4m3" else np.int8), scale.numpy(), kind) if scale is not None else np64(stored.view(torch.bfloat16))
            values.append(x)
        s = dict(pool=pool, x="bf16", q=q, out=out, lse=lse, scale=0.0, window=window, sinks=sinks)
        rows_off(s, 0, 0, total, values[0], values[1], 1)
    status_is(0)


FIRST_CALL = """
import sys
sys.path[:0] = [{root!r}, {tests!r}]
import torch
from attn_chunk import *
for kind, x in (("bf16", "bf16"), ("int8", "fp16")):
    s = batch(kind, x, [3000, 400], [7, 300], Hq=8, poison=False)
    w = window_batch(kind, x, [3000, 40], Hq=8, window=100, sinks=3, poison=False)
    spaces = [torch.empty(tc.tc_attn_chunk_workspace_bytes(s["pool"].handle, s["dq"], 2, max_new=300, max_len=3000), dtype=torch.uint8, device="cuda"),
              torch.empty(tc.tc_attn_workspace_bytes(w["pool"].handle, w["dq"], max_len=3000), dtype=torch.uint8, device="cuda")]
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        run_chunk(s, spaces[0], stream=torch.cuda.current_stream())
        run_window(w, spaces[1], stream=torch.cuda.current_stream())
    graph.replay()
    torch.cuda.synchronize()
    check_chunk(s), check_window(w)
print("captured")
"""


def test_the_first_call_of_a_process_may_be_a_captured_one():
    tests = os.path.dirname(os.path.abspath(__file__))
    r = subprocess.run([sys.executable, "-c", FIRST_CALL.format(root=os.path.dirname(tests), tests=tests)], capture_output=True, text=True, timeout=300)
    assert r.returncode == 0 and "captured" in r.stdout, r.stderr[-2000:]
