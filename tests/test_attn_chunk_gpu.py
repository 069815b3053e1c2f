"""tc_attn_chunk against 64 bits."""
import numpy as np
import pytest
import torch

import paper_2608_06007_b200 as tc
from attn_chunk import batch, check_chunk, run_chunk
from test_operators_gpu import status_is

pytestmark = pytest.mark.gpu

TYPES = [("bf16", "bf16"), ("fp16", "fp16"), ("bf16", "e4m3"), ("fp16", "int8")]
WINDOWS = [(0, 0), (1, 0), (33, 4), (200, 1), (128, 300)]


@pytest.mark.parametrize("x,kind", TYPES)
@pytest.mark.parametrize("window,sinks", WINDOWS)
def test_a_few_requests(x, kind, window, sinks):
    s = batch(kind, x, [37, 100, -1, 5, 200, 64], [7, 100, 3, 1, 13, 0], Hq=8, window=window, sinks=sinks, front=2, behind=3)
    run_chunk(s)
    check_chunk(s)
    status_is(0)


@pytest.mark.parametrize("x,kind", TYPES + [("fp16", "e4m3"), ("bf16", "int8")])
@pytest.mark.parametrize("D,H,g,B,layout", [(128, 2, 4, 16, "nhd"), (64, 1, 1, 5, "hnd"), (80, 3, 7, 16, "hnd"), (256, 1, 20, 8, "nhd"), (16, 2, 16, 1, "nhd"), (192, 1, 3, 32, "hnd"), (112, 2, 17, 7, "nhd")])
def test_types_and_shapes(x, kind, D, H, g, B, layout):
    for window, sinks in ((0, 0), (70, 3)):
        s = batch(kind, x, [300, 1, 129, 128], [150, 1, 40, 128], Hq=H * g, H=H, D=D, B=B, layout=layout, window=window, sinks=sinks, gap=32)
        run_chunk(s)
        check_chunk(s)
    status_is(0)


@pytest.mark.parametrize("x,kind", TYPES)
@pytest.mark.parametrize("lens,new,D,window,sinks", [([4000], [5], 128, 0, 0), ([1500, 20, 2600], [40, 3, 1], 128, 0, 0), ([9000], [1], 64, 0, 0), ([1300, 700], [9, 2], 256, 0, 0), ([6000], [33], 128, 3000, 500)])
def test_long_keys_of_few_rows_are_cut_into_parts(x, kind, lens, new, D, window, sinks):
    s = batch(kind, x, lens, new, Hq=8, D=D, window=window, sinks=sinks)
    for _ in range(3):
        s["out"].fill_(9.0), s["lse"].fill_(9.0)
        run_chunk(s)  # each on a workspace of 0xFF
        check_chunk(s)
    status_is(0)


@pytest.mark.parametrize("x,kind", TYPES)
@pytest.mark.parametrize("window,sinks", [(0, 0), (100, 5)])
@pytest.mark.parametrize("new", [[1] * 12, [1, 40, 1, 1, 0, 1, 300, 1, 1, 2, 1, 1], [1, 1, 1]])
def test_single_tokens_alone_and_beside_chunks(x, kind, window, sinks, new):
    lens = [n + extra if n else 50 for n, extra in zip(new, [0, 17, 900, 64, 50, 33, 200, 3000, 127, 10, 400, 1])]
    if len(new) > 8:
        lens[3] = -1
    s = batch(kind, x, lens, new, Hq=8, window=window, sinks=sinks, front=1, behind=2, strided=True)
    run_chunk(s)
    check_chunk(s)
    status_is(0)


@pytest.mark.parametrize("x,kind", [("bf16", "e4m3"), ("fp16", "int8"), ("bf16", "bf16")])
@pytest.mark.parametrize("D,H,g", [(128, 2, 4), (64, 1, 8), (80, 2, 3), (256, 1, 4)])
@pytest.mark.parametrize("window,sinks", [(0, 0), (150, 70), (40, 0)])
def test_many_blocks_of_rows(x, kind, D, H, g, window, sinks):
    """Codes that three blocks of rows meet are made fp16 before."""
    s = batch(kind, x, [700, 300, 1, 450, -1], [400, 300, 1, 129, 2], Hq=H * g, H=H, D=D, window=window, sinks=sinks)
    run_chunk(s)
    check_chunk(s)
    status_is(0)


@pytest.mark.parametrize("x,kind", [("bf16", "e4m3"), ("fp16", "int8")])
@pytest.mark.parametrize("D,g", [(128, 4), (64, 8), (256, 4)])
@pytest.mark.parametrize("window,sinks,extra_len", [(0, 0, 0), (0, 0, 100000), (0, 0, 4000000), (150, 70, 100000)])
def test_requests_of_few_and_of_many_blocks_in_one_call(x, kind, D, g, window, sinks, extra_len):
    """More requests than have many blocks; bounds so wide that only the longest have room, or none."""
    new = [1, 300, 2, 140, 135, 1, 129, 128, 0, 65, 66, 33, 1, 400, 64, 500]
    lens = [n + extra if n else 50 for n, extra in zip(new, [500, 2000, 70, 5, 3000, 40, 1000, 128, 0, 300, 0, 700, 900, 100, 64, 250])]
    lens[6] = -1
    s = batch(kind, x, lens, new, Hq=2 * g, D=D, window=window, sinks=sinks, front=3, behind=5, extra_len=extra_len, seed=D)
    need = tc.tc_attn_chunk_workspace_bytes(s["pool"].handle, s["dq"], len(lens), max_new=s["max_new"], max_len=s["max_len"], window=window, sinks=sinks)
    workspace = torch.full((need,), 0xFF, dtype=torch.uint8, device="cuda")
    run_chunk(s, workspace)
    check_chunk(s)
    first = s["out"].clone()
    run_chunk(s, workspace)  # finds what the first call left there
    assert torch.equal(s["out"], first)
    status_is(0)


@pytest.mark.parametrize("x,kind", TYPES)
@pytest.mark.parametrize("B,layout", [(4, "hnd"), (12, "nhd"), (20, "hnd"), (24, "nhd"), (256, "nhd"), (3, "nhd"), (48, "hnd")])
def test_blocks_of_all_sizes(x, kind, B, layout):
    for D in (64, 128, 256):
        s = batch(kind, x, [333, 270], [120, 64], Hq=4, H=2, D=D, B=B, layout=layout, window=100, sinks=9, gap=64)
        run_chunk(s)
        check_chunk(s)
    status_is(0)
