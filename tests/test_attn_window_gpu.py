"""tc_attn_decode_window against 64 bits."""
import numpy as np
import pytest
import torch

import paper_2608_06007_b200 as tc
from attn_chunk import batch, check_window, run_window, window_batch
from test_operators_gpu import status_is

pytestmark = pytest.mark.gpu

TYPES = [("bf16", "bf16"), ("fp16", "fp16"), ("bf16", "e4m3"), ("fp16", "int8")]
LENS = [37, 100, -1, 1, 0, 200, 64, 65, 700, 33, 1500]


@pytest.mark.parametrize("x,kind", TYPES)
@pytest.mark.parametrize("window,sinks", [(1, 0), (1, 1), (16, 0), (17, 4), (64, 16), (100, 33), (100, 500), (3000, 0), (1 << 40, 1 << 40)])
def test_lengths_and_windows(x, kind, window, sinks):
    for B in (16, 5):
        s = window_batch(kind, x, LENS, Hq=8, B=B, window=window, sinks=sinks)
        run_window(s)
        check_window(s)
    status_is(0)


@pytest.mark.parametrize("x,kind", TYPES + [("fp16", "e4m3"), ("bf16", "int8")])
@pytest.mark.parametrize("D,H,g,B,layout", [(128, 2, 4, 16, "nhd"), (64, 1, 1, 5, "hnd"), (80, 3, 7, 16, "hnd"), (256, 1, 20, 8, "nhd"), (16, 2, 16, 1, "nhd"), (192, 1, 3, 32, "hnd"), (112, 2, 17, 7, "nhd")])
def test_types_and_shapes(x, kind, D, H, g, B, layout):
    s = window_batch(kind, x, [300, 1, -1, 129, 400], Hq=H * g, H=H, D=D, B=B, layout=layout, window=130, sinks=3, gap=32, strided=True)
    run_window(s)
    check_window(s)
    status_is(0)


@pytest.mark.parametrize("x,kind", TYPES)
def test_many_requests_and_few_long_ones(x, kind):
    rng = np.random.default_rng(5)
    for lens, window, H in ((rng.integers(-1, 500, 300).tolist(), 90, 2), ([9000, 20000], 7000, 1)):
        s = window_batch(kind, x, lens, Hq=4 * H, H=H, window=window, sinks=20)
        run_window(s)
        check_window(s, only=set(range(0, len(lens), 17)) | {len(lens) - 1})
    status_is(0)
