"""tc_attn_decode_window in a workspace of the window's size."""
import pytest
import torch

import paper_2608_06007_b200 as tc
from attn_chunk import check_window, run_window, window_batch
from test_operators_gpu import status_is

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("x,kind", [("bf16", "bf16"), ("fp16", "int8")])
@pytest.mark.parametrize("lens,window,sinks", [([9000, 20000, -1, 3], 500, 20), ([2000] * 90, 33, 0), ([700], 4096, 5)])
def test_nothing_is_written_behind_it(x, kind, lens, window, sinks):
    s = window_batch(kind, x, lens, Hq=8, window=window, sinks=sinks)
    need = tc.tc_attn_workspace_bytes(s["pool"].handle, s["dq"], max_len=s["max_len"], window=window, sinks=sinks)
    memory = torch.full((need + (16 << 20),), 0xA5, dtype=torch.uint8, device="cuda")
    run_window(s, memory[:need])
    check_window(s, only={0, len(lens) - 1})
    assert (memory[need:] == 0xA5).all()
    status_is(0)
