"""tc_attn_chunk where offsets decrease: nothing is written outside outputs and workspace, and requests in front are answered."""
import numpy as np
import pytest
import torch

import paper_2608_06007_b200 as tc
from attn_chunk import batch, check_chunk, run_chunk
from test_operators_gpu import dev, status_is

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("x,kind", [("bf16", "bf16"), ("bf16", "e4m3"), ("fp16", "int8")])
@pytest.mark.parametrize("front,each,times", [(100, 73, 50), (20, 9, 200), (70, 700, 3)])
def test_requests_that_share_tokens_write_within_the_workspace(x, kind, front, each, times):
    """One request of its own, then the same tokens again and again."""
    s = batch(kind, x, [front + 400, 2000], [front, each], Hq=8, H=1, poison=False)
    R = 1 + 2 * times
    s["d"]["offsets"] = dev(np.array([0, front] + [front + each, front] * times, dtype=np.int64))
    s["d"]["lens"] = dev(np.array([front + 400] + [2000] * (R - 1), dtype=np.int32))
    s["d"]["tables"] = s["d"]["tables"][[0] + [1] * (R - 1)].contiguous()
    bounds = dict(max_new=s["max_new"], max_len=s["max_len"])
    need, beyond = tc.tc_attn_chunk_workspace_bytes(s["pool"].handle, s["dq"], R, **bounds), 64 << 20
    memory = torch.full((need + beyond,), 0xA5, dtype=torch.uint8, device="cuda")
    run_chunk(s, memory[:need])
    assert (memory[need:] == 0xA5).all()
    s["out"][front:], s["lse"][front:] = 9.0, 9.0  # the shared rows may hold anything
    check_chunk(s, left_out=[1])
    status_is(tc.TC_DEVICE_BAD_INDEX)
