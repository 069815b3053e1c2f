"""The workspace of tc_attn_decode_window without a GPU: by what the window lets a row see, not by how long its request is."""
import pytest
import torch

import paper_2608_06007_b200 as tc
from test_attn_chunk_host import window_call
from test_operators_host import BOUNDS, decode_args, layer


@pytest.mark.parametrize("dtype", [tc.TC_BF16, tc.TC_E4M3])
@pytest.mark.parametrize("R,max_len,window,sinks", [(512, 1 << 24, 1024, 16), (512, 1 << 24, 1, 0), (64, 1 << 28, 4096, 4), (3, 500, 128, 4), (1, 100, 4096, 500)])
def test_a_window_over_long_requests_needs_the_workspace_of_the_window(dtype, R, max_len, window, sinks):
    made, q = layer(dtype=dtype), torch.zeros(R, 32, 128, dtype=torch.bfloat16)
    need = tc.tc_attn_workspace_bytes(made, q, max_len=max_len, window=window, sinks=sinks)
    args = decode_args(R=R, max_prefix=0, max_len=max_len, table_width=1 << 24, table_stride=1 << 26)
    args.workspace_bytes = need
    rc, why = window_call(made, args, window, sinks)
    assert rc != BOUNDS, why  # made-up addresses: it gets no further than the device
    args.workspace_bytes = need - 1
    assert window_call(made, args, window, sinks)[0] == BOUNDS


def test_a_workspace_for_what_there_is_not_is_refused():
    made, q = layer(), torch.zeros(3, 32, 128, dtype=torch.bfloat16)
    for bad in (dict(window=-1), dict(window=4, sinks=-1), dict(sinks=4), dict(window=4, max_prefix=100)):
        with pytest.raises(ValueError):
            tc.tc_attn_workspace_bytes(made, q, max_len=100, **bad)
    assert tc.tc_attn_workspace_bytes(made, q, max_len=100) == tc.tc_attn_workspace_bytes(made, q, max_len=100, window=1000)
