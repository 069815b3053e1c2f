"""tc_attn_chunk with many query heads a KV head, up to more than a block has rows, and with queries that several tokens or heads share."""
import pytest
import torch

from attn_chunk import batch, check_chunk, run_chunk
from test_operators_gpu import status_is

pytestmark = pytest.mark.gpu

TYPES = [("bf16", "bf16"), ("fp16", "fp16"), ("bf16", "e4m3"), ("fp16", "int8")]


@pytest.mark.parametrize("x,kind", TYPES)
@pytest.mark.parametrize("g", [48, 128, 200, 600])
@pytest.mark.parametrize("D", [64, 128, 256])
def test_heads_of_a_group(x, kind, g, D):
    """Blocks of few tokens, of one and of parts of one; cut, whole, and over tiles made fp16."""
    for lens, new, window, sinks in (([1000, 40], [2, 1], 0, 0), ([90, 300, 5], [21, 3, 5], 33, 4)):
        s = batch(kind, x, lens, new, Hq=g, H=1, D=D, window=window, sinks=sinks, front=1, behind=1)
        run_chunk(s)
        check_chunk(s)
    status_is(0)


@pytest.mark.parametrize("x,kind", TYPES)
@pytest.mark.parametrize("shared", ["tokens", "heads", "both"])
def test_queries_that_are_broadcast(x, kind, shared):
    s = batch(kind, x, [200, 90, 1, 64], [150, 9, 1, 64], Hq=8)
    n, Hq, D = s["q"].shape
    one = s["q"][:1] if shared == "tokens" else s["q"][:, :1] if shared == "heads" else s["q"][:1, :1]
    s["q"] = one.expand(n, Hq, D)
    s["dq"] = one.cuda().expand(n, Hq, D)
    assert 0 in s["dq"].stride()
    run_chunk(s)
    check_chunk(s)
    status_is(0)
