"""tc_attn_chunk over values that are not finite and that rows do see: they reach the rows that see them, whole, and nobody else."""
import pytest
import torch

from attn_chunk import TOP, batch, check_chunk, run_chunk, set_rows
from test_operators_gpu import status_is

pytestmark = pytest.mark.gpu

TYPES = [("bf16", "bf16"), ("fp16", "fp16"), ("bf16", "e4m3"), ("fp16", "int8")]
CACHED, REQUESTS, BAD = 280, 12, 7  # BAD: the request that has the value


def requests(kind, x, D, new, **more):
    """Requests of `new` tokens each, of 8 KV heads with four query heads: items enough for CTAs to take one behind another."""
    return batch(kind, x, [new + CACHED] * REQUESTS, [new] * REQUESTS, Hq=32, H=8, D=D, poison=False, **more)


def answers(s):
    """(out, lse), [request, token, head, ..]."""
    s["out"].fill_(9.0), s["lse"].fill_(9.0)
    run_chunk(s)
    return s["out"].unflatten(0, (REQUESTS, -1)).clone(), s["lse"].unflatten(0, (REQUESTS, -1)).clone()


def others(t):
    return t[[r for r in range(REQUESTS) if r != BAD]]


@pytest.mark.parametrize("x,kind", TYPES)
@pytest.mark.parametrize("D", [64, 128, 256])
@pytest.mark.parametrize("new", [40, 150])  # one block or two; three or more, over whose codes tiles are made fp16 before
@pytest.mark.parametrize("bad", [float("nan"), float("inf")])
def test_a_value_that_all_rows_see_leaves_them_no_finite_output(x, kind, D, new, bad):
    s = requests(kind, x, D, new)
    pool = s["pool"]
    kept = [pool.raw.clone(), pool.scales.clone() if kind in TOP else None]
    # in the first tile of every item, in a later one, and among first tokens that stay visible
    for token, window, sinks in ((10, 0, 0), (200, 0, 0), (10, 120, 128)):
        s["window"], s["sinks"] = window, sinks
        clean, clean_lse = answers(s)
        set_rows(s, 1, BAD, [token], bad)
        out, lse = answers(s)
        assert not torch.isfinite(out[BAD]).any()
        # the weights are what they were; a sum's exponentials and logarithm are good to 2^-18 and 2^-22, relative to whichever maximum
        assert ((lse - clean_lse).abs() <= 2 * (2.0 ** -18 + 2.0 ** -22 * clean_lse.abs())).all()
        assert torch.equal(others(out), others(clean)) and torch.equal(others(lse), others(clean_lse))
        pool.raw.copy_(kept[0])
        if kind in TOP:
            pool.scales.copy_(kept[1])
    status_is(0)


@pytest.mark.parametrize("D", [64, 128, 256])
@pytest.mark.parametrize("new", [40, 150])
@pytest.mark.parametrize("token", [10, 200, CACHED + 5])
def test_one_code_that_is_no_number_leaves_its_column_alone_without_a_finite_output(D, new, token):
    s = requests("e4m3", "bf16", D, new)
    pool, h, d = s["pool"], 5, D // 2 + 3
    block, at = int(s["table"][BAD][token // pool.B]), token % pool.B
    pool.codes(1)[block, at, h, d] = 0
    s["values"][1][block, at, h, d] = 0.0
    clean, clean_lse = answers(s)
    check_chunk(s, only={BAD})
    pool.codes(1)[block, at, h, d] = 0x7F
    out, lse = answers(s)
    seen = max(0, token - CACHED)  # the first row of the request that sees it
    column = out[BAD, :, 4 * h : 4 * h + 4, d]
    assert torch.isnan(column[seen:]).all() and torch.isfinite(column[:seen]).all()
    assert torch.equal(lse, clean_lse) and torch.equal(others(out), others(clean))
    column.copy_(clean[BAD, :, 4 * h : 4 * h + 4, d])
    s["out"].copy_(out.flatten(0, 1))
    check_chunk(s, only={BAD})  # the other columns, as if the code were 0
    status_is(0)
