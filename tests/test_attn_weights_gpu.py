"""Attention over paged keys whose weights leave fp32's range, and rows that have no weight at all, in every operator and however keys are cut."""
import numpy as np
import pytest
import torch

import paper_2608_06007_b200 as tc
from attn_chunk import TOP, batch, check_chunk, check_window, run_chunk, run_window, set_rows, window_batch
from oracle import operators as orc
from test_operators_gpu import TORCH, np64, status_is

pytestmark = pytest.mark.gpu

TYPES = [("bf16", "bf16"), ("fp16", "fp16"), ("bf16", "e4m3"), ("fp16", "int8")]
# requests of one batch whose keys are: cut into parts of blocks; single tokens' stretches of the stream; the same in a call for single tokens alone
CASES = ["chunk", "blocks", "singles", "window", "decode"]


def put(s, plane, r, tokens, value):
    """Every element of these tokens becomes `value`."""
    pool, t = s["pool"], np.asarray(tokens)
    block, at = s["table"][r][t // pool.B], t % pool.B
    rows = np.full((len(t), pool.H, pool.D), value, dtype=np.float32)
    where = torch.from_numpy(block).long().cuda(), torch.from_numpy(at).cuda()
    if pool.kind in TOP:
        codes, scale = orc.quantise(rows, pool.kind)
        pool.codes(plane)[where] = torch.from_numpy(codes.view(np.uint8)).cuda()
        pool.scale(plane)[where] = torch.from_numpy(scale).cuda()
        s["values"][plane][block, at] = orc.values(codes, scale, pool.kind)
    else:
        stored = torch.from_numpy(rows).to(TORCH[pool.kind])
        pool.codes(plane)[where] = stored.view(torch.uint8).cuda()
        s["values"][plane][block, at] = np64(stored)


def made(case, kind, x, D, total, many):
    few = [50] * (70 if many else 8)  # with many requests one warp joins a row's parts, else 16
    if case in ("window", "decode"):
        s = window_batch(kind, x, [total] + few, Hq=4, H=1, D=D, window=1 << 30, poison=False)
    elif case == "singles":
        s = batch(kind, x, [total] + few, [1] * (1 + len(few)), Hq=4, H=1, D=D, poison=False)
    else:
        new = 5 if case == "chunk" else 200
        s = batch(kind, x, [total, 50], [new, 20], Hq=4, H=1, D=D, poison=False)
    s["q"].fill_(1.0), s["dq"].fill_(1.0)
    return s


def ask(case, s):
    if case == "window":
        run_window(s)
    elif case == "decode":
        ws = torch.empty(tc.tc_attn_workspace_bytes(s["pool"].handle, s["dq"], max_len=s["max_len"]), dtype=torch.uint8, device="cuda")
        tc.tc_attn_decode(s["pool"].handle, s["dq"], s["out"], s["d"]["tables"], s["d"]["lens"], max_len=s["max_len"], lse=s["lse"], workspace=ws)
    else:
        run_chunk(s)


def answer(case, s):
    ask(case, s)
    (check_window if case in ("window", "decode") else check_chunk)(s)


@pytest.mark.parametrize("x,kind", TYPES)
@pytest.mark.parametrize("D", [64, 128, 256])
@pytest.mark.parametrize("case", CASES)
@pytest.mark.parametrize("low,token", [((0, 3000), 10), ((2500, 5500), 4000)])
@pytest.mark.parametrize("bad,many", [(float("inf"), False), (float("nan"), True)])
def test_a_value_that_is_not_finite_is_seen_whatever_its_weight(case, x, kind, D, low, token, bad, many):
    """Many keys score some 20 sqrt(D) below the others: by themselves they have a sum that is nothing in fp32 beside theirs."""
    s = made(case, kind, x, D, 6000, many)
    put(s, 0, 0, np.arange(*low), -20.0)
    set_rows(s, 1, 0, [token], bad)
    answer(case, s)  # as in 64 bits
    assert not torch.isfinite(s["out"][: s["new"][0] if case in ("chunk", "blocks") else 1]).any()
    status_is(0)


@pytest.mark.parametrize("x,kind", TYPES)
@pytest.mark.parametrize("D", [64, 128, 256])
@pytest.mark.parametrize("total", [20, 290, 3000])
@pytest.mark.parametrize("case,many", [("chunk", False), ("blocks", False), ("singles", True), ("window", False), ("window", True), ("decode", False), ("decode", True)])
def test_a_row_without_weight_gets_nothing_whatever_the_values_are(case, many, x, kind, D, total):
    """Every score is -infinity: outputs are 0 and logarithms -infinity, as the header has it."""
    total += 180 if case == "blocks" else 0
    s = made(case, kind, x, D, total, many)
    put(s, 0, 0, np.arange(total), -1.0 if kind in TOP else -float("inf"))
    if kind in TOP:  # all codes are negative
        t = np.arange(total)
        s["pool"].scale(0)[torch.from_numpy(s["table"][0][t // s["pool"].B]).long().cuda(), torch.from_numpy(t % s["pool"].B).cuda()] = float("inf")
    ask(case, s)
    n = s["new"][0] if case in ("chunk", "blocks") else 1
    for _ in range(2):
        assert (s["out"][:n] == 0).all() and torch.isneginf(s["lse"][:n]).all()
        set_rows(s, 1, 0, [7, total // 2], float("inf"))
        ask(case, s)
    assert (s["out"][:n] == 0).all() and torch.isneginf(s["lse"][:n]).all()
    status_is(0)
