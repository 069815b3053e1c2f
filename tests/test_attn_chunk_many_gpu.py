"""tc_attn_chunk with more requests than a CTA has threads, and with short requests of one and of two blocks of rows one behind another."""
import numpy as np
import pytest
import torch

from attn_chunk import batch, check_chunk, run_chunk
from test_operators_gpu import status_is

pytestmark = pytest.mark.gpu

TYPES = [("bf16", "bf16"), ("fp16", "fp16"), ("bf16", "e4m3"), ("fp16", "int8")]


def check_some(s, only):
    check_chunk(s, only=only)
    first = s["out"].clone(), s["lse"].clone()
    s["out"].fill_(9.0), s["lse"].fill_(9.0)
    run_chunk(s)
    assert torch.equal(s["out"].view(torch.int16), first[0].view(torch.int16)) and torch.equal(s["lse"], first[1])
    status_is(0)


@pytest.mark.parametrize("x,kind", TYPES)
@pytest.mark.parametrize("R", [700, 1500])
@pytest.mark.parametrize("mixed", [False, True])
def test_more_requests_than_threads(x, kind, R, mixed):
    """mixed: some of them are cut, some have tiles made fp16 before, beside single tokens, requests without any and padding."""
    rng = np.random.default_rng([R, mixed])
    new, cached = rng.integers(2, 9, R), rng.integers(0, 60, R)
    if mixed:
        new = rng.choice([0, 1, 1, 1], R)
        few = rng.permutation(R)[:60]
        new[few[:50]], cached[few[:20]] = rng.integers(2, 20, 50), rng.integers(1000, 2500, 20)
        new[few[50:54]] = 150
    lens = np.where(rng.random(R) < 0.1 if mixed else np.zeros(R, dtype=bool), -1, new + cached)
    s = batch(kind, x, lens.tolist(), new.tolist(), Hq=8, H=2, D=64)
    run_chunk(s)
    only = set(range(0, R, 97)) | {R - 1} | (set(few[:54].tolist()) if mixed else set())
    check_some(s, only)


@pytest.mark.parametrize("x,kind", TYPES)
@pytest.mark.parametrize("D", [64, 128, 256])
def test_short_prompts_of_one_slot_and_of_two(x, kind, D):
    """One tile of keys each, 240 rows of a KV head and then 40 to 120: a slot may be an item behind the other."""
    rng = np.random.default_rng(D)
    new = [60 if i % 2 else int(rng.integers(10, 31)) for i in range(80)]
    s = batch(kind, x, new, new, Hq=32, H=8, D=D, spread=2.0)
    run_chunk(s)
    check_some(s, set(range(0, 80, 13)))
