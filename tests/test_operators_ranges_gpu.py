"""The operators on a paged layer where numbers are far apart, and each of decode's kernels by name.

A case says which kernel takes its prefix - none, the stream, or the prefix kernel with 128 or 256 rows a CTA - and
fails where the library's rule gives it to another."""
import ctypes
import os
import subprocess
import sys
import time

import numpy as np
import pytest
import torch

import paper_2608_06007_b200 as tc
from operators_split import prefix_taken_by
from oracle import operators as orc
from paper_2608_06007_b200 import build
from test_operators_gpu import Pool, append_case, attend_case, check_append, check_attend, dev, np64, run_append, run_attend, status_is, tokens_of

pytestmark = pytest.mark.gpu

TOP = {"e4m3": 448.0, "int8": 127.0}


# ---------------------------------------------------------------------------------------- append
@pytest.mark.parametrize("kind", ["e4m3", "int8", "bf16"])
@pytest.mark.parametrize("x", ["bf16", "fp32"])
@pytest.mark.parametrize("interleaved", [False, True])
def test_append_keeps_the_sign_of_zeros(kind, x, interleaved):
    """-0 in rows that are not zero: given, and made by a rotation of (0, 0) with a negative cosine.  D = 100 takes single
    elements, the others vectors."""
    def mutate(qkv):
        qkv[::2, :, ::3] = -0.0
        qkv[::3, :, 1::5] = 0.0
        qkv[1, :, 4:] = 0.0
        qkv[2, :, 8:] = -0.0

    rng = np.random.default_rng([interleaved, x == "bf16"])
    for D, rot in ((128, 128), (128, 0), (80, 32), (100, 50)):
        pool = Pool(kind, D=D)
        s = append_case(pool, 37, 4, x, rot, interleaved, rng, mutate=mutate)
        run_append(pool, s)
        check_append(pool, s)
    status_is(0)


# ---------------------------------------------------------------------------------------- decode
# name: (requests, KV heads, query heads of each, head dim, prefix, own tokens at most)
SHAPES = {
    "none": (3, 2, 4, 128, 0, 600),
    "none, 64": (3, 1, 3, 64, 0, 600),
    "none, 12 heads": (2, 1, 12, 128, 0, 300),
    "none, 256": (2, 1, 5, 256, 0, 300),
    "stream": (4, 2, 4, 128, 700, 60),
    "stream, 16 rows": (3, 1, 11, 80, 600, 60),
    "prefix 128": (20, 8, 6, 128, 2100, 40),
    "prefix 128, 64": (32, 8, 4, 64, 2700, 40),
    "prefix 256": (36, 8, 7, 128, 1300, 40),
    "prefix 256, 80": (36, 8, 7, 80, 1300, 40),
    "prefix 256, three blocks": (150, 3, 4, 128, 1300, 20),
}
STREAMS = [name for name in SHAPES if not name.startswith("prefix")]
PREFIXES = [name for name in SHAPES if name.startswith("prefix")]


def shaped(shape, kind, x, rng, B=16, layout="nhd", plain_tiles=False, **more):
    R, H, g, D, prefix, most = SHAPES[shape]
    if plain_tiles and prefix > 1000:
        prefix //= 2  # 16-bit pools have tiles of half as many keys
    lens = rng.integers(0, most + 1, R)
    lens[0], lens[-1] = most, 1
    lens = lens.tolist()
    if prefix:
        taken = prefix_taken_by(R, H * g, H, D, max(lens), prefix, kind in TOP)
        assert taken == shape.split(",")[0], taken
    pool = Pool(kind, layout=layout, D=D, H=H, B=B, blocks=sum(-(-n // B) for n in lens) + -(-prefix // B) + 3)
    return pool, attend_case(pool, lens, prefix, H * g, x, rng, poison=False, **more)


def rows_of(pool, s, plane, make):
    """Sets a quantised plane's codes and scales: make(t, shape) -> (codes as numbers, scales) of token t[i] of the prefix
    (then of each request, counting on behind it), for all heads."""
    codes = np.zeros((pool.blocks, pool.B, pool.H, pool.D), dtype=np.uint8)
    scale = np.zeros((pool.blocks, pool.B, pool.H), dtype=np.float32)
    for table, first, n in [(s["shared"], 0, s["prefix"])] + [(tab, s["prefix"], max(0, m)) for tab, m in zip(s["table"], s["lens"])]:
        t = np.arange(n)
        c, sc = make(first + t, (n, pool.H, pool.D))
        c = np.asarray(c, dtype=np.float64)
        codes[table[t // pool.B], t % pool.B] = orc.e4m3_round(c) if pool.kind == "e4m3" else np.rint(c).astype(np.int8).view(np.uint8)
        scale[table[t // pool.B], t % pool.B] = sc
    pool.codes(plane).copy_(torch.from_numpy(codes))
    pool.scale(plane).copy_(torch.from_numpy(scale))
    s["values"][plane] = orc.values(codes if pool.kind == "e4m3" else codes.view(np.int8), scale, pool.kind)
    s["scale_of"] = s.get("scale_of", {}) | {plane: np.abs(scale.astype(np.float64))}


def check_ranges(pool, s, x, prefix_kernel, only):
    """Outputs and logarithms of some requests against 64 bits.  A quantised pool's products are of 16-bit numbers: a
    probability is rounded once (half a step of 2^-11), a value of the prefix kernel's twice more.  A weight is 2 to the
    power of a sum of logarithms of up to some hundreds, in fp32: 2^-14 of it.  A product below fp16's normal numbers is off by half of 2^-24 at most,
    beside a largest contribution of at least 1/2 (code: up to TOP), or for values 2^-15 of their scale.  Then the output's own half step."""
    scale, top = s["scale"] or pool.D ** -0.5, TOP[pool.kind]
    out, lse, q = np64(s["out"]), np64(s["lse"]), np64(s["q"])
    g = s["q"].shape[1] // pool.H
    u_o = torch.finfo(s["out"].dtype).eps / 2
    half = 2.0 ** -25 if x == "fp16" else 2.0 ** -133
    both = lambda what, r: np.concatenate([tokens_of(what, s["shared"], 0, s["prefix"], pool.B), tokens_of(what, s["table"][r], 0, s["lens"][r], pool.B)])
    for r in only:
        if s["lens"][r] < 0:
            assert (out[r] == 9.0).all() and (lse[r] == 9.0).all()
            continue
        keys, vals = (both(v, r) for v in s["values"])
        if not len(keys):
            assert (out[r] == 0).all() and (lse[r] == -np.inf).all()
            continue
        sizes = both(s["scale_of"][1], r)
        want, want_lse, mass = orc.attend(q[r], keys, vals, scale)
        k = np.repeat(keys, g, axis=1)
        score = np.einsum("hd,nhd->hn", q[r], k) * scale
        weights = np.exp(score - want_lse[:, None]) * np.repeat(sizes, g, axis=1).T  # of each key, times its scale
        delta = (pool.D + 4) * 2.0 ** -24 * abs(scale) * np.einsum("hd,nhd->nh", np.abs(q[r]), np.abs(k)).max(0)
        most = ((3 if prefix_kernel else 1) * 2.0 ** -11 * (1 + 2.0 ** -6) + 2 * delta[:, None] + 2.0 ** -14) * mass
        most += (len(keys) * 2.0 ** -24 * top * weights.max(1) + 2.0 ** -15 * weights.sum(1))[:, None]
        most += u_o * (1 + 2.0 ** -6) * np.abs(want) + half
        off = np.abs(out[r] - want)
        assert (off <= most).all(), (r, off.max(), np.abs(want).max(), (off / np.maximum(most, 1e-300)).max())
        assert (np.abs(lse[r] - want_lse) <= delta + 2.0 ** -18 + 2.0 ** -22 * np.abs(want_lse)).all(), (r, lse[r], want_lse)


def check(pool, s, x, prefix_kernel, only):
    if pool.kind not in TOP:
        return check_attend(pool, s, x, only=set(only))
    # test_operators_gpu's bound has no term for probabilities below fp16's normal numbers in quantised pools
    check_ranges(pool, dict(s, scale_of={1: np64(pool.scale(1).abs())}), x, prefix_kernel, only)


def spread_codes(rng, kind):
    return lambda shape: np.clip(rng.standard_normal(shape) * TOP[kind] / 3, -TOP[kind], TOP[kind])


V_SCALES = {
    "smallest": lambda rng, t, H: np.full((len(t), H), 2.0 ** -126) * (1 + rng.random((len(t), H))),
    "small": lambda rng, t, H: np.full((len(t), H), 2.0 ** -113) * (1 + rng.random((len(t), H))),
    "large": lambda rng, t, H: np.full((len(t), H), 1e35) * (1 + rng.random((len(t), H))),
    "spans of 64 far apart": lambda rng, t, H: np.where(t // 64 % 2, 2.0 ** 60, 2.0 ** -90)[:, None] * np.ones(H),
    "spans of 128 far apart": lambda rng, t, H: np.where(t // 128 % 2, 2.0 ** -90, 2.0 ** 60)[:, None] * np.ones(H),
    "mixed": lambda rng, t, H: 10.0 ** rng.uniform(-30, 30, (len(t), H)),
    "mixed, zeros": lambda rng, t, H: 10.0 ** rng.uniform(-37, 5, (len(t), H)) * (rng.random((len(t), H)) > 0.3),
}


@pytest.mark.parametrize("shape", SHAPES)
@pytest.mark.parametrize("kind,x", [("e4m3", "bf16"), ("int8", "bf16")])
@pytest.mark.parametrize("scales", V_SCALES)
def test_attention_over_scales_of_v_at_the_ends_of_their_range(shape, kind, x, scales):
    """Scales that tc_kv_append may write, 2^-126 and up, together in one request; equal scores and ordinary ones."""
    rng = np.random.default_rng([len(shape), len(scales), x == "bf16"])
    pool, s = shaped(shape, kind, x, rng)
    codes = spread_codes(rng, kind)
    rows_of(pool, s, 1, lambda t, sh: (codes(sh), V_SCALES[scales](rng, t, pool.H)))
    only = sorted({0, len(s["lens"]) - 1})
    run_attend(pool, s)
    check_ranges(pool, s, x, shape.startswith("prefix"), only)
    rows_of(pool, s, 0, lambda t, sh: (np.zeros(sh), np.ones(sh[:2])))
    run_attend(pool, s)
    check_ranges(pool, s, x, shape.startswith("prefix"), only)
    status_is(0)


@pytest.mark.parametrize("shape", SHAPES)
@pytest.mark.parametrize("kind,x", [("e4m3", "bf16"), ("int8", "bf16")])
@pytest.mark.parametrize("power", [-10, -24, -40, -90])
def test_attention_that_looks_at_one_key_of_a_small_scale(shape, kind, x, power):
    """One key has all of the weight, and a V far smaller than its neighbours'."""
    rng = np.random.default_rng([len(shape), -power])
    pool, s = shaped(shape, kind, x, rng)
    at = (s["prefix"] or s["lens"][0]) // 2 + 5
    codes = spread_codes(rng, kind)
    rows_of(pool, s, 1, lambda t, sh: (codes(sh), np.where(t == at, 2.0 ** power, 1.0)[:, None] * np.ones(pool.H)))
    rows_of(pool, s, 0, lambda t, sh: ((t == at)[:, None, None] * np.full(sh, 64.0), np.full(sh[:2], 1 / 16)))
    q = torch.from_numpy(8.0 + rng.random(s["q"].shape)).to(s["q"].dtype)  # that key's scores: 34 sqrt(D), the others' 0
    s["q"] = q
    s["dq"].copy_(q)
    run_attend(pool, s)
    check_ranges(pool, s, x, shape.startswith("prefix"), [0])
    assert np.abs(np64(s["out"])[0]).max() < 2.0 ** power * TOP[kind] * 1.01 + 1e-30
    status_is(0)


@pytest.mark.parametrize("shape", SHAPES)
@pytest.mark.parametrize("kind,x", [("e4m3", "bf16"), ("int8", "fp16")])
def test_attention_over_scales_of_v_that_are_zero_or_negative(shape, kind, x):
    """A value is code * scale whatever wrote them: codes under a scale of 0 are zeros, a negative one turns signs."""
    rng = np.random.default_rng([len(shape), x == "bf16"])
    pool, s = shaped(shape, kind, x, rng)
    codes = spread_codes(rng, kind)
    only = sorted({0, len(s["lens"]) - 1})
    for sizes in ((1.0, -1.0, 0.0), (-1.0,), (0.0,), (1.0, 0.0), (-40.0, 1.0)):
        rows_of(pool, s, 1, lambda t, sh: (codes(sh), rng.choice(sizes, (len(t), pool.H)) * (1 + rng.random((len(t), pool.H))) / TOP[kind]))
        run_attend(pool, s)
        check_ranges(pool, s, x, shape.startswith("prefix"), only)
    status_is(0)


@pytest.mark.parametrize("shape", SHAPES)
@pytest.mark.parametrize("kind", ["fp16", "e4m3", "int8"])
def test_attention_over_many_small_probabilities(shape, kind):
    """One key above all the others, whose probabilities are then below fp16's normal numbers, but are most of the output."""
    rng = np.random.default_rng([len(shape), 4])
    pool, s = shaped(shape, kind, "fp16", rng, plain_tiles=kind == "fp16")
    n = s["prefix"] or s["lens"][0]
    at = 3
    one = np.zeros((n, pool.H, pool.D))
    key = one.copy()
    key[at] = 1.0
    val = one + 1.0
    val[at] = 0.0
    table = s["shared"] if s["prefix"] else s["table"][0]
    t = np.arange(n)
    for plane, rows in ((0, key), (1, val)):
        if kind == "fp16":
            pool.codes(plane).zero_()
            pool.codes(plane)[dev(table[t // 16]).long(), dev(t % 16)] = torch.from_numpy(rows).half().view(torch.uint8).cuda()
            s["values"][plane] = np64(pool.codes(plane).contiguous().view(torch.float16))
        else:
            rows_of(pool, s, plane, lambda i, sh: (rows[i] if len(i) and i[0] < n and len(i) == n else np.zeros(sh), np.ones(sh[:2])))
    for above in (9.0, 12.0, 14.0):  # natural logarithms: 2^-13 to 2^-20
        q = torch.full(s["q"].shape, above * pool.D ** 0.5 / pool.D).half()
        s["q"] = q
        s["dq"].copy_(q)
        run_attend(pool, s)
        r = 0
        keys, vals = (np.concatenate([tokens_of(v, s["shared"], 0, s["prefix"], 16), tokens_of(v, s["table"][r], 0, s["lens"][r], 16)]) for v in s["values"])
        want, want_lse, mass = orc.attend(np64(q)[r], keys, vals, pool.D ** -0.5)
        # probabilities: half a step of 2^-11 (and the prefix kernel's values, 1, exactly), down to 2^-21 of the largest; below that 2^-32 of it
        most = (2.0 ** -11 * (1 + 2.0 ** -6) + 2.0 ** -15) * mass + len(keys) * 2.0 ** -32 * np.abs(vals).max() + 2.0 ** -11 * np.abs(want) + 2.0 ** -25
        off = np.abs(np64(s["out"])[r] - want)
        assert (off <= most).all(), (above, off.max(), want.max(), (off / most).max())
    status_is(0)


@pytest.mark.parametrize("shape", SHAPES)
@pytest.mark.parametrize("kind", ["bf16", "e4m3", "int8"])
def test_attention_over_values_next_to_the_largest_number(shape, kind):
    """Means of many values near 2^127, whose sums no fp32 holds; equal scores and ordinary ones."""
    rng = np.random.default_rng([len(shape), 12])
    pool, s = shaped(shape, kind, "bf16", rng)
    for equal in (True, False):
        if kind in TOP:
            rows_of(pool, s, 1, lambda t, sh: (np.full(sh, TOP[kind]), np.full(sh[:2], 2.0 ** 127 * 0.9 / TOP[kind])))
        else:
            big = torch.full((pool.blocks, pool.B, pool.H, pool.D), 2.0 ** 127 * 0.9).bfloat16()
            pool.codes(1).copy_(big.view(torch.uint8))
            s["values"][1] = np64(big)
        if equal:
            s["dq"].zero_()
        else:
            s["dq"].copy_(s["q"])
        run_attend(pool, s)
        # a mean of equal numbers is that number: probabilities and their sum are off by a half step of 2^-8 (bf16) or 2^-11 each
        want = s["values"][1].max()
        out = np64(s["out"])[np.array(s["lens"]) + s["prefix"] > 0]
        assert (np.abs(out - want) <= (2.0 ** -8 + 2.0 ** -8 + 2.0 ** -10) * want).all(), (equal, out.min(), out.max(), want)
    status_is(0)


@pytest.mark.parametrize("shape", SHAPES)
@pytest.mark.parametrize("kind", ["e4m3", "int8"])
@pytest.mark.parametrize("bad", [float("inf"), float("-inf"), float("nan")])
def test_attention_over_a_scale_of_v_that_is_not_finite(shape, kind, bad):
    rng = np.random.default_rng([len(shape), 14])
    pool, s = shaped(shape, kind, "bf16", rng)
    R, Hq = s["q"].shape[:2]
    table = s["shared"] if s["prefix"] else s["table"][0]
    pool.codes(1)[int(table[2]), 3, 0] = 0x31  # a code that is not 0
    pool.scale(1)[int(table[2]), 3, 0] = bad
    run_attend(pool, s)
    spoilt = torch.zeros(R, Hq, dtype=torch.bool)
    spoilt[slice(None) if s["prefix"] else 0, : Hq // pool.H] = True
    finite = s["out"].cpu().isfinite()
    assert torch.equal(finite.all(-1), ~spoilt) and torch.equal(finite.any(-1), ~spoilt) and torch.isfinite(s["lse"]).all()
    status_is(0)


# The prefix kernel in the cases that the stream is tested in.
PLAIN = [("bf16", "bf16"), ("fp16", "fp16"), ("bf16", "e4m3"), ("fp16", "int8")]


@pytest.mark.parametrize("shape", PREFIXES)
@pytest.mark.parametrize("x,kind", PLAIN)
@pytest.mark.parametrize("layout,B", [("nhd", 16), ("hnd", 5)])
def test_a_prefix_shared_by_many(shape, x, kind, layout, B):
    rng = np.random.default_rng([len(shape), B])
    pool, s = shaped(shape, kind, x, rng, layout=layout, B=B)
    s["lens"][1] = -1
    s["d"]["lens"][1] = -1
    run_attend(pool, s)
    check(pool, s, x, True, {0, 1, 2, len(s["lens"]) - 1})
    status_is(0)
    # a negative scale, and scores far apart
    for scale in (-0.2, 0.9):
        run_attend(pool, s, scale=scale)
        check(pool, dict(s, q=-s["q"] if scale < 0 else s["q"], scale=abs(scale)), x, True, {0, 2, len(s["lens"]) - 1})
    status_is(0)


@pytest.mark.parametrize("shape", PREFIXES)
@pytest.mark.parametrize("x,kind", PLAIN)
def test_a_prefix_shorter_than_announced_or_out_of_range(shape, x, kind):
    rng = np.random.default_rng([len(shape), 6])
    pool, s = shaped(shape, kind, x, rng)
    full, some = s["prefix"], {0, len(s["lens"]) - 1}
    for n in (full - 1, full // 2 + 3, 129, 128, 1, 0):
        s["d"]["prefix_len"][0] = n
        run_attend(pool, s, max_prefix=full)
        check(pool, dict(s, prefix=n), x, True, some)
    status_is(0)
    for n, cut in ((-7, 0), (full + 5000, full)):
        s["d"]["prefix_len"][0] = n
        run_attend(pool, s, max_prefix=full)
        status_is(tc.TC_DEVICE_BAD_INDEX)
        check(pool, dict(s, prefix=cut), x, True, some)
    # block ids that the pool does not have: their keys are left out, as if the prefix were without them
    s["d"]["prefix_len"][0] = full
    for i, bad in ((2, -1), (9, pool.blocks), (full // 16 - 1, 2 ** 31 - 1)):
        s["d"]["prefix_table"][i] = bad
    run_attend(pool, s)
    status_is(tc.TC_DEVICE_BAD_INDEX)
    keep = [i for i in range(len(s["shared"])) if i not in (2, 9, full // 16 - 1)]
    check(pool, dict(s, prefix=full - 48, shared=s["shared"][keep]), x, True, some)
    status_is(0)


@pytest.mark.parametrize("shape", PREFIXES)
@pytest.mark.parametrize("x,kind,apart", [(x, kind, False) for x, kind in PLAIN] + [("bf16", "e4m3", True), ("bf16", "int8", True)])
def test_a_prefix_with_rows_that_are_not_finite(shape, x, kind, apart):
    rng = np.random.default_rng([len(shape), 8])
    pool, s = shaped(shape, kind, x, rng)
    if apart:  # scales of V far from one another
        pool.scale(1).mul_(dev(10.0 ** rng.uniform(-20, 0, (pool.blocks, pool.B, pool.H)), torch.float32))
    R, Hq = s["q"].shape[:2]
    g = Hq // pool.H
    block = int(s["shared"][7])
    nan = torch.zeros(R, Hq, dtype=torch.bool)
    # V: the outputs of its KV head are NaN, the logarithms are not
    if kind in TOP:
        pool.scale(1)[block, 5, 0] = float("nan")
        pool.codes(1)[block, 5, 0] = 0
    else:
        pool.codes(1)[block, 5, 0] = 0xFF
    run_attend(pool, s)
    nan[:, :g] = True
    out = s["out"].cpu()
    assert torch.equal(out.isnan().all(-1), nan) and torch.equal(out.isnan().any(-1), nan) and torch.isfinite(s["lse"]).all()
    # K: both
    if kind in TOP:
        pool.scale(0)[block, 5, 1] = float("nan")
    else:
        pool.codes(0)[block, 5, 1] = 0xFF
    run_attend(pool, s)
    nan[:, g : 2 * g] = True
    out, lse = s["out"].cpu(), s["lse"].cpu()
    want = torch.zeros_like(nan)
    want[:, g : 2 * g] = True
    assert torch.equal(out.isnan().any(-1), nan) and torch.equal(lse.isnan(), want)
    # a query: its row
    s["dq"][1, 2 * g] = float("nan")
    run_attend(pool, s)
    nan[1, 2 * g] = want[1, 2 * g] = True
    assert torch.equal(s["out"].cpu().isnan().any(-1), nan) and torch.equal(s["lse"].cpu().isnan(), want)
    status_is(0)


@pytest.mark.parametrize("shape", SHAPES)
@pytest.mark.parametrize("x,kind", PLAIN)
def test_attention_into_strided_outputs_from_strided_tables(shape, x, kind):
    """Outputs with heads outside requests and a gap behind every row, tables that are a window of wider ones, no logarithms."""
    rng = np.random.default_rng([len(shape), 17])
    pool, s = shaped(shape, kind, x, rng)
    s["lens"][-2] = -1
    s["d"]["lens"][-2] = -1
    run_attend(pool, s)
    R, Hq, D = s["q"].shape
    whole = torch.full((Hq, R, D + 24), 9.0, dtype=s["q"].dtype, device="cuda")
    wide = torch.full((R, s["table"].shape[1] + 5), -1, dtype=torch.int32, device="cuda")
    wide[:, 3:-2] = s["d"]["tables"]
    want, s["out"] = s["out"], whole.transpose(0, 1)[..., :D]
    run_attend(pool, s, lse=None, tables=wide[:, 3:-2])
    assert torch.equal(s["out"], want) and (whole[..., D:] == 9.0).all()
    check(pool, s, x, shape.startswith("prefix"), {0, R - 2, R - 1})
    status_is(0)


@pytest.mark.parametrize("x,kind,prefix", [("bf16", "bf16", 40000), ("fp16", "int8", 80000)])
def test_a_long_prefix_of_one_request_with_many_heads(x, kind, prefix):
    assert prefix_taken_by(1, 20, 1, 128, 30, prefix, kind in TOP) == "prefix 128"
    rng = np.random.default_rng(prefix)
    pool = Pool(kind, H=1, blocks=prefix // 16 + 4)
    s = attend_case(pool, [30], prefix, 20, x, rng, poison=False)
    run_attend(pool, s)
    check(pool, s, x, True, {0})
    status_is(0)


@pytest.mark.parametrize("shape", ["stream", "prefix 128", "prefix 256"])
@pytest.mark.parametrize("kind", ["bf16", "e4m3"])
def test_a_captured_decode_replays_with_new_lengths(shape, kind):
    """Outputs after every replay, of all requests, the padded ones' untouched."""
    rng = np.random.default_rng([len(shape), 33])
    R, H, g, D, prefix, most = SHAPES[shape]
    assert prefix_taken_by(R, H * g, H, D, most, prefix, kind in TOP) == shape
    pool = Pool(kind, D=D, H=H, blocks=R * -(-most // 16) + -(-prefix // 16) + 3)
    s = attend_case(pool, [most] * R, prefix, H * g, "bf16", rng, poison=False)
    run_attend(pool, s)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        run_attend(pool, s, stream=torch.cuda.current_stream())
    for lens, n in (([most] * R, prefix), (rng.integers(-1, most + 1, R).tolist(), prefix // 3), ([0] * (R - 1) + [-1], 1), (rng.integers(0, 3, R).tolist(), 0), ([most] * R, prefix - 1)):
        s["d"]["lens"].copy_(dev(np.array(lens, dtype=np.int32)))
        s["d"]["prefix_len"].fill_(n)
        s["out"].fill_(9.0), s["lse"].fill_(9.0)
        s["workspace"].fill_(0xFF)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        check(pool, dict(s, lens=lens, prefix=n), "bf16", shape != "stream", set(range(0, R, max(1, R // 6))) | {R - 1})
    status_is(0)


FIRST_CALLS = """
import sys, threading
sys.path[:0] = [{root!r}, {tests!r}]
from test_operators_ranges_gpu import *
rng = np.random.default_rng(5)
cases = [(kind, *shaped(shape, kind, "bf16", rng)) for shape in ("stream", "prefix 128", "prefix 256") for kind in ("bf16", "e4m3") for _ in (0, 1)]
streams = [torch.cuda.Stream() for _ in cases]
torch.cuda.synchronize()
begin = threading.Barrier(len(cases))
failed = []
def go(case, stream):
    kind, pool, s = case
    begin.wait()
    try:
        run_attend(pool, s, stream=stream)
    except Exception as e:
        failed.append(e)
threads = [threading.Thread(target=go, args=x) for x in zip(cases, streams)]
for t in threads: t.start()
for t in threads: t.join()
torch.cuda.synchronize()
assert not failed, failed
for i, (kind, pool, s) in enumerate(cases):
    check(pool, s, "bf16", i >= 4, {{0, len(s["lens"]) - 1}})
print("answered")
"""


def test_threads_may_make_the_first_calls_of_a_process_at_once():
    """Every kernel's first launch, on a stream and a workspace of its own."""
    here = os.path.dirname(os.path.abspath(__file__))
    got = subprocess.run([sys.executable, "-c", FIRST_CALLS.format(root=os.path.dirname(here), tests=here)], capture_output=True, text=True, timeout=300)
    assert got.returncode == 0 and "answered" in got.stdout, got.stderr[-2000:]


WAITS = """
#include "barrier.cuh"
__global__ void waits(int *got)
{
    __shared__ __align__(8) unsigned long long bars[2];
    const uint32_t bar = static_cast<uint32_t>(__cvta_generic_to_shared(bars));
    tc::barrier_init(bar, 1), tc::barrier_init(bar + 8, 1);
    tc::barrier_arrive(bar + 8);
    got[0] = tc::barrier_wait(bar + 8, 0);
    got[1] = tc::barrier_wait(bar + 8, 1);
    got[2] = tc::barrier_wait(bar, 0);
    tc::barrier_arrive(bar);
    got[3] = tc::barrier_wait(bar, 0);
}
extern "C" __attribute__((visibility("default"))) int run(int *got)
{
    waits<<<1, 1>>>(got);
    return static_cast<int>(cudaDeviceSynchronize());
}
"""


def test_waits_of_the_prefix_kernel_end_by_themselves(tmp_path):
    """On a phase that has passed, one that nothing ends (a second or two, then false), and one that ends after that."""
    src, lib = tmp_path / "waits.cu", tmp_path / "waits.so"
    src.write_text(WAITS)
    subprocess.check_call([os.environ.get("NVCC", "/usr/local/cuda/bin/nvcc"), *build.NVCC_FLAGS, "-I", build.CSRC, "-shared", "-cudart", "static", "-o", str(lib), str(src)])
    got = torch.full((4,), 7, dtype=torch.int32, device="cuda")
    torch.cuda.synchronize()
    begin = time.monotonic()
    assert ctypes.CDLL(str(lib)).run(ctypes.c_void_p(got.data_ptr())) == 0
    assert 0.2 < time.monotonic() - begin < 20
    assert got.tolist() == [1, 0, 0, 1]
