"""The operators on a paged layer against the oracle.

What is written or read back as numbers is compared bit for bit with the definition carried out in its own
arithmetic (fp32 steps, each rounded once).  Attention is compared with 64 bits, within a bound derived for every
element from the roundings that the operator makes (see `bound`)."""
import numpy as np
import pytest
import torch

import paper_2608_06007_b200 as tc
from oracle import operators as orc

pytestmark = pytest.mark.gpu

KIND = {"bf16": tc.TC_BF16, "fp16": tc.TC_FP16, "fp32": tc.TC_FP32, "e4m3": tc.TC_E4M3, "int8": tc.TC_INT8}
TORCH = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32, "e4m3": torch.float8_e4m3fn, "int8": torch.int8}
SENTINEL = 0x5A


def np64(t):
    return t.detach().double().cpu().numpy()


class Pool:
    """A layer (the `layer`-th of two) in a pool filled with a sentinel, and its logical [block][slot][head][dim] views."""

    def __init__(self, kind, layout="nhd", blocks=9, B=16, H=2, D=128, gap=0, shift=0, layer=1):
        self.kind, self.layout, self.blocks, self.B, self.H, self.D = kind, layout, blocks, B, H, D
        e = TORCH[kind].itemsize
        self.stride = B * H * D * e + gap
        self.plane = blocks * self.stride + 64
        self.raw = torch.full((4 * self.plane + shift,), SENTINEL, dtype=torch.uint8, device="cuda")
        self.base, self.first = shift, 2 * layer
        pool = tc.pool(tc.TC_NHD if layout == "nhd" else tc.TC_HND, blocks, 1, plane_stride=self.plane, block_stride=self.stride)
        more = {}
        if kind in ("e4m3", "int8"):
            self.scales = torch.full((4, blocks, B * H), -1.0, device="cuda")
            more = dict(scale_pool=tc.pool(pool.layout, blocks, 1, plane_stride=blocks * B * H * 4), scale_bases=[self.scales])
        self.handle = tc.kv_layer(pool, (B, H, D), KIND[kind], [self.raw[shift:]], layer=layer, **more)

    def codes(self, c):
        """A plane as uint8 [blocks, B, H, D * e] (a view)."""
        at = self.base + (self.first + c) * self.plane
        x = self.raw[at : at + self.blocks * self.stride].view(self.blocks, self.stride)[:, : self.B * self.H * self.D * TORCH[self.kind].itemsize]
        x = x.unflatten(1, (self.B, self.H, -1) if self.layout == "nhd" else (self.H, self.B, -1))
        return x if self.layout == "nhd" else x.transpose(1, 2)

    def scale(self, c):
        x = self.scales[self.first + c].view(self.blocks, *((self.B, self.H) if self.layout == "nhd" else (self.H, self.B)))
        return x if self.layout == "nhd" else x.transpose(1, 2)

    def fill(self, rng, spread=1.0):
        """Random contents; returns K and V as 64-bit values [blocks, B, H, D]."""
        got = []
        for c in (0, 1):
            shape = (self.blocks, self.B, self.H, self.D)
            x = (rng.standard_normal(shape) * spread).astype(np.float32)
            if self.kind in ("e4m3", "int8"):
                codes, scale = orc.quantise(x, self.kind)
                self.codes(c).copy_(torch.from_numpy(codes.view(np.uint8)))
                self.scale(c).copy_(torch.from_numpy(scale))
                got.append(orc.values(codes, scale, self.kind))
            else:
                t = torch.from_numpy(x).to(TORCH[self.kind])
                self.codes(c).copy_(t.view(torch.uint8))
                got.append(np64(t))
        return got


def status_is(flags):
    assert tc.tc_device_status() == flags


def dev(x, dtype=None):
    return torch.as_tensor(np.ascontiguousarray(x), dtype=dtype).cuda()


# ---------------------------------------------------------------------------------------- append
def append_case(pool, n, Hq, x, rot, interleaved, rng, positions=64, fused=True, mutate=None):
    """Runs an append and returns everything that the oracle needs."""
    H, D = pool.H, pool.D
    qkv = torch.from_numpy(rng.standard_normal((n, Hq + 2 * H, D)).astype(np.float32)).to(TORCH[x])
    if mutate is not None:
        mutate(qkv)
    d = qkv.cuda()
    q, k, v = (d[:, :Hq], d[:, Hq : Hq + H], d[:, Hq + H :]) if fused else [t.contiguous() for t in (d[:, :Hq], d[:, Hq : Hq + H], d[:, Hq + H :])]
    slots = rng.permutation(pool.blocks * pool.B)[:n].astype(np.int64)
    pos = rng.integers(0, positions, n)
    angle = np.arange(positions)[:, None] * 50.0 ** (-np.arange(rot // 2) / max(1, rot // 2))
    cos, sin = np.cos(angle).astype(np.float32), np.sin(angle).astype(np.float32)
    return dict(qkv=qkv, q=q, k=k, v=v, q_out=torch.full((n, Hq, D), 7.0, dtype=TORCH[x], device="cuda"), slots=slots, pos=pos, cos=cos, sin=sin, rot=rot, interleaved=interleaved, Hq=Hq)


def run_append(pool, s, q=True, stream=None):
    rope = dict(positions=dev(s["pos"]), cos=dev(s["cos"]), sin=dev(s["sin"]), interleaved=s["interleaved"]) if s["rot"] else {}
    tc.tc_kv_append(pool.handle, s["k"], s["v"], dev(s["slots"]), **(dict(q=s["q"], q_out=s["q_out"]) if q else {}), **rope, stream=stream)


def expect_append(pool, s, live=None):
    """(q rows fp32, per plane: stored bytes [n, H, D*e], scales)."""
    x = s["qkv"].float().numpy()
    H, Hq = pool.H, s["Hq"]
    with np.errstate(all="ignore"):
        turned = orc.rotate(x[:, : Hq + H], s["cos"][s["pos"]], s["sin"][s["pos"]], s["interleaved"]) if s["rot"] else x[:, : Hq + H].copy()
    rows = []
    for y in (turned[:, Hq:], x[:, Hq + H :]):
        y = np.ascontiguousarray(y)
        if pool.kind in ("e4m3", "int8"):
            codes, scale = orc.quantise(y, pool.kind)
            rows.append((torch.from_numpy(codes.view(np.uint8)), torch.from_numpy(scale)))
        else:
            rows.append((torch.from_numpy(y).to(TORCH[pool.kind]).view(torch.uint8), None))
    return torch.from_numpy(turned[:, :Hq].copy()).to(s["qkv"].dtype), rows


def check_append(pool, s, q=True):
    live = np.flatnonzero((s["slots"] >= 0) & (s["slots"] < pool.blocks * pool.B) & ((s["rot"] == 0) | ((s["pos"] >= 0) & (s["pos"] < len(s["cos"])))))
    keep = dict(s, pos=np.clip(s["pos"], 0, len(s["cos"]) - 1))
    want_q, rows = expect_append(pool, keep)
    q_out = torch.full_like(s["q_out"].cpu(), 7.0)
    if q:
        q_out[live] = want_q[live]
    assert torch.equal(s["q_out"].cpu().view(torch.uint8), q_out.view(torch.uint8))
    want = pool.raw.cpu().clone().fill_(SENTINEL)
    block, at = torch.from_numpy(s["slots"][live] // pool.B), torch.from_numpy(s["slots"][live] % pool.B)
    device, scales = pool.raw, getattr(pool, "scales", None)
    got = pool.raw.cpu()
    pool.raw = want  # the views of the expected bytes
    if scales is not None:
        got_scales = scales.cpu()
        pool.scales = torch.full_like(got_scales, -1.0)
    try:
        for c, (bytes_, scale) in enumerate(rows):
            pool.codes(c)[block, at] = bytes_[live]
            if scale is not None:
                pool.scale(c)[block, at] = scale[live]
        if scales is not None:
            assert torch.equal(torch.nan_to_num(pool.scales, nan=-5.0), torch.nan_to_num(got_scales, nan=-5.0))
    finally:
        pool.raw = device
        if scales is not None:
            pool.scales = scales
    assert torch.equal(got, want)  # the whole allocation: rows, gaps, other layers


@pytest.mark.parametrize("kind", ["bf16", "fp16", "fp32", "e4m3", "int8"])
@pytest.mark.parametrize("x", ["bf16", "fp16", "fp32"])
@pytest.mark.parametrize("interleaved", [False, True])
def test_append_types_and_rotations(kind, x, interleaved):
    rng = np.random.default_rng([KIND[kind], KIND[x], interleaved])
    for D, rot in ((128, 128), (128, 32), (80, 16), (100, 50), (64, 0), (40, 24)):
        pool = Pool(kind, layout="hnd" if interleaved else "nhd", D=D, H=3, B=16, gap=32)
        s = append_case(pool, 37, 7, x, rot, interleaved, rng)
        s["slots"][5] = s["slots"][36] = -1
        run_append(pool, s)
        check_append(pool, s)
    status_is(0)


@pytest.mark.parametrize("D,H,Hq,n,B", [(1, 1, 1, 1, 1), (2, 3, 5, 9, 7), (65, 2, 4, 33, 5), (256, 1, 1, 3, 16), (512, 2, 3, 5, 4), (16, 1, 40, 70, 3), (8, 64, 64, 2, 2), (504, 1, 2, 4, 3), (256, 1, 21, 3, 4), (512, 6, 9, 3, 4), (16, 200, 3, 5, 2)])
@pytest.mark.parametrize("kind", ["bf16", "e4m3", "int8"])
def test_append_sizes(D, H, Hq, n, B, kind):
    rng = np.random.default_rng([D, H, n])
    for rot in {0, D // 2 // 2 * 2, D // 2 * 2, D // 32 * 16}:
        pool = Pool(kind, D=D, H=H, B=B, blocks=max(4, -(-n // B) + 1))
        s = append_case(pool, n, Hq, "bf16", rot, rot % 4 == 0, rng)
        run_append(pool, s)
        check_append(pool, s)
    status_is(0)


@pytest.mark.parametrize("shift,gap", [(2, 0), (0, 2), (8, 8), (4, 12)])
def test_append_into_a_pool_off_16_bytes(shift, gap):
    rng = np.random.default_rng([shift, gap])
    for kind in ("bf16", "e4m3"):
        pool = Pool(kind, shift=shift, gap=gap, D=64, layer=0)
        s = append_case(pool, 20, 4, "bf16", 32, False, rng)
        run_append(pool, s)
        check_append(pool, s)
    status_is(0)


def test_append_without_queries_in_place_and_from_strided_inputs():
    rng = np.random.default_rng(5)
    for D, rot in ((128, 64), (100, 50)):
        pool = Pool("bf16", D=D)
        s = append_case(pool, 19, 4, "bf16", rot, False, rng)
        run_append(pool, s, q=False)
        check_append(pool, s, q=False)
        # queries rotated in place, inside the projection's own output
        pool = Pool("int8", D=D)
        s = append_case(pool, 19, 4, "bf16", rot, True, rng)
        s["q_out"] = s["q"]
        run_append(pool, s)
        want_q, _ = expect_append(pool, s)
        assert torch.equal(s["q"].cpu(), want_q)
        # heads before tokens, and one K head broadcast to all
        pool = Pool("e4m3", D=D)
        s = append_case(pool, 19, 4, "fp32", rot, False, rng, fused=False)
        s["q"] = s["q"].transpose(0, 1).contiguous().transpose(0, 1)
        s["k"] = s["k"][:, :1].expand(-1, pool.H, -1)
        s["qkv"][:, 4 : 4 + pool.H] = s["qkv"][:, 4:5].clone()
        run_append(pool, s)
        check_append(pool, s)
    status_is(0)


def test_append_rows_that_are_not_finite_zero_or_tiny():
    def mutate(x):
        x[0, 5, 3] = float("nan")   # K head
        x[1, 5, 3] = float("inf")
        x[2, 7, 0] = float("-inf")  # V head
        x[3] = 0
        x[4] = 1e-38 if x.dtype == torch.float32 else 0
        x[5] *= 1e30 if x.dtype == torch.float32 else 1
        x[6, 4:] = 1e-41 if x.dtype == torch.float32 else 0
        x[7] *= 5e37                # products and quotients next to the largest numbers
        x[8] *= 1e-36
        x[9] *= 3e-24               # scales on both sides of 2^-80
        x[10] *= 4e-22

    rng = np.random.default_rng(6)
    for kind in ("e4m3", "int8", "fp32"):
        for x in ("fp32", "bf16"):
            for rot in (0, 128):
                pool = Pool(kind)
                s = append_case(pool, 12, 4, x, rot, False, rng, mutate=mutate)
                # a rotation makes NaN of any sign out of an infinity: those elements are compared as NaN
                run_append(pool, s)
                if kind == "fp32" and rot:
                    for c, (bytes_, _) in enumerate(expect_append(pool, s)[1]):
                        got = pool.codes(c).cpu()[torch.from_numpy(s["slots"] // 16), torch.from_numpy(s["slots"] % 16)].contiguous().view(torch.float32)
                        assert torch.equal(torch.nan_to_num(got, nan=3.5), torch.nan_to_num(bytes_.view(torch.float32), nan=3.5))
                else:
                    check_append(pool, s)
    status_is(0)


def test_append_leaves_out_what_is_out_of_range_and_says_so():
    rng = np.random.default_rng(7)
    for D in (128, 100):
        pool = Pool("e4m3", D=D)
        s = append_case(pool, 24, 4, "bf16", 32, False, rng)
        limit = pool.blocks * pool.B
        s["slots"][[1, 2, 3]] = [limit, 1 << 40, -(1 << 50)]
        s["pos"][[7, 8]] = [64, -1]
        run_append(pool, s)
        check_append(pool, s)
        status_is(tc.TC_DEVICE_BAD_INDEX)
        status_is(0)


def test_append_to_blocks_past_32_bits_of_bytes():
    blocks, B, H, D = 600, 64, 8, 128
    gap = 8 << 20  # 600 blocks 8 MiB apart: 5 GB from the first to the last
    pool = Pool("bf16", blocks=blocks, B=B, H=H, D=D, gap=gap, layer=0)
    rng = np.random.default_rng(8)
    s = append_case(pool, 6, 2, "bf16", 0, False, rng)
    s["slots"][:] = [0, 599 * 64 + 63, 520 * 64, 300 * 64 + 1, 511 * 64 + 63, 512 * 64]
    run_append(pool, s)
    _, rows = expect_append(pool, s)
    for c in (0, 1):
        got = torch.stack([pool.codes(c)[t // 64, t % 64] for t in s["slots"].tolist()]).cpu()
        assert torch.equal(got, rows[c][0])
    out = [torch.zeros(6, H, D, dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    tc.tc_kv_gather(pool.handle, dev(np.array([[0, 599], [599, 0]], dtype=np.int32)), dev(np.array([0, 1, 2])), out[0][:2], out[1][:2], first=dev(np.array([0, 63])))
    for c in (0, 1):
        assert torch.equal(out[c][:2].cpu().view(torch.uint8), rows[c][0][:2])
    status_is(0)


# ---------------------------------------------------------------------------------------- gather
def tables_for(lens, pool, rng, width=None):
    need = [-(-t // pool.B) for t in lens]
    ids = rng.permutation(pool.blocks)[: sum(need)].astype(np.int32)
    table = np.full((max(1, len(lens)), width or max(1, max(need, default=0))), -1, dtype=np.int32)
    at = 0
    for r, m in enumerate(need):
        table[r, :m] = ids[at : at + m]
        at += m
    return table


def tokens_of(values, table, lo, hi, B):
    t = np.arange(lo, hi)
    return values[table[t // B], t % B]


@pytest.mark.parametrize("kind", ["bf16", "fp16", "fp32", "e4m3", "int8"])
@pytest.mark.parametrize("out", ["bf16", "fp16", "fp32"])
@pytest.mark.parametrize("D,layout,B,shift", [(128, "nhd", 16, 0), (80, "hnd", 5, 0), (65, "nhd", 3, 0), (64, "hnd", 16, 4), (256, "nhd", 1, 0), (4, "nhd", 2, 0)])
def test_gather_reads_back_the_values(kind, out, D, layout, B, shift):
    rng = np.random.default_rng([KIND[kind], KIND[out], D])
    lens = [37, 0, 1, 100, 0, 2 * B, 5]
    pool = Pool(kind, layout=layout, D=D, H=3, B=B, blocks=-(-160 // B) + 9, shift=shift, gap=16)
    values = pool.fill(rng)
    table = tables_for(lens, pool, rng)
    off = np.concatenate([[0], np.cumsum(lens)])
    k, v = (torch.full((off[-1] + 4, 3, D), 9.0, dtype=TORCH[out], device="cuda") for _ in range(2))
    tc.tc_kv_gather(pool.handle, dev(table), dev(off), k, v)
    for got, x in ((k, values[0]), (v, values[1])):
        want = np.concatenate([tokens_of(x, table[r], 0, n, B) for r, n in enumerate(lens)])
        # code * scale is one fp32 product, then one rounding to the output's type
        want = torch.from_numpy(want.astype(np.float32)).to(TORCH[out])
        assert torch.equal(got[: off[-1]].cpu(), want)
        assert (got[off[-1] :] == 9.0).all()  # rows behind the last request
    status_is(0)


def test_gather_of_one_plane_a_window_of_tokens_and_strided_outputs():
    rng = np.random.default_rng(11)
    pool = Pool("int8", D=96, H=2, B=4, blocks=60)
    values = pool.fill(rng)
    lens, first = [10, 7, 23], np.array([3, 60, 0])
    table = rng.permutation(60)[: 3 * 20].reshape(3, 20).astype(np.int32)
    wide = torch.zeros(3, 40, dtype=torch.int32, device="cuda")
    wide[:, :20] = dev(table)
    off = np.concatenate([[0], np.cumsum(lens)])
    v = torch.zeros(2, 40, 96, dtype=torch.float16, device="cuda").transpose(0, 1)  # heads outside tokens
    tc.tc_kv_gather(pool.handle, wide[:, :20], dev(off), None, v, first=dev(first))
    want = np.concatenate([tokens_of(values[1], table[r], first[r], first[r] + n, 4) for r, n in enumerate(lens)])
    assert torch.equal(v[:40].cpu(), torch.from_numpy(want.astype(np.float32)).half())
    k = torch.zeros(40, 2, 96, dtype=torch.float16, device="cuda")
    tc.tc_kv_gather(pool.handle, wide[:, :20], dev(off), k, first=dev(first))
    want = np.concatenate([tokens_of(values[0], table[r], first[r], first[r] + n, 4) for r, n in enumerate(lens)])
    assert torch.equal(k.cpu(), torch.from_numpy(want.astype(np.float32)).half())
    status_is(0)


def test_gather_leaves_out_what_is_out_of_range_and_says_so():
    rng = np.random.default_rng(12)
    pool = Pool("bf16", D=64, H=2, B=4, blocks=8)
    values = pool.fill(rng)
    table = np.array([[1, 8, 2], [-1, 3, 4], [5, 6, 7]], dtype=np.int32)
    off, first = np.array([0, 12, 20, 40]), np.array([0, 2, 0])
    k = torch.full((32, 2, 64), 9.0, dtype=torch.bfloat16, device="cuda")
    v = k.clone()
    tc.tc_kv_gather(pool.handle, dev(table), dev(off), k, v, first=dev(first))
    want = np.full((32, 2, 64), 9.0)
    for r in range(3):
        for i in range(off[r + 1] - off[r]):
            t, row = first[r] + i, off[r] + i
            if row < 32 and t // 4 < 3 and 0 <= table[r, t // 4] < 8:
                want[row] = values[0][table[r, t // 4], t % 4]
    assert np.array_equal(np64(k), want)
    status_is(tc.TC_DEVICE_BAD_INDEX)
    status_is(0)


# ------------------------------------------------------------------------------------- attention
def bound(q, keys, vals, scale, out, mass, x, quantised):
    """Most that a row of outputs may be off.  Each probability is rounded once, to 16 bits: half a step u_p of
    it (bf16 with a quantised pool, whatever the queries are), so u_p * sum w|v|.  A score is an fp32 sum of D exact
    products and three fp32 factors: off by at most (D + 4) 2^-24 scale sum |q k|, which moves weights by
    twice that relatively; the exponential is good to 2^-21.  The output is rounded once, half a step u_o; in fp16
    numbers below 2^-14 have steps of 2^-24, so there half a step is 2^-25 (an output of 1e-18 becomes 0).
    Half-precision probabilities below 2^-14 of the row's reference have a step of 2^-24 instead; the largest
    probability is at least 1, so each is off by 2^-25 of the sum at most."""
    u_o = torch.finfo(TORCH[x]).eps / 2
    u_p = torch.finfo(torch.bfloat16).eps / 2 if quantised else u_o
    if not len(keys):
        return np.zeros_like(out)
    g = q.shape[0] // keys.shape[1]
    k, v = np.repeat(keys, g, axis=1), np.repeat(vals, g, axis=1)
    delta = (q.shape[-1] + 4) * 2.0 ** -24 * scale * np.einsum("hd,nhd->nh", np.abs(q), np.abs(k)).max(0)
    tiny = len(keys) * 2.0 ** -25 * np.abs(v).max(0) if u_p < 2.0 ** -9 else 0
    return (u_p * (1 + 2.0 ** -6) + 2 * delta[:, None] + 2.0 ** -18) * mass + tiny + u_o * (1 + 2.0 ** -6) * np.abs(out) + (2.0 ** -25 if x == "fp16" else 1e-30)


def attend_case(pool, lens, prefix, Hq, x, rng, spread=1.0, scale=None, strided=False, poison=True):
    values = pool.fill(rng, spread)
    own = [max(0, n) for n in lens]
    both = tables_for(own + [prefix], pool, rng)
    table, shared = both[:-1], both[-1][: max(1, -(-prefix // pool.B))]
    if poison:  # slots that no key is in hold NaN (e4m3: scales)
        used = np.zeros((pool.blocks, pool.B), dtype=bool)
        for tab, n in list(zip(table, own)) + [(shared, prefix)]:
            t = np.arange(n)
            used[tab[t // pool.B], t % pool.B] = True
        idle = torch.from_numpy(~used).cuda()
        for c in (0, 1):
            if pool.kind in ("e4m3", "int8"):
                pool.scale(c)[idle] = float("nan")
            else:
                pool.codes(c)[idle] = 0xFF
    R = len(lens)
    q = torch.from_numpy(rng.standard_normal((R, Hq, pool.D)).astype(np.float32) * spread).to(TORCH[x])
    dq = q.cuda()
    if strided:
        dq = torch.zeros(Hq, R, pool.D + 16, dtype=q.dtype, device="cuda").transpose(0, 1)[..., : pool.D]
        dq.copy_(q)
    s = dict(q=q, dq=dq, lens=lens, prefix=prefix, table=table, shared=shared, values=values, scale=scale or 0.0, max_len=max(1, max(own)),
             out=torch.full((R, Hq, pool.D), 9.0, dtype=q.dtype, device="cuda"), lse=torch.full((R, Hq), 9.0, device="cuda"))
    s["d"] = dict(tables=dev(table), lens=dev(np.array(lens, dtype=np.int32)), prefix_table=dev(shared), prefix_len=dev(np.array([prefix], dtype=np.int32)))
    s["workspace"] = torch.full((tc.tc_attn_workspace_bytes(pool.handle, dq, max_len=s["max_len"], max_prefix=prefix) + 16,), 0xFF, dtype=torch.uint8, device="cuda")
    return s


def run_attend(pool, s, **changes):
    args = dict(max_len=s["max_len"], max_prefix=s["prefix"], scale=s["scale"], lse=s["lse"], workspace=s["workspace"]) | s["d"] | changes
    tc.tc_attn_decode(pool.handle, s["dq"], s["out"], args.pop("tables"), args.pop("lens"), **args)


def check_attend(pool, s, x, only=None):
    D, scale = pool.D, s["scale"] or pool.D ** -0.5
    out, lse, q = np64(s["out"]), np64(s["lse"]), np64(s["q"])
    kv = [tokens_of(v, s["shared"], 0, s["prefix"], pool.B) for v in s["values"]]
    for r, n in enumerate(s["lens"]):
        if only is not None and r not in only:
            continue
        if n < 0:
            assert (out[r] == 9.0).all() and (lse[r] == 9.0).all()
            continue
        keys, vals = (np.concatenate([kv[c], tokens_of(s["values"][c], s["table"][r], 0, n, pool.B)]) for c in (0, 1))
        want, want_lse, mass = orc.attend(q[r], keys, vals, scale)
        off = np.abs(out[r] - want)
        most = bound(q[r], keys, vals, scale, want, mass, x, pool.kind in ("e4m3", "int8"))
        assert (off <= most).all(), (r, n, off.max(), (off - most).max())
        if not len(keys):
            assert (lse[r] == -np.inf).all()
            continue
        g = s["q"].shape[1] // pool.H
        delta = (D + 4) * 2.0 ** -24 * scale * np.einsum("hd,nhd->nh", np.abs(q[r]), np.abs(np.repeat(keys, g, axis=1))).max(0)
        assert (np.abs(lse[r] - want_lse) <= delta + 2.0 ** -18 + 2.0 ** -22 * np.abs(want_lse)).all()


@pytest.mark.parametrize("x,kind", [("bf16", "bf16"), ("fp16", "fp16"), ("bf16", "e4m3"), ("fp16", "e4m3"), ("bf16", "int8"), ("fp16", "int8")])
@pytest.mark.parametrize("D,H,g,B,layout", [(128, 2, 4, 16, "nhd"), (64, 1, 1, 5, "hnd"), (80, 3, 7, 16, "hnd"), (256, 1, 20, 8, "nhd"), (16, 2, 16, 1, "nhd"), (192, 1, 3, 32, "hnd"), (112, 2, 17, 7, "nhd")])
def test_attention_types_and_shapes(x, kind, D, H, g, B, layout):
    rng = np.random.default_rng([KIND[kind], KIND[x], D, B])
    lens, prefix = [37, 1, 0, -1, 130, 64], 77
    pool = Pool(kind, layout=layout, D=D, H=H, B=B, blocks=-(-330 // B) + 8, gap=16)
    s = attend_case(pool, lens, prefix, H * g, x, rng, strided=B == 16)
    run_attend(pool, s)
    check_attend(pool, s, x)
    status_is(0)


@pytest.mark.parametrize("lens,prefix", [([0], 0), ([1], 0), ([0], 1), ([0, 0, 0], 5), ([1, 2, 3], 1), ([-1, -1], 40), ([15, 16, 17, 63, 64, 65], 16), ([2000], 0), ([3, 1500], 1111), ([5] * 70, 200), ([0, 7] * 150, 64)])
@pytest.mark.parametrize("kind", ["bf16", "int8"])
def test_attention_lengths(lens, prefix, kind):
    rng = np.random.default_rng([len(lens), prefix, 3])
    pool = Pool(kind, blocks=sum(-(-max(0, n) // 16) for n in lens) + -(-prefix // 16) + 3)
    s = attend_case(pool, lens, prefix, 8, "bf16", rng)
    run_attend(pool, s)
    check_attend(pool, s, "bf16")
    status_is(0)


@pytest.mark.parametrize("R,prefix,D,x,kind", [(9, 1000, 128, "bf16", "bf16"), (64, 777, 128, "fp16", "fp16"), (33, 513, 64, "bf16", "e4m3"), (130, 300, 128, "bf16", "int8"), (40, 700, 80, "fp16", "e4m3"), (65, 129, 96, "bf16", "bf16"), (12, 450, 256, "bf16", "bf16")])
def test_attention_over_a_prefix_shared_by_many(R, prefix, D, x, kind):
    rng = np.random.default_rng([R, prefix])
    lens = rng.integers(-1, 20, R).tolist()
    pool = Pool(kind, D=D, H=2, B=16, blocks=R * 2 + prefix // 16 + 4, layout="hnd" if R % 2 else "nhd")
    s = attend_case(pool, lens, prefix, 8, x, rng, spread=1.7)
    run_attend(pool, s)
    check_attend(pool, s, x)
    status_is(0)


@pytest.mark.parametrize("x,kind", [("bf16", "bf16"), ("fp16", "fp16"), ("bf16", "e4m3"), ("fp16", "int8")])
@pytest.mark.parametrize("R,H,g,prefix,D,B", [(160, 8, 4, 6000, 128, 16), (70, 8, 7, 2500, 64, 5), (30, 8, 4, 5001, 128, 32), (12, 16, 5, 9000, 80, 16), (300, 3, 1, 4096, 128, 1)])
def test_attention_over_many_tiles_of_a_prefix(x, kind, R, H, g, prefix, D, B):
    """Every CTA of the prefix goes round its ring of tiles several times, with one block of rows and with several."""
    rng = np.random.default_rng([R, prefix, KIND[kind]])
    lens = rng.integers(0, 3, R).tolist()
    pool = Pool(kind, D=D, H=H, B=B, blocks=2 * R + prefix // B + 4, layout="hnd" if R % 4 else "nhd")
    s = attend_case(pool, lens, prefix, H * g, x, rng, spread=1.3)
    run_attend(pool, s)
    check_attend(pool, s, x, only={0, 1, R // 2, R - 1})
    assert torch.isfinite(s["out"].float()).all() and torch.isfinite(s["lse"]).all()
    status_is(0)


@pytest.mark.parametrize("kind", ["e4m3", "int8"])
@pytest.mark.parametrize("R,prefix", [(2, 0), (2, 70), (40, 200), (80, 1000)])
def test_attention_over_values_of_very_different_sizes(kind, R, prefix):
    """Rows of V from 1e-30 to 1e30, and rows of zeros, in one request: no common scale."""
    rng = np.random.default_rng([R, prefix])
    lens = rng.integers(1, 90, R).tolist()
    pool = Pool(kind, blocks=sum(-(-n // 16) for n in lens) + prefix // 16 + 4)
    s = attend_case(pool, lens, prefix, 8, "bf16", rng, poison=False)
    for power in ((-3, 4), (-30, -20), (20, 29)):
        v = (rng.standard_normal((pool.blocks, pool.B, pool.H, pool.D)) * 10.0 ** rng.integers(*power, (pool.blocks, pool.B, pool.H, 1))).astype(np.float32)
        v[rng.random(v.shape[:3]) < 0.1] = 0
        codes, scale = orc.quantise(v, kind)
        pool.codes(1).copy_(torch.from_numpy(codes.view(np.uint8)))
        pool.scale(1).copy_(torch.from_numpy(scale))
        s["values"] = [s["values"][0], orc.values(codes, scale, kind)]
        run_attend(pool, s)
        check_attend(pool, s, "bf16")
    status_is(0)


@pytest.mark.parametrize("kind", ["e4m3", "int8"])
@pytest.mark.parametrize("R,prefix", [(2, 0), (2, 40), (30, 200)])
def test_attention_where_a_quantised_row_was_not_finite(kind, R, prefix):
    rng = np.random.default_rng([R, prefix, 9])
    pool = Pool(kind, blocks=R * 4 + 20)
    s = attend_case(pool, [50] * R, prefix, 8, "bf16", rng)
    block = int(s["table"][1, 1])
    pool.scale(1)[block, 5, 0] = float("nan")  # V: the outputs are NaN, the logarithms are not
    pool.codes(1)[block, 5, 0] = 0
    run_attend(pool, s)
    nan = torch.zeros(R, 8, dtype=torch.bool)
    nan[1, :4] = True
    out = s["out"].cpu()
    assert torch.equal(out.isnan().all(-1), nan) and torch.equal(out.isnan().any(-1), nan) and torch.isfinite(s["lse"]).all()
    pool.scale(0)[block, 5, 1] = float("nan")  # K: both
    run_attend(pool, s)
    nan[1, 4:] = True
    out = s["out"].cpu()
    assert torch.equal(out.isnan().any(-1), nan) and torch.equal(s["lse"].cpu().isnan(), nan & (torch.arange(8) >= 4))
    status_is(0)


def test_attention_with_a_negative_scale():
    rng = np.random.default_rng(27)
    for kind, x in (("bf16", "bf16"), ("int8", "fp16")):
        pool = Pool(kind, blocks=60)
        s = attend_case(pool, [30, 40, 5, 0, 17], 300, 16, x, rng, scale=-0.2)
        s["scale"] = -0.2
        run_attend(pool, s)
        check = dict(s, q=-s["q"], scale=0.2)  # the same scores
        check_attend(pool, check, x)
    status_is(0)


def test_attention_with_scores_far_apart_and_a_given_scale():
    rng = np.random.default_rng(21)
    for kind, x in (("bf16", "bf16"), ("fp16", "fp16"), ("e4m3", "bf16"), ("int8", "fp16")):
        pool = Pool(kind, blocks=60)
        s = attend_case(pool, [300, 40, 5], 400, 8, x, rng, spread=4.0, scale=0.7)  # scores of some hundreds
        run_attend(pool, s)
        check_attend(pool, s, x)
    status_is(0)


def test_attention_where_keys_or_queries_are_not_finite():
    rng = np.random.default_rng(22)
    pool = Pool("bf16", blocks=30)
    s = attend_case(pool, [40, 40, 40, 40], 33, 8, "bf16", rng)
    s["dq"][1, 2] = float("nan")                       # one row of one request
    k = pool.codes(0).view(torch.bfloat16)
    block = int(s["table"][2, 0])
    k[block, 3, 0, 0] = float("inf")                   # a key of request 2, KV head 0
    sign = s["dq"][2, :4, 0] > 0
    run_attend(pool, s)
    out, lse = s["out"].cpu(), s["lse"].cpu()
    nan = torch.zeros(4, 8, dtype=torch.bool)
    nan[1, 2] = True
    nan[2, :4] = sign.cpu()                            # exp(inf - inf); a score of -inf just drops the key
    assert torch.equal(out.isnan().all(-1), nan) and torch.equal(out.isnan().any(-1), nan) and torch.equal(lse.isnan(), nan)
    # every score -inf: the key's first element is infinite, all queries have the other sign
    s["dq"][3, :, 0] = -1.0
    for t in range(40):
        k[int(s["table"][3, t // 16]), t % 16, :, 0] = float("inf")
    run_attend(pool, s, max_prefix=0)
    assert (s["out"][3] == 0).all() and (s["lse"][3] == float("-inf")).all()
    status_is(0)


def test_attention_leaves_out_what_is_out_of_range_and_says_so():
    rng = np.random.default_rng(23)
    pool = Pool("bf16", blocks=30)
    s = attend_case(pool, [40, 33], 50, 8, "bf16", rng)
    s["d"]["tables"][0, 1] = 30
    s["d"]["prefix_table"][2] = -1
    run_attend(pool, s)
    values = s["values"]
    for r, n in enumerate([40, 33]):
        own = [t for t in range(n) if not (r == 0 and 16 <= t < 32)]
        shared = [t for t in range(50) if not 32 <= t < 48]
        keys, vals = (np.concatenate([x[s["shared"][np.array(shared) // 16], np.array(shared) % 16], x[s["table"][r][np.array(own) // 16], np.array(own) % 16]]) for x in values)
        want, _, mass = orc.attend(np64(s["q"])[r], keys, vals, 128 ** -0.5)
        assert (np.abs(np64(s["out"])[r] - want) <= bound(np64(s["q"])[r], keys, vals, 128 ** -0.5, want, mass, "bf16", False)).all()
    status_is(tc.TC_DEVICE_BAD_INDEX)
    # lengths past the promised bounds are cut to them
    s = attend_case(pool, [40, 33], 50, 8, "bf16", rng)
    s["d"]["lens"][0] = 4000
    s["d"]["prefix_len"][0] = 5000
    run_attend(pool, s)
    check_attend(pool, s, "bf16")
    status_is(tc.TC_DEVICE_BAD_INDEX)
    # a length where none was announced
    run_attend(pool, s, max_len=0, max_prefix=0, tables=s["d"]["tables"])
    assert (s["out"] == 0).all() and (s["lse"] == float("-inf")).all()
    status_is(tc.TC_DEVICE_BAD_INDEX)
    s["d"]["prefix_len"][0] = -3
    s["d"]["lens"][0] = 40
    run_attend(pool, s)
    s["prefix"] = 0
    check_attend(pool, s, "bf16")
    status_is(tc.TC_DEVICE_BAD_INDEX)
    status_is(0)


def test_attention_reads_pages_past_32_bits_of_bytes():
    pool = Pool("bf16", blocks=600, B=16, H=1, gap=8 << 20, layer=0)
    for c in (0, 1):
        pool.codes(c).zero_()
    table = np.array([[599, 0, 515, 511]], dtype=np.int32)
    rng = np.random.default_rng(24)
    x = rng.standard_normal((2, 4, 16, 1, 128)).astype(np.float32)
    for c in (0, 1):
        for i, blk in enumerate(table[0]):
            pool.codes(c)[int(blk)] = torch.from_numpy(x[c, i]).bfloat16().view(torch.uint8).cuda()
    vals = [np64(torch.from_numpy(x[c]).bfloat16()).reshape(64, 1, 128) for c in (0, 1)]
    q = torch.from_numpy(rng.standard_normal((1, 4, 128)).astype(np.float32)).bfloat16()
    for prefix in (0, 64):
        out = torch.zeros(1, 4, 128, dtype=torch.bfloat16, device="cuda")
        n = 64 - prefix
        ws = torch.empty(tc.tc_attn_workspace_bytes(pool.handle, q, max_len=64, max_prefix=prefix), dtype=torch.uint8, device="cuda")
        tc.tc_attn_decode(pool.handle, q.cuda(), out, dev(table), dev(np.array([n], dtype=np.int32)), max_len=64, workspace=ws, prefix_table=dev(table[0]), prefix_len=dev(np.array([prefix], dtype=np.int32)), max_prefix=prefix)
        want, _, mass = orc.attend(np64(q)[0], *vals, 128 ** -0.5)
        assert (np.abs(np64(out)[0] - want) <= bound(np64(q)[0], *vals, 128 ** -0.5, want, mass, "bf16", False)).all()
    status_is(0)


# -------------------------------------------------------------------------- streams, graphs, the run
def test_other_streams_and_replays_with_new_lengths():
    """Two captured steps on their own streams and workspaces, replayed together and with other lengths and slots."""
    rng = np.random.default_rng(31)
    steps = []
    for kind in ("bf16", "e4m3"):
        pool = Pool(kind, blocks=80)
        s = attend_case(pool, [40, 33, 100, -1], 200, 8, "bf16", rng, poison=False)
        app = append_case(pool, 4, 8, "bf16", 64, False, rng)
        free = np.setdiff1d(np.arange(80), np.concatenate([s["table"].ravel(), s["shared"]]))
        app["slots"] = free[:4].astype(np.int64) * 16
        d = dict(slots=dev(app["slots"]), pos=dev(app["pos"]), cos=dev(app["cos"]), sin=dev(app["sin"]))
        steps.append((pool, s, app, d, torch.cuda.Stream()))
    torch.cuda.synchronize()
    graphs = []
    for pool, s, app, d, stream in steps:
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=stream):
            tc.tc_kv_append(pool.handle, app["k"], app["v"], d["slots"], q=app["q"], q_out=s["dq"], positions=d["pos"], cos=d["cos"], sin=d["sin"], stream=torch.cuda.current_stream())
            run_attend(pool, s, stream=torch.cuda.current_stream())
        graphs.append(graph)
    for lens, prefix in (([40, 33, 100, -1], 200), ([1, -1, 64, 17], 0), ([0, 0, 100, 100], 199)):
        for (pool, s, app, d, stream), graph in zip(steps, graphs):
            s["d"]["lens"].copy_(dev(np.array(lens, dtype=np.int32)))
            s["d"]["prefix_len"].fill_(prefix)
            s["out"].fill_(9.0), s["lse"].fill_(9.0)
        torch.cuda.synchronize()
        for _ in range(3):
            for (pool, s, app, d, stream), graph in zip(steps, graphs):
                with torch.cuda.stream(stream):
                    graph.replay()
        torch.cuda.synchronize()
        for pool, s, app, d, stream in steps:
            want_q, _ = expect_append(pool, app)
            assert torch.equal(s["dq"].cpu(), want_q)
            # a table holds the first request's blocks only as far as it was allocated
            have = [min(n, m) if n > 0 else n for n, m in zip(lens, [48, 48, 112, 0])]
            if have == lens:
                check_attend(pool, dict(s, q=want_q, lens=lens, prefix=prefix), "bf16")
    tc.tc_device_status()


def test_a_request_written_published_hydrated_and_answered_from():
    """append (quantised) -> the existing pack and unpack plans carry codes and scales to another pool -> gather reads
    them back and attention answers from them, the same as from the first pool."""
    rng = np.random.default_rng(41)
    B, H, D, Hq, lens, prefix = 16, 8, 128, 32, [37, 100, 5, 200], 64
    for kind in ("e4m3", "int8", "bf16"):
        a, z = (Pool(kind, blocks=64, B=B, H=H, D=D, layer=0, layout=lay) for lay in ("nhd", "hnd"))
        src, dst = (tables_for(lens + [prefix], p, np.random.default_rng(i)) for i, p in enumerate((a, z)))
        n = sum(lens) + prefix
        app = append_case(a, n, Hq, "bf16", D, False, rng, positions=256)
        seq = [(r, t) for r, m in enumerate(lens + [prefix]) for t in range(m)]
        app["slots"] = np.array([src[r, t // B] * B + t % B for r, t in seq], dtype=np.int64)
        run_append(a, app)
        T = lens + [prefix]
        off = np.concatenate([[0], np.cumsum([-(-t // B) for t in T])])
        flat = lambda tab: np.concatenate([tab[r, : -(-t // B)] for r, t in enumerate(T)])
        e = TORCH[kind].itemsize
        moves = [(D, e, a.raw, z.raw, a.plane, z.plane)] + ([(1, 4, a.scales, z.scales, 64 * B * H * 4, 64 * B * H * 4)] if e == 1 else [])
        for width, size, x, y, px, py in moves:
            shape = (1, B, H, width, size)
            pack = tc.tc_plan_create(tc.kv_spec(tc.TC_KV_PACK, shape, src_pool=tc.pool(tc.TC_NHD, 64, 1, plane_stride=px), packed_layout=tc.TC_HND, T=T, bt_off=off, bt_src=flat(src)))
            unpack = tc.tc_plan_create(tc.kv_spec(tc.TC_KV_UNPACK, shape, dst_pool=tc.pool(tc.TC_HND, 64, 1, plane_stride=py), packed_layout=tc.TC_HND, T=T, bt_off=off, bt_dst=flat(dst)))
            packed = torch.empty(pack.stats().packed_bytes_required, dtype=torch.uint8, device="cuda")
            tc.tc_kv_pack(pack, [x], [packed])
            tc.tc_kv_unpack(unpack, [packed], [y])
            torch.cuda.synchronize()
        outs = []
        for p, tab in ((a, src), (z, dst)):
            k, v = (torch.zeros(n, H, D, dtype=torch.bfloat16, device="cuda") for _ in range(2))
            tc.tc_kv_gather(p.handle, dev(tab), dev(np.concatenate([[0], np.cumsum(T)])), k, v)
            out = torch.zeros(4, Hq, D, dtype=torch.bfloat16, device="cuda")
            q = app["q_out"][:4].contiguous()
            ws = torch.empty(tc.tc_attn_workspace_bytes(p.handle, q, max_len=200, max_prefix=prefix), dtype=torch.uint8, device="cuda")
            tc.tc_attn_decode(p.handle, q, out, dev(tab[:4]), dev(np.array(lens, dtype=np.int32)), max_len=200, workspace=ws, prefix_table=dev(tab[4]), prefix_len=dev(np.array([prefix], dtype=np.int32)), max_prefix=prefix)
            outs.append((k, v, out))
        for x, y in zip(*outs):
            assert torch.equal(x, y)
        want_q, rows = expect_append(a, app)
        for c in (0, 1):
            stored, scale = rows[c]
            x = orc.values(stored.numpy().view(np.uint8 if kind == "e4m3" else np.int8), scale.numpy(), kind) if scale is not None else np64(stored.view(torch.bfloat16))
            assert torch.equal(outs[0][c].cpu(), torch.from_numpy(x.astype(np.float32)).bfloat16())
    status_is(0)


FIRST_CALL = """
import sys
sys.path[:0] = [{root!r}, {tests!r}]
import numpy as np, torch
from test_operators_gpu import *
rng = np.random.default_rng(0)
for kind in ("bf16", "e4m3"):
    pool = Pool(kind, blocks=80)
    s = attend_case(pool, [40, 33], 200, 32, "bf16", rng, poison=False)
    app = append_case(pool, 2, 32, "bf16", 64, False, rng)
    free = np.setdiff1d(np.arange(80), np.concatenate([s["table"].ravel(), s["shared"]]))
    app["slots"] = free[:2].astype(np.int64) * 16
    k, v = (torch.zeros(73, 2, 128, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    d = [dev(x) for x in (app["slots"], app["pos"], app["cos"], app["sin"], np.array([0, 40, 73]))]
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        stream = torch.cuda.current_stream()
        tc.tc_kv_append(pool.handle, app["k"], app["v"], d[0], q=app["q"], q_out=s["dq"], positions=d[1], cos=d[2], sin=d[3], stream=stream)
        tc.tc_kv_gather(pool.handle, s["d"]["tables"], d[4], k, v, stream=stream)
        run_attend(pool, s, stream=stream)
    graph.replay()
    torch.cuda.synchronize()
    want_q, _ = expect_append(pool, app)
    assert torch.equal(s["dq"].cpu(), want_q)
    check_attend(pool, dict(s, q=want_q), "bf16")
    want = np.concatenate([tokens_of(s["values"][0], s["table"][r], 0, n, 16) for r, n in enumerate([40, 33])])
    assert torch.equal(k.cpu(), torch.from_numpy(want.astype(np.float32)).bfloat16())
print("captured")
"""


def test_the_first_call_of_a_process_may_be_a_captured_one():
    import os
    import subprocess
    import sys
    here = os.path.dirname(os.path.abspath(__file__))
    code = FIRST_CALL.format(root=os.path.dirname(here), tests=here)
    got = subprocess.run([sys.executable, "-c", code], capture_output=True, text=True, timeout=300)
    assert got.returncode == 0 and "captured" in got.stdout, got.stderr[-2000:]


def test_pinned_host_memory_serves_and_pageable_memory_is_refused():
    pool = Pool("bf16", blocks=4)
    values = pool.fill(np.random.default_rng(51))
    k = torch.zeros(20, 2, 128, dtype=torch.bfloat16).pin_memory()
    v = torch.zeros(20, 2, 128, dtype=torch.bfloat16).pin_memory()
    table, off = dev(np.array([[2, 0]], dtype=np.int32)), dev(np.array([0, 20]))
    tc.tc_kv_gather(pool.handle, table, off, k, v)
    torch.cuda.synchronize()
    assert np.array_equal(np64(k), tokens_of(values[0], np.array([2, 0]), 0, 20, 16))
    with pytest.raises(tc.TensorCastError, match="pageable"):
        tc.tc_kv_gather(pool.handle, table, off, torch.zeros(20, 2, 128, dtype=torch.bfloat16), v)
    with pytest.raises(tc.TensorCastError, match="pageable"):
        tc.tc_kv_append(pool.handle, k, v, torch.zeros(20, dtype=torch.int64))
    q = torch.zeros(1, 2, 128, dtype=torch.bfloat16, device="cuda")
    with pytest.raises(tc.TensorCastError, match="pageable"):
        tc.tc_attn_decode(pool.handle, q, torch.zeros_like(q), table, torch.ones(1, dtype=torch.int32), max_len=20, workspace=torch.empty(1 << 20, dtype=torch.uint8, device="cuda"))
