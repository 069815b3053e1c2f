"""The operators on a paged layer without a GPU: what they refuse, the sizes of their workspace, the kernels' index
arithmetic, and the oracle that the GPU tests compare with."""
import ctypes as C
import os
import subprocess

import numpy as np
import pytest
import torch

import paper_2608_06007_b200 as tc
from oracle import operators as orc
from paper_2608_06007_b200 import binding as b

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
INVALID, SHAPE, BOUNDS, OVERLAP, TOO_LARGE = -1, -2, -3, -4, -9
BASE = 1 << 20  # a made-up, aligned address: nothing below reaches a device


def layer(B=16, H=8, D=128, dtype=tc.TC_BF16, layout=tc.TC_NHD, blocks=10, block_stride=0, base=BASE, **changes):
    pool = tc.pool(layout, blocks, 1, plane_stride=1 << 24, block_stride=block_stride)
    scales = dict(scale_pool=tc.pool(layout, blocks, 1, plane_stride=1 << 16), scale_bases=[2 * BASE]) if dtype in (tc.TC_E4M3, tc.TC_INT8) else {}
    made = tc.kv_layer(pool, (B, H, D), dtype, [base], **scales)
    for name, value in changes.items():
        setattr(made.struct, name, value)
    return made


def call(name, made, args):
    lib = tc.load_library()
    return getattr(lib, name)(made.ref if made is not None else None, C.byref(args) if args is not None else None, None), lib.tc_last_error().decode()


def append_args(n=4, Hq=8, H=8, D=128, e=2, **changes):
    a = b.tc_kv_append_t(C.sizeof(b.tc_kv_append_t), 0, n, Hq, tc.TC_BF16, D)
    for i, name in enumerate(("q", "q_out", "k", "v")):
        setattr(a, name, BASE * (4 + i))
        setattr(a, name + "_stride", (C.c_int64 * 2)((Hq if "q" in name else H) * D * e, D * e))
    a.slots, a.positions, a.cos, a.sin, a.n_positions = 3 * BASE, 3 * BASE + 4096, BASE * 9, BASE * 10, 100
    for name, value in changes.items():
        setattr(a, name, (C.c_int64 * 2)(*value) if name.endswith("_stride") and isinstance(value, tuple) else value)
    return a


def gather_args(R=2, n=5, H=8, D=128, e=2, **changes):
    a = b.tc_kv_gather_t(C.sizeof(b.tc_kv_gather_t), tc.TC_BF16, R, n, 3 * BASE, 4, 16, 4 * BASE, None, 5 * BASE, 6 * BASE)
    a.k_stride = a.v_stride = (C.c_int64 * 2)(H * D * e, D * e)
    for name, value in changes.items():
        setattr(a, name, (C.c_int64 * 2)(*value) if isinstance(value, tuple) else value)
    return a


def decode_args(R=3, Hq=32, D=128, **changes):
    row = D * 2
    a = b.tc_attn_decode_t(C.sizeof(b.tc_attn_decode_t), tc.TC_BF16, R, Hq, 3 * BASE, 4 * BASE, (C.c_int64 * 2)(Hq * row, row), (C.c_int64 * 2)(Hq * row, row), 5 * BASE, 0.0, 0,
                           6 * BASE, 4, 16, 7 * BASE, 64, 8 * BASE, 9 * BASE, 100, 10 * BASE, 1 << 40)
    for name, value in changes.items():
        setattr(a, name, (C.c_int64 * 2)(*value) if isinstance(value, tuple) else value)
    return a


LAYERS = [
    (dict(struct_size=8), INVALID), (dict(dtype=9), INVALID), (dict(dtype=0), INVALID), (dict(B=0), SHAPE), (dict(H=-1), SHAPE), (dict(D=0), SHAPE), (dict(D=1 << 30), SHAPE),
    (dict(k=None), INVALID), (dict(v=None), INVALID), (dict(k_scale=64), INVALID), (dict(k=BASE + 1), INVALID), (dict(B=1 << 22), TOO_LARGE),
]


@pytest.mark.parametrize("op,args", [("tc_kv_append", append_args()), ("tc_kv_gather", gather_args()), ("tc_attn_decode", decode_args())], ids=["append", "gather", "decode"])
def test_a_layer_that_makes_no_sense_is_refused_by_every_operator(op, args):
    for changes, status in LAYERS:
        rc, why = call(op, layer(**changes), args)
        assert rc == status and why, (changes, rc, why)
    assert call(op, None, args)[0] == INVALID
    assert call(op, layer(), None)[0] == INVALID
    for made, status in ((layer(block_stride=16 * 8 * 128 * 2 - 16), OVERLAP), (layer(blocks=-1), SHAPE), (layer(layout=2), INVALID), (layer(block_stride=1 << 60), TOO_LARGE)):
        assert call(op, made, args)[0] == status
    quantised = layer(dtype=tc.TC_E4M3)
    quantised.struct.v_scale = None
    assert call(op, quantised, args)[0] == INVALID
    quantised = layer(dtype=tc.TC_INT8)
    quantised.struct.scale_pool.num_blocks = 9
    assert call(op, quantised, args)[0] == BOUNDS
    quantised = layer(dtype=tc.TC_INT8)
    quantised.struct.k_scale += 2
    assert call(op, quantised, args)[0] == INVALID


@pytest.mark.parametrize("changes,status", [
    (dict(struct_size=8), INVALID), (dict(flags=2), INVALID), (dict(dtype=tc.TC_E4M3), INVALID), (dict(n_tokens=-1), SHAPE), (dict(rot_dim=3), SHAPE), (dict(rot_dim=130), SHAPE),
    (dict(rot_dim=-2), SHAPE), (dict(q=None), INVALID), (dict(q_out=None), INVALID), (dict(Hq=0), SHAPE), (dict(k=None), INVALID), (dict(v=None), INVALID), (dict(k=BASE + 1), INVALID),
    (dict(k_stride=(-256, 256)), SHAPE), (dict(k_stride=(2047, 256)), INVALID), (dict(q_out_stride=(1024, 256)), OVERLAP), (dict(q_out_stride=(2048, 128)), OVERLAP),
    (dict(q_out_stride=(0, 256)), OVERLAP), (dict(slots=None), INVALID), (dict(slots=3 * BASE + 4), INVALID), (dict(positions=None), INVALID), (dict(cos=None), INVALID),
    (dict(sin=BASE + 2), INVALID), (dict(n_positions=0), SHAPE), (dict(table_stride=128), SHAPE), (dict(table_stride=258), INVALID),
    (dict(q_out=BASE * 4, q_out_stride=(4096, 256)), OVERLAP),
])
def test_append_refuses(changes, status):
    rc, why = call("tc_kv_append", layer(), append_args(**changes))
    assert rc == status and why, (rc, why)


def test_append_refuses_rows_that_are_too_long():
    assert call("tc_kv_append", layer(D=528), append_args(D=528))[0] == TOO_LARGE


@pytest.mark.parametrize("changes,status", [
    (dict(struct_size=8), INVALID), (dict(dtype=tc.TC_INT8), INVALID), (dict(R=-1), SHAPE), (dict(n_rows=-1), SHAPE), (dict(k_out=None, v_out=None), INVALID), (dict(tables=None), INVALID),
    (dict(tables=3 * BASE + 2), INVALID), (dict(table_stride=6), INVALID), (dict(table_stride=-4), INVALID), (dict(table_width=0), SHAPE), (dict(offsets=None), INVALID),
    (dict(offsets=BASE + 4), INVALID), (dict(first=BASE + 4), INVALID), (dict(k_stride=(2048, 128)), OVERLAP), (dict(v_stride=(256, 256)), OVERLAP), (dict(v_out=BASE + 1), INVALID),
])
def test_gather_refuses(changes, status):
    rc, why = call("tc_kv_gather", layer(), gather_args(**changes))
    assert rc == status and why, (rc, why)


@pytest.mark.parametrize("changes,status", [
    (dict(struct_size=8), INVALID), (dict(dtype=tc.TC_FP32), INVALID), (dict(dtype=tc.TC_FP16), INVALID), (dict(R=-1), SHAPE), (dict(Hq=12), SHAPE), (dict(Hq=0), SHAPE), (dict(R=1 << 20, Hq=1 << 16), TOO_LARGE),
    (dict(max_len=-1), SHAPE), (dict(max_prefix=1 << 31), SHAPE), (dict(scale=float("nan")), INVALID), (dict(scale=float("inf")), INVALID), (dict(scale=-2e30), INVALID), (dict(q=None), INVALID), (dict(out=None), INVALID),
    (dict(out=3 * BASE), OVERLAP), (dict(q=3 * BASE + 8), INVALID), (dict(out_stride=(8192, 128)), OVERLAP), (dict(lse=BASE + 2), INVALID), (dict(lens=None), INVALID), (dict(tables=None), INVALID),
    (dict(table_stride=2), INVALID), (dict(table_width=3), BOUNDS), (dict(prefix_table=None), INVALID), (dict(prefix_len=None), INVALID), (dict(workspace=None), INVALID),
    (dict(workspace=BASE + 8), INVALID), (dict(workspace_bytes=100), BOUNDS),
])
def test_decode_refuses(changes, status):
    rc, why = call("tc_attn_decode", layer(), decode_args(**changes))
    assert rc == status and why, (rc, why)


def test_decode_refuses_head_dims_and_alignments_that_it_has_no_kernel_for():
    for D in (8, 72, 272):
        assert call("tc_attn_decode", layer(D=D), decode_args(D=D))[0] == SHAPE
    assert call("tc_attn_decode", layer(base=BASE + 8), decode_args())[0] == INVALID
    assert call("tc_attn_decode", layer(block_stride=16 * 8 * 128 * 2 + 8), decode_args())[0] == INVALID


def test_a_call_for_nothing_returns_before_it_needs_a_device():
    assert call("tc_kv_append", layer(), append_args(n=0, k=None, slots=None))[0] == 0
    assert call("tc_kv_gather", layer(), gather_args(R=0))[0] == 0
    assert call("tc_kv_gather", layer(), gather_args(n=0, k_out=None, v_out=None))[0] == 0
    assert call("tc_attn_decode", layer(), decode_args(R=0))[0] == 0


@pytest.mark.skipif(torch.cuda.is_available(), reason="asks for the error without a device")
def test_without_a_device_a_good_call_says_so():
    for op, args in (("tc_kv_append", append_args()), ("tc_kv_gather", gather_args()), ("tc_attn_decode", decode_args())):
        rc, why = call(op, layer(), args)
        assert rc == b.TC_ERR_CUDA and why


def test_the_workspace_depends_on_the_sizes_alone_and_stays_small():
    lib, out = tc.load_library(), C.c_int64()
    for R, Hq, H, max_len, max_prefix in ((1, 8, 8, 0, 0), (1, 32, 8, 131072, 0), (512, 32, 8, 1024, 4000), (4096, 64, 8, 32768, 131072), (1, 128, 1, 1, 1), (7, 28, 4, 0, 100)):
        assert lib.tc_attn_workspace(layer(H=H).ref, C.byref(decode_args(R=R, Hq=Hq, max_len=max_len, max_prefix=max_prefix)), C.byref(out)) == 0
        one = R * Hq * 129 * 4  # the outputs and sums of one part
        assert (out.value == 0) == (max_len == max_prefix == 0)
        assert out.value >= one * ((max_len > 0) + (max_prefix > 0))
        assert out.value <= 2 * max(256 << 20, 2 * one) + 4096
    assert lib.tc_attn_workspace(layer().ref, C.byref(decode_args()), None) == INVALID


def test_binding_checks_what_the_library_cannot_see():
    made = layer()
    k = torch.zeros(3, 8, 128, dtype=torch.bfloat16)
    slots = torch.zeros(3, dtype=torch.int64)
    for bad in (dict(k=k[:, :4]), dict(v=k.half()), dict(slots=slots[:2]), dict(slots=slots.int()), dict(k=k.transpose(1, 2).contiguous().transpose(1, 2)), dict(q=k), dict(q=k, q_out=k.half()),
                dict(cos=torch.zeros(4, 64), sin=torch.zeros(4, 32)), dict(k=k.to(torch.int16), v=k.to(torch.int16))):
        args = dict(k=k, v=k, slots=slots) | bad
        with pytest.raises(ValueError):
            tc.tc_kv_append(made, **args)
    tables, offsets = torch.zeros(2, 3, dtype=torch.int32), torch.zeros(3, dtype=torch.int64)
    for bad in (dict(tables=tables.long()), dict(tables=tables[:1]), dict(offsets=offsets.int()), dict(k_out=k[:, :, :64]), dict(v_out=k.float()), dict(first=offsets[:1])):
        with pytest.raises(ValueError):
            tc.tc_kv_gather(made, **(dict(tables=tables, offsets=offsets, k_out=k, v_out=k) | bad))
    q, lens, ws = torch.zeros(2, 16, 128, dtype=torch.bfloat16), torch.zeros(2, dtype=torch.int32), torch.zeros(64, dtype=torch.uint8)
    for bad in (dict(out=q.half()), dict(out=q[:1]), dict(lens=lens.long()), dict(lens=lens[:1]), dict(lse=torch.zeros(2, 8)), dict(prefix_table=lens[:0], max_prefix=5, prefix_len=lens), dict(q=q.float())):
        with pytest.raises(ValueError):
            tc.tc_attn_decode(made, **(dict(q=q, out=q.clone(), tables=tables, lens=lens, max_len=16, workspace=ws) | bad))
    with pytest.raises(ValueError):
        tc.kv_layer(tc.pool(tc.TC_NHD, 4, 4), (16, 8, 128), tc.TC_BF16, [BASE, BASE], layer=0)
    with pytest.raises(ValueError):
        tc.kv_layer(tc.pool(tc.TC_NHD, 4, 2), (16, 8, 128), tc.TC_BF16, [BASE, BASE], layer=1)


def test_layer_planes_follow_the_pool_formula():
    one = tc.kv_layer(tc.pool(tc.TC_NHD, 4, 1, plane_stride=4096), (2, 2, 2), tc.TC_BF16, [BASE], layer=3)
    assert (one.struct.k, one.struct.v) == (BASE + 6 * 4096, BASE + 7 * 4096)
    many = tc.kv_layer(tc.pool(tc.TC_NHD, 4, 4), (2, 2, 2), tc.TC_BF16, [BASE, 2 * BASE, 3 * BASE, 4 * BASE], layer=1)
    assert (many.struct.k, many.struct.v) == (3 * BASE, 4 * BASE)


INDEX_CHECK = r"""
#include <stdio.h>
#include <vector>
#include "kv_index.h"
using namespace tc;
int main() {
    // every token, head and byte offset of both layouts, in 64 bits
    for (int B : {1, 3, 16}) for (int H : {1, 5}) for (int row : {2, 160}) for (int hnd : {0, 1}) {
        PlaneGeo g{(int64_t)B * H * row + 32, hnd ? row : H * row, hnd ? B * row : row};
        for (long b : {0l, 7l, 2000000000l}) for (int n = 0; n < B; n++) for (int h = 0; h < H; h++) {
            __int128 want = (__int128)b * (B * H * row + 32) + (hnd ? ((__int128)h * B + n) * row : ((__int128)n * H + h) * row);
            if (g.at(b, n, h) != (int64_t)want) return printf("at\n"), 1;
        }
        for (uint32_t t : {0u, 1u, 15u, 16u, 2147483647u}) {
            uint32_t e, n;
            token_place(t, B, &e, &n);
            if ((uint64_t)e * B + n != t || n >= (uint32_t)B) return printf("token\n"), 1;
        }
        // slots: outside is refused on both sides, past 32 bits too
        for (int64_t blocks : {(int64_t)0, (int64_t)4, (int64_t)2147483647}) for (int64_t s : {(int64_t)-1, INT64_MIN, (int64_t)0, blocks * B - 1, blocks * B, (int64_t)1 << 40, INT64_MAX}) {
            int64_t b; int32_t n;
            bool in = slot_place(s, B, blocks, &b, &n);
            if (in != (s >= 0 && s < blocks * B)) return printf("slot %lld of %lld\n", (long long)s, (long long)blocks), 1;
            if (in && (b * B + n != s || n < 0 || n >= B)) return printf("place\n"), 1;
        }
    }
    // offsets that are in order, have empty requests, or make no sense: never outside [0, R]
    std::vector<std::vector<int64_t>> all = {{0, 3, 3, 7}, {0, 0, 0, 0}, {5, 9, 9, 12}, {0, 100, 2, 50}, {9, 3, 1, 10}};
    for (auto &o : all) for (int64_t row = -2; row < 60; row++) {
        int64_t r = request_of(o.data(), 3, row);
        bool inside = row >= o[0] && row < o[3];
        if (inside != (r >= 0) || r >= 3) return printf("request\n"), 1;
        bool ordered = o[0] <= o[1] && o[1] <= o[2] && o[2] <= o[3];
        if (r >= 0 && ordered && !(o[r] <= row && row < o[r + 1])) return printf("wrong request\n"), 1;
    }
    if (request_of(nullptr, 0, 0) != -1) return 1;
    printf("ok\n");
    return 0;
}
"""


def test_the_kernels_index_arithmetic_compiled_for_the_host(tmp_path):
    src, exe = tmp_path / "index.cpp", tmp_path / "index"
    src.write_text(INDEX_CHECK)
    subprocess.check_call(["g++", "-std=c++17", "-O1", "-fsanitize=undefined,address", "-fno-sanitize-recover", "-I", os.path.join(ROOT, "paper_2608_06007_b200", "csrc"), str(src), "-o", str(exe)])
    assert subprocess.check_output([str(exe)], text=True) == "ok\n"


# ------------------------------------------------------------------------------------ the oracle
def test_oracle_e4m3_agrees_with_torch():
    codes = np.arange(256, dtype=np.uint8)
    want = torch.from_numpy(codes.copy()).view(torch.float8_e4m3fn).double().numpy()
    assert np.array_equal(orc.e4m3_values(), want, equal_nan=True)
    x = np.concatenate([np.random.default_rng(0).standard_normal(20000) * 100, want[~np.isnan(want)], (want[:126] + want[1:127]) / 2, [0.0, -0.0, 448.0, 2.0 ** -10, 3 * 2.0 ** -11]]).astype(np.float32)
    x = np.clip(x, -448, 448)
    assert np.array_equal(orc.e4m3_round(x), torch.from_numpy(x).to(torch.float8_e4m3fn).view(torch.uint8).numpy())


def test_oracle_rotation_keeps_lengths_and_depends_on_distances_alone():
    rng = np.random.default_rng(1)
    q, k = rng.standard_normal((2, 1, 1, 16))
    freq = 100.0 ** (-np.arange(6) / 6)
    for interleaved in (False, True):
        at = lambda x, pos: orc.rotate(x, np.cos(pos * freq)[None], np.sin(pos * freq)[None], interleaved)
        assert np.allclose(np.linalg.norm(at(q, 12.0)), np.linalg.norm(q))
        assert np.allclose((at(q, 12.0) * at(k, 5.0)).sum(), (at(q, 107.0) * at(k, 100.0)).sum())
        assert np.array_equal(at(q, 3.0)[..., 12:], q[..., 12:])


@pytest.mark.parametrize("kind,half", [("e4m3", 2.0 ** -4), ("int8", None)])
def test_oracle_quantisation_is_within_half_a_step(kind, half):
    y = np.random.default_rng(2).standard_normal((50, 3, 40)).astype(np.float32)
    y[0, 0] = 0
    y[1, 0] = 1e-40
    codes, scale = orc.quantise(y, kind)
    v = orc.values(codes, scale, kind)
    assert not codes[0, 0].any() and scale[0, 0] == 0 and scale[1, 0] == 0
    step = np.abs(y) * half + scale[..., None] * 2.0 ** -10 if half else np.broadcast_to(scale[..., None] * 0.5, y.shape)
    assert (np.abs(v - y)[2:] <= (step * (1 + 1e-6))[2:]).all()
    y[2, 1, 5], y[3, 1, 5] = np.nan, np.inf
    codes, scale = orc.quantise(y, kind)
    assert np.isnan(scale[2, 1]) and np.isnan(scale[3, 1]) and not codes[2, 1].any() and np.isfinite(scale[2, 0])


def test_oracle_attention_of_one_key_and_of_none():
    rng = np.random.default_rng(3)
    q, k, v = rng.standard_normal((4, 8)), rng.standard_normal((1, 2, 8)), rng.standard_normal((1, 2, 8))
    out, lse, _ = orc.attend(q, k, v, 0.5)
    assert np.allclose(out, np.repeat(v[0], 2, axis=0)) and np.allclose(lse, (q * np.repeat(k[0], 2, axis=0)).sum(-1) * 0.5)
    out, lse, _ = orc.attend(q, k[:0], v[:0], 0.5)
    assert not out.any() and (lse == -np.inf).all()
