"""The paged-cache operators as they are measured: appending tokens to a pool, gathering pages out of
one, and decoding against one with a prefix that the batch shares.

`run` computes them in elementary torch operations, or, where `own` is true, calls the library.
Lengths come from the case alone, contents and block tables from the seed.
"""
import math

import numpy as np
import torch

own = False

_TORCH = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32, "e4m3": torch.float8_e4m3fn, "int8": torch.int8}
_BYTES = {"bf16": 2, "fp16": 2, "fp32": 4, "e4m3": 1, "int8": 1}
_TOP = {"e4m3": 448.0, "int8": 127.0}
_TINY = 2.0 ** -126


# ---------------------------------------------------------------------------------------- cases
def listed():
    """Shapes: 32 query and 8 KV heads of 128, blocks of 16 (the 8B model's cache); 64 and 8, blocks of 32
    (the 70B model's); generic others."""
    append = dict(op="append", hq=32, hkv=8, d=128, rot=128, interleaved=False, block=16, layout="nhd", x="bf16", pool="bf16", padded=0)
    gather = dict(op="gather", hkv=8, d=128, block=16, layout="nhd", pool="e4m3", out="bf16")
    attend = dict(op="attend", hq=32, hkv=8, d=128, block=16, layout="nhd", x="bf16", pool="bf16", padded=0)
    return [
        # one decode step of a few requests: latency
        dict(append, name="append 37 tokens", n=37),
        # one decode step of the agent burst's 512 sessions, the batch padded up for a captured graph
        dict(append, name="append 512 sessions e4m3", n=512, padded=12, pool="e4m3", layout="hnd"),
        # an odd chunk of a prompt: part of the head rotated, adjacent pairs, blocks of 20
        dict(append, name="append 5003 tokens int8", n=5003, hq=16, hkv=2, d=80, rot=32, interleaved=True, block=20, x="fp16", pool="int8"),
        # the prompts of a long prefill at once
        dict(append, name="append 32768 tokens e4m3", n=32768, hq=64, block=32, pool="e4m3"),
        # reading the correctness workload's four requests back
        dict(gather, name="gather 4 requests e4m3", lengths="37,100,5,200"),
        # the agent burst's prefixes, 1 to 64 blocks each
        dict(gather, name="gather 512 prefixes e4m3", lengths="geometric", r=512, lo=16, hi=1024, mean=192),
        # long contexts of the 70B model
        dict(gather, name="gather 40 contexts int8", lengths="uniform", r=40, lo=512, hi=8192, block=32, layout="hnd", pool="int8", out="fp16"),
        # a few short requests: latency
        dict(attend, name="attend 4 requests", lengths="37,100,5,200", prefix=48),
        # a serving batch behind one system prompt
        dict(attend, name="attend 64 behind 8192", lengths="lognormal", r=64, lo=1, hi=2048, mean=256, prefix=8192),
        # the agent burst's sessions behind a common preamble, on a quantised cache; some rows are padding
        dict(attend, name="attend 512 behind 4000 e4m3", lengths="geometric", r=512, lo=1, hi=1024, mean=192, prefix=4000, pool="e4m3", layout="hnd", padded=7),
        # many short questions about one long document
        dict(attend, name="attend 128 behind 32768", lengths="uniform", r=128, lo=1, hi=64, prefix=32768, hq=64, block=32, x="fp16", pool="fp16"),
        # a few very long contexts that share nothing
        dict(attend, name="attend 3 long int8", lengths="65536,99991,131072", prefix=0, hq=28, hkv=4, pool="int8"),
    ]


def draw(rng):
    """A case of the same ranges."""
    def spread(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))

    op = rng.choice(["append", "gather", "attend", "attend"])
    hkv = rng.choice([1, 2, 3, 4, 8])
    case = dict(op=op, hkv=hkv, block=rng.choice([1, 8, 16, 20, 32, 64]), layout=rng.choice(["nhd", "hnd"]), draw=rng.randrange(1 << 30))
    if op == "append":
        d = rng.choice([64, 80, 100, 128, 192, 256])
        case.update(hq=hkv * rng.choice([1, 2, 4, 5, 7, 8]), d=d, rot=rng.choice([0, 32, 64, d // 4 * 2, d]), interleaved=rng.random() < 0.5,
                    x=rng.choice(["bf16", "fp16", "fp32"]), pool=rng.choice(["bf16", "fp16", "fp32", "e4m3", "int8"]))
        case["n"] = min(spread(1, 32768), 320_000_000 // ((case["hq"] + hkv) * d * 2))
        case["padded"] = rng.choice([0, rng.randint(0, case["n"] - 1)])
        return case
    case["pool"] = rng.choice(["bf16", "fp16", "e4m3", "int8"])
    kind = rng.choice(["geometric", "lognormal", "uniform"])
    if op == "gather":
        r = spread(1, 512)
        mean = spread(1, max(1, 100_000_000 // (r * hkv * 256)) if r * hkv * 256 < 100_000_000 else 1)
        case.update(d=rng.choice([64, 80, 100, 128, 192, 256]), out=rng.choice(["bf16", "fp16", "fp32"]), lengths=kind, r=r, lo=rng.choice([0, 1]), hi=2 * min(mean, 16384), mean=min(mean, 16384))
        return case
    d, g, r = rng.choice([64, 80, 96, 128, 128, 256]), rng.choice([1, 2, 4, 5, 7, 8, 12]), spread(1, 512)
    x = rng.choice(["bf16", "fp16"])
    if case["pool"] in ("bf16", "fp16"):
        case["pool"] = x
    mean = min(spread(1, 2048), 1 + 64_000_000 // (r * hkv * d))
    prefix = rng.choice([0, spread(1, 32768), spread(1, 32768)])
    case.update(hq=hkv * g, d=d, x=x, lengths=kind, r=r, lo=rng.choice([0, 1]), hi=2 * mean, mean=mean, prefix=min(prefix, 60_000_000_000 // (4 * r * hkv * g * d)), padded=rng.choice([0, rng.randint(0, r - 1)]))
    return case


def _lengths(case):
    if case["lengths"][0].isdigit():
        return np.array([int(v) for v in case["lengths"].split(",")], dtype=np.int64)
    rng, r = np.random.default_rng([26, case["r"], case["hi"], case.get("draw", 0)]), case["r"]
    if case["lengths"] == "geometric":
        v = rng.geometric(1.0 / max(1.0, case["mean"] / 16), r) * 16 - rng.integers(0, 16, r)
    elif case["lengths"] == "lognormal":
        v = np.rint(np.exp(math.log(case["mean"]) + rng.standard_normal(r)))
    else:
        v = rng.integers(case["lo"], case["hi"] + 1, r)
    v = np.clip(v, case["lo"], case["hi"]).astype(np.int64)
    v[0] = max(v[0], 1)
    return v


# --------------------------------------------------------------------------------------- inputs
def _normal(gen, shape, kind, chunk=1 << 28):
    t = torch.empty(shape, dtype=_TORCH[kind], device="cuda")
    flat = t.view(-1)
    for a in range(0, flat.numel(), chunk):
        b = min(flat.numel(), a + chunk)
        flat[a:b] = torch.randn(b - a, generator=gen, device="cuda")
    return t


def _pool(case, blocks, gen):
    """K and V planes of a filled pool, [2, blocks, block, heads, d] or [2, blocks, heads, block, d], and its scales."""
    inner = (case["block"], case["hkv"]) if case["layout"] == "nhd" else (case["hkv"], case["block"])
    shape = (2, blocks, *inner, case["d"])
    kind = case["pool"]
    if kind not in _TOP:
        return _normal(gen, shape, kind), None
    # codes of normal values whose row maximum sits near the top of the range, as a quantised row's does
    codes = torch.empty(shape, dtype=_TORCH[kind], device="cuda")
    flat = codes.view(-1)
    for a in range(0, flat.numel(), 1 << 28):
        b = min(flat.numel(), a + (1 << 28))
        v = (torch.randn(b - a, generator=gen, device="cuda") * (_TOP[kind] / 3)).clamp_(-_TOP[kind], _TOP[kind])
        flat[a:b] = (v if kind == "e4m3" else v.round_()).to(codes.dtype)
    scales = (0.5 + torch.rand(shape[:-1], generator=gen, device="cuda")) * (3 / _TOP[kind])
    return codes, scales


def _tables(lengths, block, blocks, rng):
    """A block table a request, padded with an id that is never to be read, over a seeded permutation of the pool."""
    need = (lengths + block - 1) // block
    free = rng.permutation(blocks)[: int(need.sum())].astype(np.int32)
    table = np.full((len(lengths), max(1, int(need.max(initial=0)))), -1, dtype=np.int32)
    table[np.arange(table.shape[1])[None, :] < need[:, None]] = free
    return table


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    rng = np.random.default_rng(seed)
    s = dict(case=case)
    block, hkv, d = case["block"], case["hkv"], case["d"]
    if case["op"] == "append":
        n, hq, rot = case["n"], case["hq"], case["rot"]
        blocks = -(-n * 5 // (4 * block)) + 1
        # q, k and v are the slices of one projection's output
        qkv = _normal(gen, (n, hq + 2 * hkv, d), case["x"])
        s["q"], s["k"], s["v"] = qkv[:, :hq], qkv[:, hq : hq + hkv], qkv[:, hq + hkv :]
        s["q_out"] = torch.zeros((n, hq, d), dtype=qkv.dtype, device="cuda")
        slots = rng.permutation(blocks * block)[:n].astype(np.int64)
        slots[n - case["padded"] :] = -1
        s["slots"] = torch.from_numpy(slots).cuda()
        positions = 131072 if n > 1024 else 16384
        s["positions"] = torch.from_numpy(rng.integers(0, positions, n)).cuda()
        # by wavelength: far ones stretched eightfold, near ones kept, a ramp between
        i = torch.arange(rot // 2, dtype=torch.float64, device="cuda")
        freq = 500000.0 ** (-2 * i / max(1, rot))
        keep = ((8192 * freq / (2 * math.pi) - 1) / 3).clamp(0, 1)
        angle = torch.arange(positions, dtype=torch.float64, device="cuda")[:, None] * (freq * keep + freq / 8 * (1 - keep))
        s["cos"], s["sin"] = angle.cos().float(), angle.sin().float()
        inner = (block, hkv) if case["layout"] == "nhd" else (hkv, block)
        # one block more than the pool has: the plain form drops padded tokens there
        s["pool"] = torch.zeros((2, blocks + 1, *inner, d), dtype=_TORCH[case["pool"]], device="cuda")
        s["scales"] = torch.zeros((2, blocks + 1, *inner), device="cuda") if case["pool"] in _TOP else None
        s["blocks"] = blocks
        s["top"] = torch.tensor(_TOP.get(case["pool"], 1.0), device="cuda")
        return s
    lengths = _lengths(case)
    prefix = case.get("prefix", 0)
    own_blocks, shared = int(((lengths + block - 1) // block).sum()), -(-prefix // block)
    blocks = (own_blocks + shared) * 9 // 8 + 1
    s["blocks"], s["lengths"], s["prefix"] = blocks, lengths, prefix
    s["pool"], s["scales"] = _pool(case, blocks, gen)
    table = _tables(np.concatenate([lengths, [prefix]]), block, blocks, rng)
    width = max(1, int(((lengths + block - 1) // block).max(initial=0)))
    s["tables"] = torch.from_numpy(np.ascontiguousarray(table[:-1, :width])).cuda()
    if case["op"] == "gather":
        off = np.concatenate([[0], np.cumsum(lengths)]).astype(np.int64)
        s["offsets"], s["total"] = torch.from_numpy(off).cuda(), int(off[-1])
        s["k_out"] = torch.zeros((s["total"] + 3, hkv, d), dtype=_TORCH[case["out"]], device="cuda")
        s["v_out"] = torch.zeros_like(s["k_out"])
        return s
    s["shared"] = torch.from_numpy(np.ascontiguousarray(table[-1, : max(1, shared)])).cuda()
    s["prefix_len"] = torch.tensor([prefix], dtype=torch.int32, device="cuda")
    marked = lengths.copy()
    marked[len(lengths) - case["padded"] :] = -1
    s["lens"] = torch.from_numpy(marked.astype(np.int32)).cuda()
    s["longest"] = int(max(1, lengths.max(initial=0)))
    s["q"] = _normal(gen, (len(lengths), case["hq"], d), case["x"])
    s["out"] = torch.zeros_like(s["q"])
    s["lse"] = torch.zeros(s["q"].shape[:2], device="cuda")
    return s


# ------------------------------------------------------------------------------- the plain forms
def _rotated(x, cos, sin, rot, interleaved):
    if rot == 0:
        return x
    a, rest = x[..., :rot], x[..., rot:]
    if interleaved:
        lo, hi = a[..., 0::2], a[..., 1::2]
        return torch.cat([torch.stack([lo * cos - hi * sin, hi * cos + lo * sin], -1).flatten(-2), rest], -1)
    lo, hi = a[..., : rot // 2], a[..., rot // 2 :]
    return torch.cat([lo * cos - hi * sin, hi * cos + lo * sin, rest], -1)


def _quantised(x, kind, top):
    most = x.abs().amax(-1)
    scale = most / top
    scale = torch.where(torch.isfinite(most), torch.where(scale < _TINY, 0.0, scale), math.nan)
    y = torch.where((scale > 0)[..., None], x / scale[..., None], 0.0)
    return (y.clamp(-448, 448) if kind == "e4m3" else y.round()).to(_TORCH[kind]), scale


def _put(plane, case, slot, rows):
    b, t = slot // case["block"], slot % case["block"]
    plane = plane.view(torch.uint8) if plane.dtype == torch.float8_e4m3fn else plane
    rows = rows.view(torch.uint8) if rows.dtype == torch.float8_e4m3fn else rows
    if case["layout"] == "nhd":
        plane[b, t] = rows
    else:
        plane[b, :, t] = rows


def _plain_append(s):
    case = s["case"]
    cos, sin = s["cos"][s["positions"]][:, None], s["sin"][s["positions"]][:, None]
    valid = s["slots"] >= 0
    slot = torch.where(valid, s["slots"], s["blocks"] * case["block"])
    q = _rotated(s["q"].float(), cos, sin, case["rot"], case["interleaved"])
    k = _rotated(s["k"].float(), cos, sin, case["rot"], case["interleaved"])
    s["q_out"].copy_(torch.where(valid[:, None, None], q.to(s["q_out"].dtype), s["q_out"]))
    rows = torch.stack([k, s["v"].float()])
    if case["pool"] in _TOP:
        rows, scale = _quantised(rows, case["pool"], s["top"])
        _put(s["scales"][0], case, slot, scale[0])
        _put(s["scales"][1], case, slot, scale[1])
    rows = rows.to(s["pool"].dtype)
    _put(s["pool"][0], case, slot, rows[0])
    _put(s["pool"][1], case, slot, rows[1])


def _pages(s, plane, block, at):
    """Rows (block, at) of a plane as 32-bit numbers, [..., heads, d]."""
    nhd = s["case"]["layout"] == "nhd"
    codes = s["pool"][plane]
    codes = codes.view(torch.uint8) if codes.dtype == torch.float8_e4m3fn else codes
    x = codes[block, at] if nhd else codes[block, :, at]
    x = (x.view(torch.float8_e4m3fn) if x.dtype == torch.uint8 else x).float()
    if s["scales"] is not None:
        x = x * (s["scales"][plane][block, at] if nhd else s["scales"][plane][block, :, at])[..., None]
    return x


def _plain_gather(s):
    size = s["case"]["block"]
    token = torch.arange(s["total"], device="cuda")
    r = torch.searchsorted(s["offsets"], token, right=True) - 1
    t = token - s["offsets"][r]
    block = s["tables"][r, t // size].long()
    s["k_out"][: s["total"]] = _pages(s, 0, block, t % size).to(s["k_out"].dtype)
    s["v_out"][: s["total"]] = _pages(s, 1, block, t % size).to(s["v_out"].dtype)


def _plain_attend(s):
    case = s["case"]
    size, hkv, d = case["block"], case["hkv"], case["d"]
    r, hq = s["q"].shape[:2]
    q = s["q"].float().view(r, hkv, hq // hkv, d) * (1 / math.sqrt(d))
    j = torch.arange(s["prefix"], device="cuda")
    pk, pv = (_pages(s, c, s["shared"][j // size].long(), j % size) for c in (0, 1))  # [p, hkv, d]
    score = torch.matmul(q.permute(1, 0, 2, 3).reshape(hkv, -1, d), pk.permute(1, 2, 0)).view(hkv, r, hq // hkv, s["prefix"]).transpose(0, 1)
    i = torch.arange(s["longest"], device="cuda")
    block = s["tables"][:, (i // size).clamp(max=s["tables"].shape[1] - 1)].clamp(min=0).long()
    seen = i[None, :] < s["lens"][:, None]
    ok, ov = (torch.where(seen[..., None, None], _pages(s, c, block, (i % size).expand_as(block)), 0.0) for c in (0, 1))  # [r, i, hkv, d]
    mine = torch.matmul(q, ok.permute(0, 2, 3, 1))
    score = torch.cat([score, torch.where(seen[:, None, None, :], mine, -math.inf)], -1)
    most = score.amax(-1, keepdim=True)
    e = torch.exp(score - torch.where(most == -math.inf, 0.0, most))
    total = e.sum(-1, keepdim=True)
    out = torch.matmul(e[..., : s["prefix"]].transpose(0, 1).reshape(hkv, r * hq // hkv, s["prefix"]), pv.permute(1, 0, 2)).view(hkv, r, hq // hkv, d).transpose(0, 1)
    out = out + torch.matmul(e[..., s["prefix"] :], ov.permute(0, 2, 1, 3))
    out = torch.where(total > 0, out / total, 0.0).reshape(r, hq, d)
    lse = (most + torch.log(total)).reshape(r, hq)
    live = s["lens"] >= 0
    s["out"].copy_(torch.where(live[:, None, None], out.to(s["out"].dtype), s["out"]))
    s["lse"].copy_(torch.where(live[:, None], lse, s["lse"]))


# ------------------------------------------------------------------------------------- one pass
def _handle(s):
    """The layer's description and the workspace: a user's program makes them once and keeps them."""
    import paper_2608_06007_b200 as tc
    if "layer" not in s:
        case = s["case"]
        layout = tc.TC_NHD if case["layout"] == "nhd" else tc.TC_HND
        kind = {"bf16": tc.TC_BF16, "fp16": tc.TC_FP16, "fp32": tc.TC_FP32, "e4m3": tc.TC_E4M3, "int8": tc.TC_INT8}[case["pool"]]
        planes, scales = s["pool"], s["scales"]
        pool = tc.pool(layout, s["blocks"], 1, plane_stride=planes.stride(0) * planes.element_size())
        more = {} if scales is None else dict(scale_pool=tc.pool(layout, s["blocks"], 1, plane_stride=scales.stride(0) * 4), scale_bases=[scales])
        s["layer"] = tc.kv_layer(pool, (case["block"], case["hkv"], case["d"]), kind, [planes], **more)
        if case["op"] == "attend":
            s["workspace"] = torch.empty(tc.tc_attn_workspace_bytes(s["layer"], s["q"], max_len=s["longest"], max_prefix=s["prefix"]), dtype=torch.uint8, device="cuda")
    return tc, s["layer"]


def run(s):
    case = s["case"]
    if case["op"] == "append":
        if own:
            tc, layer = _handle(s)
            tc.tc_kv_append(layer, s["k"], s["v"], s["slots"], q=s["q"], q_out=s["q_out"], positions=s["positions"], cos=s["cos"], sin=s["sin"], interleaved=case["interleaved"])
        else:
            _plain_append(s)
        # codes are e4m3 or int8 numbers; with its row's scale each is the value that it stands for
        pool = s["pool"][:, : s["blocks"]]
        return dict(q=s["q_out"], pool=pool, **({} if s["scales"] is None else dict(scales=s["scales"][:, : s["blocks"]])))
    if case["op"] == "gather":
        if own:
            tc, layer = _handle(s)
            tc.tc_kv_gather(layer, s["tables"], s["offsets"], s["k_out"], s["v_out"])
        else:
            _plain_gather(s)
        return dict(k=s["k_out"], v=s["v_out"])
    if own:
        tc, layer = _handle(s)
        tc.tc_attn_decode(layer, s["q"], s["out"], s["tables"], s["lens"], max_len=s["longest"], prefix_table=s["shared"], prefix_len=s["prefix_len"], max_prefix=s["prefix"], lse=s["lse"], workspace=s["workspace"])
    else:
        _plain_attend(s)
    return dict(out=s["out"], lse=s["lse"])


def work(case):
    row, e = case["hkv"] * case["d"], _BYTES[case["pool"]]
    page = 2 * (row * e + (4 * case["hkv"] if case["pool"] in _TOP else 0))  # one token of a pool, K and V
    if case["op"] == "append":
        n, x = case["n"] - case["padded"], _BYTES[case["x"]]
        q = case["hq"] * case["d"]
        return dict(bytes=n * ((2 * q + 2 * row) * x + page + case["rot"] * 4 + 8) + case["n"] * 8, flops=n * 3 * case["rot"] * (case["hq"] + case["hkv"]))
    lengths = _lengths(case)
    if case["op"] == "gather":
        t = max(1, int(lengths.sum()))
        return dict(bytes=t * (page + 2 * row * _BYTES[case["out"]]) + 4 * int((-(-lengths // case["block"])).sum()), flops=0 if case["pool"] not in _TOP else t * 2 * row)
    live = lengths[: len(lengths) - case["padded"]]
    keys = int(live.sum()) + len(live) * case["prefix"]
    qo = len(live) * case["hq"] * (2 * case["d"] * _BYTES[case["x"]] + 4)
    pages = int((-(-live // case["block"])).sum()) - (-case["prefix"] // case["block"])
    return dict(bytes=(int(live.sum()) + (case["prefix"] if len(live) else 0)) * page + qo + 4 * pages + 4 * len(lengths), flops=4 * keys * case["hq"] * case["d"])


# --------------------------------------------------------------------- the definitions in 64 bits
def _value(s, plane, tokens, table):
    """Tokens of a table as 64-bit values, [tokens, heads, d]."""
    case = s["case"]
    t = torch.arange(tokens, device="cuda")
    b = table.long()[torch.div(t, case["block"], rounding_mode="floor")]
    flat = s["pool"][plane].transpose(1, 2) if case["layout"] == "hnd" else s["pool"][plane]
    codes = flat.view(torch.uint8)[b, t % case["block"]].view(torch.float8_e4m3fn) if case["pool"] == "e4m3" else flat[b, t % case["block"]]
    x = codes.double()
    if s["scales"] is not None:
        scale = s["scales"][plane].transpose(1, 2) if case["layout"] == "hnd" else s["scales"][plane]
        x *= scale[b, t % case["block"]].double().unsqueeze(-1)
    return x


def _exact_append(s):
    case = s["case"]
    rot, block = case["rot"], case["block"]
    live = torch.nonzero(s["slots"] >= 0).flatten()

    def turned(x):
        x = x[live].double()
        z = torch.complex(s["cos"][s["positions"][live]].double(), s["sin"][s["positions"][live]].double()).unsqueeze(1)
        first, second = (slice(0, rot, 2), slice(1, rot, 2)) if case["interleaved"] else (slice(0, rot // 2), slice(rot // 2, rot))
        w = torch.complex(x[..., first], x[..., second]) * z
        x[..., first], x[..., second] = w.real, w.imag
        return x

    q = torch.zeros(s["q_out"].shape, dtype=torch.float64, device="cuda")
    q[live] = turned(s["q"])
    shape = s["pool"][:, : s["blocks"]].shape
    want = torch.zeros(shape, dtype=torch.float64, device="cuda")
    scales = torch.zeros(shape[:-1], dtype=torch.float64, device="cuda")
    b, t = s["slots"][live] // block, s["slots"][live] % block
    for c, x in enumerate((turned(s["k"]), s["v"][live].double())):
        if case["pool"] in _TOP:
            most = x.abs().max(-1).values / _TOP[case["pool"]]
            x = x / most.clamp(min=_TINY)[..., None]
            (scales[c] if case["layout"] == "nhd" else scales[c].transpose(1, 2))[b, t] = most
        (want[c] if case["layout"] == "nhd" else want[c].transpose(1, 2))[b, t] = x
    if case["pool"] == "int8":
        return dict(q=q, pool=None, scales=scales)
    return dict(q=q, pool=want, **(dict(scales=scales) if case["pool"] in _TOP else {}))


def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] == "append":
        return _exact_append(s)
    if case["op"] == "gather":
        got = []
        for plane in (0, 1):
            out = torch.zeros(s["k_out"].shape, dtype=torch.float64, device="cuda")
            at = 0
            for r, n in enumerate(s["lengths"].tolist()):
                out[at : at + n] = _value(s, plane, n, s["tables"][r])
                at += n
            got.append(out)
        return dict(k=got[0], v=got[1])
    hkv, d = case["hkv"], case["d"]
    out = torch.zeros(s["out"].shape, dtype=torch.float64, device="cuda")
    lse = torch.zeros(s["lse"].shape, dtype=torch.float64, device="cuda")
    shared = [_value(s, c, s["prefix"], s["shared"]) for c in (0, 1)]
    for r, n in enumerate(s["lens"].tolist()):
        if n < 0:
            continue
        k, v = (torch.cat([shared[c], _value(s, c, n, s["tables"][r])]) for c in (0, 1))
        if not len(k):
            lse[r] = -math.inf
            continue
        q = s["q"][r].double().view(hkv, -1, d)
        score = torch.einsum("hgd,nhd->hgn", q, k) / math.sqrt(d)
        lse[r] = torch.logsumexp(score, -1).flatten()
        out[r] = torch.einsum("hgn,nhd->hgd", torch.softmax(score, -1), v).reshape(-1, d)
    return dict(out=out, lse=lse)
