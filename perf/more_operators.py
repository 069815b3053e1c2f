"""More paged-cache operators as they are measured: attention of chunks of new tokens over a paged cache, and attention
with a sliding window and a few first tokens that stay visible, for chunks and for one token per request.

`run` computes them in elementary torch operations, or, where `own` is true, calls the library.
Lengths come from the case alone, contents and block tables from the seed.
"""
import math

import numpy as np
import torch

own = False

_TORCH = {"bf16": torch.bfloat16, "fp16": torch.float16, "e4m3": torch.float8_e4m3fn, "int8": torch.int8}
_BYTES = {"bf16": 2, "fp16": 2, "e4m3": 1, "int8": 1}
_TOP = {"e4m3": 448.0, "int8": 127.0}


# ---------------------------------------------------------------------------------------- cases
def listed():
    """`new` tokens of each of r requests stand behind `cached` ones.  Shapes: 32 query and 8 KV heads of 128, blocks of 16
    (the 8B model's cache); 64 and 8, blocks of 32 (the 70B model's); generic others."""
    chunk = dict(op="chunk", hq=32, hkv=8, d=128, block=16, layout="nhd", x="bf16", pool="bf16", window=0, sinks=0, padded=0)
    window = dict(chunk, op="window", sinks=4)
    single = dict(window, op="single", new="1")
    return [
        # a few requests whose last tokens were guessed ahead and are looked at together: latency
        dict(chunk, name="chunk 4 of 1 to 7", r=4, new="7,1,5,3", cached="30,99,0,197"),
        # one piece of a long prompt, as a scheduler cuts it
        dict(chunk, name="chunk 2048 behind 6144", r=1, new="2048", cached="6144"),
        # a serving step: pieces of four prompts beside sessions that decode, on a quantised cache, padded up for a captured graph
        dict(chunk, name="chunk mixed 64 e4m3", r=64, new="some:4:100:1000", cached="log:200:16000", pool="e4m3", layout="hnd", padded=9),
        # a short question about a very long document
        dict(chunk, name="chunk 33 behind 120000 int8", r=1, new="33", cached="120000", hq=28, hkv=4, pool="int8"),
        # whole prompts, nothing cached, a KV head per query head
        dict(chunk, name="chunk 16 prompts d 80", r=16, new="log:50:6000", cached="0", hq=16, hkv=16, d=80, block=20, x="fp16", pool="fp16"),
        # a large piece of a very long prompt of the 70B model
        dict(chunk, name="chunk 8192 behind 24576", r=1, new="8192", cached="24576", hq=64, block=32, x="fp16", pool="fp16"),
        # a few short requests, one of them shorter than the window: latency
        dict(single, name="window single 3", r=3, cached="36,499,1200", window=128),
        # a serving batch of long conversations
        dict(single, name="window single 64", r=64, cached="log:500:60000", window=4096),
        # the agent burst's 512 sessions on a quantised cache; some rows are padding
        dict(single, name="window single 512 e4m3", r=512, cached="log:100:8000", window=1024, sinks=16, pool="e4m3", layout="hnd", padded=7),
        # a piece of a prompt in a layer that looks at its neighbourhood
        dict(window, name="window 4096 behind 12288 d 64", r=1, new="4096", cached="12288", hq=64, d=64, window=1024),
        # whole prompts of mixed lengths on a quantised cache
        dict(window, name="window 8 prompts int8", r=8, new="log:500:16000", cached="0", window=2048, sinks=64, pool="int8"),
        # pieces of prompts in a model of wide heads
        dict(window, name="window 5 of about 1500 d 256", r=5, new="uniform:1000:2001", cached="log:1:4000", hq=16, hkv=4, d=256, block=64, window=512, sinks=1),
    ]


def draw(rng):
    """A case of the same ranges."""
    def spread(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))

    op = rng.choice(["chunk", "chunk", "window", "single"])
    hkv, d, x = rng.choice([1, 2, 4, 8]), rng.choice([64, 80, 96, 128, 128, 128, 256]), rng.choice(["bf16", "fp16"])
    hq = hkv * rng.choice([1, 2, 4, 5, 7, 8])
    r = spread(1, 64 if op != "single" else 512)
    # tokens of a cache that keep the pool and the products within bounds
    most = max(1, min(131072 if r == 1 else 32768, 150_000_000 // (r * hkv * d)))
    cached = spread(1, most)
    case = dict(op=op, r=r, hq=hq, hkv=hkv, d=d, block=rng.choice([8, 16, 20, 32, 64]), layout=rng.choice(["nhd", "hnd"]), x=x, pool=rng.choice([x, x, "e4m3", "int8"]),
                window=0, sinks=0, draw=rng.randrange(1 << 30))
    case["cached"] = rng.choice([f"log:1:{cached + 1}", f"uniform:0:{cached}", f"uniform:{cached - cached // 8}:{cached}"])
    case["padded"] = rng.choice([0, rng.randint(0, r - 1)])
    if op != "chunk":
        case["window"], case["sinks"] = spread(1, 8192), rng.choice([0, 1, 4, 16, 100])
    if op == "single":
        return dict(case, new="1")
    seen = min(cached + 8192, case["window"] + case["sinks"] if case["window"] else 1 << 30)
    new = spread(1, max(1, min(8192, 1_000_000_000_000 // (4 * r * hq * d * seen), 150_000_000 // (r * hq * d))))
    case["new"] = rng.choice([f"log:1:{new + 1}", f"uniform:{new - new // 8}:{new}", f"some:{min(r, 3)}:1:{new + 1}"])
    return case


def _lengths(case):
    """(new, cached) tokens of every request; the last `padded` requests have none."""
    r = case["r"]
    got = []
    for i, spec in enumerate((case["new"], case["cached"])):
        rng = np.random.default_rng([27 + i, r, case.get("draw", 0)])
        kind, *numbers = spec.split(":")
        if kind == "log":
            lo, hi = map(int, numbers)
            v = np.rint(np.exp(rng.uniform(math.log(lo), math.log(hi), r))).astype(np.int64)
        elif kind == "uniform":
            v = rng.integers(int(numbers[0]), int(numbers[1]) + 1, r)
        elif kind == "some":
            some, lo, hi = map(int, numbers)
            v = np.ones(r, dtype=np.int64)
            v[rng.permutation(r)[:some]] = np.rint(np.exp(rng.uniform(math.log(lo), math.log(hi), some)))
        else:
            v = np.array([int(x) for x in spec.split(",")], dtype=np.int64)
            v = np.broadcast_to(v, r).copy()
        got.append(v)
    for v in got:
        v[r - case["padded"] :] = 0
    return got


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
    shape, kind = (2, blocks, *inner, case["d"]), case["pool"]
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


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    rng = np.random.default_rng(seed)
    new, cached = _lengths(case)
    total, r, size = new + cached, case["r"], case["block"]
    need = -(-total // size)
    blocks = int(need.sum()) * 9 // 8 + 1
    s = dict(case=case, new=new.tolist(), total=total.tolist(), blocks=blocks, max_new=int(max(1, new.max())), max_len=int(max(1, total.max())))
    s["pool"], s["scales"] = _pool(case, blocks, gen)
    # a block table a request over a seeded permutation of the pool, padded with an id that is never to be read
    tables = np.full((r, max(1, int(need.max()))), -1, dtype=np.int32)
    tables[np.arange(tables.shape[1])[None, :] < need[:, None]] = rng.permutation(blocks)[: int(need.sum())]
    s["tables"] = torch.from_numpy(tables).cuda()
    lens = total.astype(np.int32)
    lens[r - case["padded"] :] = -1
    s["lens"] = torch.from_numpy(lens).cuda()
    offsets = np.concatenate([[0], np.cumsum(new)]).astype(np.int64)
    s["starts"], s["offsets"] = offsets.tolist(), torch.from_numpy(offsets).cuda()
    # one row of queries a request, or the new tokens of all and some rows of padding behind them
    rows = r if case["op"] == "single" else int(offsets[-1]) + case["padded"]
    s["q"] = _normal(gen, (max(1, rows), case["hq"], case["d"]), case["x"])
    s["out"] = torch.zeros_like(s["q"])
    s["lse"] = torch.zeros(s["q"].shape[:2], device="cuda")
    return s


# ------------------------------------------------------------------------------- the plain forms
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


def _plain_chunk(s):
    """Request by request, as many new tokens at a time as 2^28 scores allow."""
    case = s["case"]
    size, hkv, hq, d, window, sinks = case["block"], case["hkv"], case["hq"], case["d"], case["window"], case["sinks"]
    for r, (n, total, start) in enumerate(zip(s["new"], s["total"], s["starts"])):
        step = max(1, (1 << 28) // (hq * (min(total, window + 1024 + sinks) if window else max(total, 1))))
        step = min(step, 1024) if window else step
        for a in range(0, n, step):
            b = min(n, a + step)
            pos = torch.arange(total - n + a, total - n + b, device="cuda")
            last = total - n + b
            j = torch.arange(last, device="cuda")
            if window and total - n + a - window + 1 > sinks:
                j = torch.cat([j[:sinks], j[total - n + a - window + 1 :]])
            block = s["tables"][r, j // size].long()
            k, v = (_pages(s, c, block, j % size).permute(1, 0, 2) for c in (0, 1))  # [hkv, keys, d]
            q = (s["q"][start + a : start + b].float() * (1 / math.sqrt(d))).view(b - a, hkv, hq // hkv, d).permute(1, 0, 2, 3)
            seen = j[None, :] <= pos[:, None]
            if window:
                seen &= (j[None, :] > pos[:, None] - window) | (j[None, :] < sinks)
            score = torch.matmul(q.reshape(hkv, -1, d), k.transpose(1, 2)).view(hkv, b - a, hq // hkv, len(j))
            score.masked_fill_(~seen[None, :, None, :], -math.inf)
            most = score.amax(-1, keepdim=True)
            e = score.sub_(most).exp_()
            sums = e.sum(-1, keepdim=True)
            out = torch.matmul(e.view(hkv, -1, len(j)), v).view(hkv, b - a, hq // hkv, d) / sums
            s["out"][start + a : start + b] = out.permute(1, 0, 2, 3).reshape(b - a, hq, d).to(s["out"].dtype)
            s["lse"][start + a : start + b] = (most + torch.log(sums)).permute(1, 0, 2, 3).reshape(b - a, hq)


def _plain_single(s):
    """All requests at once over the first tokens and the window, some of them not there."""
    case = s["case"]
    size, hkv, hq, d, sinks = case["block"], case["hkv"], case["hq"], case["d"], case["sinks"]
    window = min(case["window"], s["max_len"])
    lens = s["lens"].long()[:, None]
    first = (lens - window).clamp(min=0)
    for a in range(0, len(lens), 64):
        part = slice(a, min(len(lens), a + 64))
        near = first[part] + torch.arange(window, device="cuda")
        far = torch.arange(sinks, device="cuda").expand(len(near), -1)
        j = torch.cat([far, near], 1)
        seen = torch.cat([far < first[part], near < lens[part]], 1) & (j < lens[part])
        block = torch.gather(s["tables"][part].long(), 1, (j // size).clamp(max=s["tables"].shape[1] - 1)).clamp(min=0)
        k, v = (_pages(s, c, block, j % size) for c in (0, 1))  # [r, keys, hkv, d]
        q = s["q"][part].float().view(len(near), hkv, hq // hkv, d) * (1 / math.sqrt(d))
        score = torch.matmul(q, k.permute(0, 2, 3, 1)).masked_fill_(~seen[:, None, None, :], -math.inf)
        most = score.amax(-1, keepdim=True)
        e = torch.exp(score - torch.where(most == -math.inf, 0.0, most))
        sums = e.sum(-1, keepdim=True)
        out = torch.where(sums > 0, torch.matmul(e, torch.where(seen[..., None, None], v, 0.0).permute(0, 2, 1, 3)) / sums, 0.0).reshape(len(near), hq, d)
        live = lens[part] >= 0
        s["out"][part] = torch.where(live[..., None], out.to(s["out"].dtype), s["out"][part])
        s["lse"][part] = torch.where(live, (most + torch.log(sums)).reshape(len(near), hq), s["lse"][part])


# ------------------------------------------------------------------------------------- one pass
def _handle(s):
    """The layer's description and the workspace: a user's program makes them once and keeps them."""
    import paper_2608_06007_b200 as tc
    if "layer" not in s:
        case = s["case"]
        layout = tc.TC_NHD if case["layout"] == "nhd" else tc.TC_HND
        kind = {"bf16": tc.TC_BF16, "fp16": tc.TC_FP16, "e4m3": tc.TC_E4M3, "int8": tc.TC_INT8}[case["pool"]]
        planes, scales = s["pool"], s["scales"]
        pool = tc.pool(layout, s["blocks"], 1, plane_stride=planes.stride(0) * planes.element_size())
        more = {} if scales is None else dict(scale_pool=tc.pool(layout, s["blocks"], 1, plane_stride=scales.stride(0) * 4), scale_bases=[scales])
        s["layer"] = tc.kv_layer(pool, (case["block"], case["hkv"], case["d"]), kind, [planes], **more)
        if case["op"] == "single":
            need = tc.tc_attn_workspace_bytes(s["layer"], s["q"], max_len=s["max_len"])
        else:
            need = tc.tc_attn_chunk_workspace_bytes(s["layer"], s["q"], case["r"], max_new=s["max_new"], max_len=s["max_len"], window=case["window"], sinks=case["sinks"])
        s["workspace"] = torch.empty(need, dtype=torch.uint8, device="cuda")
    return tc, s["layer"]


def run(s):
    case = s["case"]
    if own:
        tc, layer = _handle(s)
        if case["op"] == "single":
            tc.tc_attn_decode_window(layer, s["q"], s["out"], s["tables"], s["lens"], window=case["window"], sinks=case["sinks"], max_len=s["max_len"], lse=s["lse"], workspace=s["workspace"])
        else:
            tc.tc_attn_chunk(layer, s["q"], s["out"], s["tables"], s["offsets"], s["lens"], max_new=s["max_new"], max_len=s["max_len"], window=case["window"], sinks=case["sinks"],
                             lse=s["lse"], workspace=s["workspace"])
    elif case["op"] == "single":
        _plain_single(s)
    else:
        _plain_chunk(s)
    return dict(out=s["out"], lse=s["lse"])


def work(case):
    new, cached = _lengths(case)
    window, sinks = case["window"] or 1 << 40, case["sinks"]
    pairs = keys = pages = 0
    for n, c in zip(new.tolist(), cached.tolist()):
        if not n:
            continue
        pos = np.arange(c, c + n)
        near = np.minimum(pos + 1, window)
        pairs += int((near + np.minimum(sinks, pos + 1 - near)).sum())
        first = max(0, c - window + 1)  # of the keys that any of the new tokens sees, behind the first ones
        keys += c + n - first + min(sinks, first)
        pages += -(-(c + n - first + min(sinks, first)) // case["block"])
    page = 2 * (case["hkv"] * case["d"] * _BYTES[case["pool"]] + (4 * case["hkv"] if case["pool"] in _TOP else 0))
    return dict(bytes=keys * page + int(new.sum()) * case["hq"] * (2 * case["d"] * 2 + 4) + 4 * pages + 12 * case["r"], flops=4 * pairs * case["hq"] * case["d"])


# --------------------------------------------------------------------- the definitions in 64 bits
def _value(s, plane, tokens, table):
    """Tokens (a vector of them) of a table as 64-bit values, [heads, tokens, d]."""
    case = s["case"]
    b, t = table.long()[torch.div(tokens, case["block"], rounding_mode="floor")], tokens % case["block"]
    flat = s["pool"][plane].transpose(1, 2) if case["layout"] == "hnd" else s["pool"][plane]
    x = (flat.view(torch.uint8)[b, t].view(torch.float8_e4m3fn) if case["pool"] == "e4m3" else flat[b, t]).double()
    if s["scales"] is not None:
        scale = s["scales"][plane].transpose(1, 2) if case["layout"] == "hnd" else s["scales"][plane]
        x *= scale[b, t].double().unsqueeze(-1)
    return x.transpose(0, 1)


def exact(case, seed):
    s = prepare(case, seed)
    hkv, hq, d = case["hkv"], case["hq"], case["d"]
    window, sinks = case["window"] or 1 << 40, case["sinks"]
    out = torch.zeros(s["out"].shape, dtype=torch.float64, device="cuda")
    lse = torch.zeros(s["lse"].shape, dtype=torch.float64, device="cuda")
    for r, (n, total) in enumerate(zip(s["new"], s["total"])):
        row0 = r if case["op"] == "single" else s["starts"][r]
        for a in range(0, n, 128):
            m = min(n, a + 128) - a
            p0 = total - n + a  # position of the first of these m tokens
            lo = max(0, p0 - window + 1)
            tokens = torch.cat([torch.arange(min(sinks, lo)), torch.arange(lo, p0 + m)]).cuda()
            k, v = _value(s, 0, tokens, s["tables"][r]), _value(s, 1, tokens, s["tables"][r])
            distance = (p0 + torch.arange(m, device="cuda"))[:, None] - tokens
            hidden = (distance < 0) | ((distance >= window) & (tokens >= sinks))
            rows = slice(row0 + a, row0 + a + m)
            q = s["q"][rows].double().view(m, hkv, -1, d).transpose(0, 1)  # [hkv, m, g, d]
            score = torch.einsum("hmgd,hnd->hgmn", q, k) / math.sqrt(d)
            score[:, :, hidden] = -math.inf
            lse[rows] = torch.logsumexp(score, -1).permute(2, 0, 1).reshape(m, hq)
            out[rows] = torch.einsum("hgmn,hnd->mhgd", torch.softmax(score, -1), v).reshape(m, hq, d)
    return dict(out=out, lse=lse)
