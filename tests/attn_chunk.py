"""What the tests of tc_attn_chunk and tc_attn_decode_window share: a batch over a paged layer, and its comparison with 64 bits."""
import numpy as np
import torch

import paper_2608_06007_b200 as tc
from oracle import operators as orc
from test_operators_gpu import KIND, TORCH, Pool, dev, np64, tables_for, tokens_of

TOP = {"e4m3": 448.0, "int8": 127.0}


def batch(kind, x, lens, new, *, Hq, H=2, D=128, B=16, layout="nhd", window=0, sinks=0, scale=0.0, spread=1.0, seed=0, front=0, behind=0, extra_len=0, extra_new=0, poison=True, strided=False, gap=0):
    """A pool with the requests' tokens and the arguments of a call: lens[r] < 0 is padding (new[r] rows of q all the same)."""
    rng = np.random.default_rng([seed, KIND[kind], KIND[x], D, len(lens)])
    own = [max(0, n) for n in lens]
    pool = Pool(kind, layout=layout, D=D, H=H, B=B, blocks=sum(-(-n // B) for n in own) + 3, gap=gap)
    values = pool.fill(rng, spread)
    table = tables_for(own, pool, rng)
    if poison:  # slots that no token is in, and tokens that no row sees, hold NaN (codes: scales)
        used = np.zeros((pool.blocks, pool.B), dtype=bool)
        for tab, n, m in zip(table, own, new):
            t = np.arange(n)
            if window and n:
                t = t[(t < sinks) | (t > n - m - window)]
            if m:
                used[tab[t // B], t % B] = True
        idle = torch.from_numpy(~used).cuda()
        for c in (0, 1):
            if kind in TOP:
                pool.scale(c)[idle] = float("nan")
            else:
                pool.codes(c)[idle] = 0xFF
    offsets = front + np.concatenate([[0], np.cumsum(new)]).astype(np.int64)
    n = max(1, int(offsets[-1]) + behind)
    q = torch.from_numpy(rng.standard_normal((n, Hq, D)).astype(np.float32) * spread).to(TORCH[x])
    s = dict(pool=pool, x=x, q=q, dq=q.cuda(), lens=list(lens), new=list(new), table=table, values=values, offsets=offsets, window=window, sinks=sinks, scale=scale)
    if strided:
        s["dq"] = torch.zeros(Hq, n, D + 16, dtype=q.dtype, device="cuda").transpose(0, 1)[..., :D]
        s["dq"].copy_(q)
        s["out"] = torch.full((Hq, n, D + 8), 9.0, dtype=q.dtype, device="cuda").transpose(0, 1)[..., :D]
    else:
        s["out"] = torch.full((n, Hq, D), 9.0, dtype=q.dtype, device="cuda")
    s["lse"] = torch.full((n, Hq), 9.0, device="cuda")
    s["max_len"], s["max_new"] = max(1, max(own)) + extra_len, max(1, max(new)) + extra_new
    if extra_len:
        table = np.pad(table, ((0, 0), (0, -(-extra_len // B) + 1)), constant_values=-1)
    s["d"] = dict(tables=dev(table), offsets=dev(offsets), lens=dev(np.array(lens, dtype=np.int32)))
    return s


def run_chunk(s, workspace=None, **changes):
    pool = s["pool"]
    bounds = dict(max_new=s["max_new"], max_len=s["max_len"], window=s["window"], sinks=s["sinks"])
    if workspace is None:
        need = tc.tc_attn_chunk_workspace_bytes(pool.handle, s["dq"], len(s["lens"]), **bounds)
        workspace = torch.full((need,), 0xFF, dtype=torch.uint8, device="cuda")
    tc.tc_attn_chunk(pool.handle, s["dq"], s["out"], **(bounds | s["d"] | dict(scale=s["scale"], lse=s["lse"], workspace=workspace) | changes))


def rows_off(s, r, row0, n, keys, vals, kernel_rounds, there=None, far=False):
    """Outputs and logarithms of one request against 64 bits, within what each rounding may do.

    Half a step is 2^-9 of a bf16 number and 2^-12 of an fp16 one at most relative to it where steps are taken at the
    power of two below it, eps / 2 = 2^-8 and 2^-11 for the worst of them: a probability is rounded once, or as often as
    kernel_rounds says.  A score is an fp32 sum of D exact products and
    three fp32 factors, so (D + 4) 2^-24 of sum |q k| scale; it moves weights by twice that, relatively.  The exponential, the sum and
    the powers are good to 2^-18 together.  Half-precision products below 2^-14 of a row's largest contribution are off by 2^-25
    each, and where codes' scales are taken in, by 2^-15 of a key's weight times its scale.  far: weights are 2 to the power of sums of
    logarithms of up to some hundreds, in fp32, and off by 2^-14.  Then the output's own half step."""
    pool, x = s["pool"], s["x"]
    scale = s["scale"] or pool.D ** -0.5
    g = s["q"].shape[1] // pool.H
    q = np64(s["q"])[row0 : row0 + n]
    want, want_lse, w = orc.attend_chunk(q, keys, vals, scale, s["window"], s["sinks"], there)
    out, lse = np64(s["out"])[row0 : row0 + n], np64(s["lse"])[row0 : row0 + n]
    codes = pool.kind in TOP
    u_o = torch.finfo(TORCH[x]).eps / 2
    u_p = kernel_rounds * 2.0 ** -11 if codes else u_o
    k, v = (np.repeat(np.where(np.isfinite(y).all(-1)[..., None], y, 0), g, axis=1) for y in (keys, vals))
    w = np.nan_to_num(w)
    mass = np.einsum("nhl,lhd->nhd", w, np.abs(v))
    length = np.einsum("nhd,lhd->nhl", np.abs(q), np.abs(k)) * abs(scale)
    delta = ((pool.D + 4) * 2.0 ** -24 * np.where(w > 0, length, 0).max(-1)) if len(keys) else np.zeros(q.shape[:2])
    most = (u_p * (1 + 2.0 ** -6) + 2 * delta[..., None] + 2.0 ** (-14 if far else -18)) * mass + u_o * (1 + 2.0 ** -6) * np.abs(want) + (2.0 ** -25 if x == "fp16" else 1e-30)
    if codes or x == "fp16":
        size = np.abs(v).max(-1) if len(v) else np.zeros((0, q.shape[1]))  # [len, Hq]
        seen = w > 0
        largest = np.where(seen, w * size.T, 0).max(-1) if len(v) else 0
        most += (seen.sum(-1) * 2.0 ** -24 * largest)[..., None]
        if codes:
            most += (2.0 ** -15 * (w * size.T).sum(-1))[..., None]
    most, finite = np.nan_to_num(most, nan=np.inf), np.isfinite(want)
    assert (np.isfinite(out) == finite).all(), (r, "finite")
    off = np.where(finite, np.abs(np.where(finite, out, 0) - np.where(finite, want, 0)), 0)
    assert (off <= np.where(finite, most, 0)).all(), (r, off.max(), (off / np.maximum(np.where(finite, most, 1), 1e-300)).max(), np.unravel_index((off - np.where(finite, most, 0)).argmax(), off.shape))
    good = np.isfinite(want_lse)
    assert (np.isnan(lse) == np.isnan(want_lse)).all() and (lse[np.isneginf(want_lse)] == -np.inf).all(), r
    assert (np.abs(lse - want_lse)[good] <= (delta + 2.0 ** -18 + 2.0 ** -22 * np.abs(want_lse))[good]).all(), r


def check_chunk(s, only=None, left_out=(), there=None, far=False):
    """Every request against the oracle, and every row that is nobody's as it was.  there: of a request, which of its keys can be read."""
    pool, offsets = s["pool"], s["offsets"]
    mine = np.zeros(len(s["q"]), dtype=bool)
    for r, (n, m) in enumerate(zip(s["lens"], s["new"])):
        if n < 0 or m == 0 or r in left_out:
            continue
        row0 = int(offsets[r])
        mine[row0 : row0 + m] = True
        if only is not None and r not in only:
            continue
        keys, vals = (tokens_of(v, s["table"][r], 0, n, pool.B) for v in s["values"])
        rows_off(s, r, row0, m, keys, vals, 1, None if there is None else there.get(r), far)
    out, lse = np64(s["out"]), np64(s["lse"])
    assert (out[~mine] == 9.0).all() and (lse[~mine] == 9.0).all()


def window_batch(kind, x, lens, **more):
    """One query token per request: a batch whose rows of q are the requests', padding among them."""
    s = batch(kind, x, lens, [1 if n > 0 else 0 for n in lens], **more)
    Hq, D, R = s["q"].shape[1], s["pool"].D, len(lens)
    rng = np.random.default_rng(R)
    s["q"] = torch.from_numpy(rng.standard_normal((R, Hq, D)).astype(np.float32) * more.get("spread", 1.0)).to(TORCH[x])
    if more.get("strided"):
        s["dq"] = torch.zeros(Hq, R, D + 16, dtype=s["q"].dtype, device="cuda").transpose(0, 1)[..., :D]
        s["dq"].copy_(s["q"])
        s["out"] = torch.full((Hq, R, D + 8), 9.0, dtype=s["q"].dtype, device="cuda").transpose(0, 1)[..., :D]
    else:
        s["dq"], s["out"] = s["q"].cuda(), torch.full((R, Hq, D), 9.0, dtype=s["q"].dtype, device="cuda")
    s["lse"] = torch.full((R, Hq), 9.0, device="cuda")
    s["offsets"] = np.arange(R + 1)
    del s["d"]["offsets"]
    return s


def run_window(s, workspace=None, **changes):
    pool = s["pool"]
    if workspace is None:
        workspace = torch.full((tc.tc_attn_workspace_bytes(pool.handle, s["dq"], max_len=s["max_len"]),), 0xFF, dtype=torch.uint8, device="cuda")
    args = dict(window=s["window"], sinks=s["sinks"], max_len=s["max_len"], scale=s["scale"], lse=s["lse"], workspace=workspace) | s["d"] | changes
    tc.tc_attn_decode_window(pool.handle, s["dq"], s["out"], **args)


def check_window(s, only=None, there=None):
    pool = s["pool"]
    out, lse = np64(s["out"]), np64(s["lse"])
    for r, n in enumerate(s["lens"]):
        if n < 0:
            assert (out[r] == 9.0).all() and (lse[r] == 9.0).all()
        elif n == 0:
            assert (out[r] == 0).all() and (lse[r] == -np.inf).all()
        elif only is None or r in only:
            keys, vals = (tokens_of(v, s["table"][r], 0, n, pool.B) for v in s["values"])
            rows_off(s, r, r, 1, keys, vals, 1, None if there is None else there.get(r))


def set_rows(s, plane, r, tokens, value):
    """Tokens of request r in a plane: every element (of codes: every scale) becomes `value`, in the oracle's values too."""
    pool, t = s["pool"], np.asarray(tokens)
    block, at = s["table"][r][t // pool.B], t % pool.B
    if pool.kind in TOP:
        pool.scale(plane)[torch.from_numpy(block).long().cuda(), torch.from_numpy(at).cuda()] = value
    else:
        bits = torch.full((len(t), pool.H, pool.D), value, dtype=TORCH[pool.kind]).view(torch.uint8)
        pool.codes(plane)[torch.from_numpy(block).long().cuda(), torch.from_numpy(at).cuda()] = bits.cuda()
    s["values"][plane][block, at] = value if pool.kind not in TOP else np.nan


def set_scales(s, plane, make):
    """New scales of a pool of codes: make(t, shape) -> powers of two, of the tokens t of each request, for all heads."""
    pool = s["pool"]
    old = np64(pool.scale(plane)).copy()
    new = old.copy()
    for table, n in zip(s["table"], s["lens"]):
        t = np.arange(max(0, n))
        new[table[t // pool.B], t % pool.B] = make(t, (len(t), pool.H))
    pool.scale(plane).copy_(torch.from_numpy(new.astype(np.float32)))
    with np.errstate(invalid="ignore"):
        s["values"][plane] = s["values"][plane] / old[..., None] * new.astype(np.float32).astype(np.float64)[..., None]
