"""The operators of a decode step over many live streams, as cases: inputs, one pass, and what a pass
cannot do without.

Whoever scores the macroblocks of live streams with a transformer that remembers each stream's past
runs one token per stream and frame through it: the scores go to select_regions.  A stream is what a
request is elsewhere, a token is one frame (or one macroblock of one) of it.

Kinds of case
  plan     RH.cache_plan: pages of the key-value cache for the new tokens of every stream, the block
           table and the slot of every token, pages of ended streams given back
  write    RH.cache_write: keys and values of the new tokens into their slots, rounded or quantised
  attend   RH.cache_attend: one new token of every stream over the stream's cached tokens
  norm     RH.norm_residual: residual addition and root-mean-square norm, output also in 8 bits
  matvec   RH.matvec_packed: products with weights in 4 bits that share a scale by 32

Frames are those of the benchmark configurations (workloads/): 510 macroblocks for 480 x 272, 920
for 640 x 368, 8 streams, 16 or 30 frames a chunk; widths and heads are generic.
"""
import math
import random

import torch

own = False

E4M3 = torch.float8_e4m3fn
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "e4m3": E4M3}
SIZE = {"f32": 4, "bf16": 2, "e4m3": 1}
FP4 = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)          # magnitudes of the codes 0..7; bit 3 is the sign
EPS = 1e-6


def listed():
    return [
        # the step of one batch as a frame of each of 8 streams arrives: nothing but latency
        {"name": "plan_8_streams_1_token", "op": "plan", "streams": 8, "chunk": 1, "history": 300, "page": 16, "ended": 0.0, "room": 1.5},
        # 500 streams join with chunks of up to 4096 macroblock tokens while others end; pages that divide nothing
        {"name": "plan_500_streams_chunks", "op": "plan", "streams": 500, "chunk": 4096, "history": 8192, "page": 48, "ended": 0.1, "room": 1.1},
        # keys and values of one frame of 64 streams, out of the fused projection's rows
        {"name": "write_64_bf16", "op": "write", "tokens": 64, "kv_heads": 8, "dim": 128, "page": 16, "type": "bf16", "cache": "bf16", "order": "token"},
        # the macroblock tokens of a chunk of 30 frames of 920, quantised
        {"name": "write_27600_e4m3", "op": "write", "tokens": 27600, "kv_heads": 8, "dim": 128, "page": 64, "type": "bf16", "cache": "e4m3", "order": "head"},
        # 8 streams with ten seconds of frames behind them, a small fp32 predictor
        {"name": "attend_8x300_f32", "op": "attend", "streams": 8, "length": 300, "heads": 8, "kv_heads": 8, "dim": 64, "page": 16,
         "type": "f32", "cache": "f32", "order": "token", "window": 0, "idle": 0},
        # 64 streams of very different ages, grouped heads: the ordinary large step
        {"name": "attend_64x8192_bf16", "op": "attend", "streams": 64, "length": 8192, "heads": 32, "kv_heads": 8, "dim": 128, "page": 16,
         "type": "bf16", "cache": "bf16", "order": "token", "window": 0, "idle": 1},
        # one stream, an hour of frames: all the work is along one axis; the cache in 8 bits
        {"name": "attend_1x108000_e4m3", "op": "attend", "streams": 1, "length": 108000, "heads": 16, "kv_heads": 2, "dim": 128, "page": 64,
         "type": "bf16", "cache": "e4m3", "order": "head", "window": 0, "idle": 0},
        # odd head size, odd pages, the last 1000 tokens only, idle streams among them
        {"name": "attend_30x5000_window", "op": "attend", "streams": 30, "length": 5000, "heads": 12, "kv_heads": 4, "dim": 96, "page": 20,
         "type": "bf16", "cache": "bf16", "order": "token", "window": 1000, "idle": 3},
        # one frame of 8 streams: a row a stream, output in 8 bits for the next product
        {"name": "norm_8x1024_bf16", "op": "norm", "rows": 8, "cols": 1024, "type": "bf16", "residual": True, "out": "e4m3"},
        # the macroblock tokens of 16 frames of 920 at once, both outputs; a width that no vector divides
        {"name": "norm_14720x4095_f32", "op": "norm", "rows": 14720, "cols": 4095, "type": "f32", "residual": True, "out": "both"},
        # one stream: macroblock features of a 480 x 272 frame into the predictor
        {"name": "matvec_1x1024x510_f32", "op": "matvec", "rows": 1, "outputs": 1024, "inputs": 510, "type": "f32", "out": "f32", "relu": False},
        # the widest product of 16 streams, 8-bit rows from the norm
        {"name": "matvec_16x16384x4096_e4m3", "op": "matvec", "rows": 16, "outputs": 16384, "inputs": 4096, "type": "e4m3", "out": "bf16", "relu": True},
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng: random.Random):
    most = max(work(c)["bytes"] for c in listed())
    while True:
        op = rng.choice(("plan", "write", "attend", "attend", "norm", "matvec", "matvec"))
        if op == "plan":
            c = {"op": op, "streams": _log(rng, 1, 1000), "chunk": rng.choice((1, 1, _log(rng, 2, 4096))), "history": _log(rng, 1, 16384),
                 "page": rng.choice((1, 8, 16, 20, 48, 64, 128)), "ended": rng.choice((0.0, 0.1, 0.5)), "room": rng.choice((0.6, 1.0, 1.5))}
        elif op == "write":
            kind, cache = rng.choice((("f32", "f32"), ("f32", "bf16"), ("f32", "e4m3"), ("bf16", "bf16"), ("bf16", "e4m3")))
            c = {"op": op, "tokens": _log(rng, 1, 32768), "kv_heads": rng.choice((1, 2, 3, 4, 8, 16)), "dim": 32 * rng.randint(1, 8),
                 "page": rng.choice((1, 8, 16, 20, 48, 64, 128)), "type": kind, "cache": cache, "order": rng.choice(("token", "head"))}
        elif op == "attend":
            kind, cache = rng.choice((("f32", "f32"), ("bf16", "bf16"), ("bf16", "bf16"), ("bf16", "e4m3")))
            h = rng.choice((1, 2, 3, 4, 8))
            c = {"op": op, "streams": _log(rng, 1, 128), "length": _log(rng, 1, 131072), "heads": h * rng.choice((1, 2, 3, 4, 6, 8, 16, 20)),
                 "kv_heads": h, "dim": 32 * rng.randint(1, 8), "page": rng.choice((1, 8, 16, 20, 48, 64, 128)), "type": kind, "cache": cache,
                 "order": rng.choice(("token", "head")), "window": 0, "idle": rng.choice((0, 1, 4))}
            if rng.random() < 0.25:
                c["window"] = _log(rng, 1, 4096)
            if c["streams"] * c["length"] * h * c["dim"] > 64 * 8192 * 8 * 128:
                continue
        elif op == "norm":
            c = {"op": op, "rows": _log(rng, 1, 16384), "cols": rng.choice((_log(rng, 1, 16384), 64 * rng.randint(1, 128))),
                 "type": rng.choice(("f32", "bf16")), "residual": rng.random() < 0.7, "out": rng.choice(("same", "e4m3", "both"))}
        else:
            c = {"op": op, "rows": rng.choice((1, 1, _log(rng, 1, 64))), "outputs": rng.choice((_log(rng, 1, 32768), 256 * rng.randint(1, 64))),
                 "inputs": rng.choice((_log(rng, 1, 16384), 256 * rng.randint(1, 64))), "type": rng.choice(("f32", "bf16", "e4m3")),
                 "out": rng.choice(("f32", "bf16")), "relu": rng.random() < 0.3}
            if c["outputs"] * c["inputs"] > 16384 * 4096:
                continue
        if 3072 not in c.values() and c.get("heads", 0) * c.get("dim", 0) != 3072 and work(c)["bytes"] <= most:
            return c


def _spread(n, most, least=1):
    """n whole numbers between least and most: the largest first, then the smallest, the others spread evenly."""
    return [most if i == 0 else least if i == 1 else least + int((most - least) * ((i * 0.6180339887498949) % 1.0)) for i in range(n)]


def _lengths(case):
    """Cached tokens of every stream (the idle ones have none)."""
    got = _spread(case["streams"], case["length"])
    for i in range(min(case["idle"], case["streams"] - 1)):
        got[-1 - i] = 0
    return got


def _kept(case):
    w = case["window"]
    return [min(n, w) if w else n for n in _lengths(case)]


def _plan_lists(case):
    """(tokens at hand, new tokens) of every stream; -1 new: the stream has ended."""
    n, ends = case["streams"], int(case["streams"] * case["ended"])
    new = [1] * n if case["chunk"] == 1 else _spread(n, case["chunk"], 0)
    for i in range(ends):
        new[(i * 7 + 3) % n] = -1
    return _spread(n, case["history"], 0), new


def work(case):
    op = case["op"]
    if op == "plan":
        old, new = _plan_lists(case)
        p = case["page"]
        tokens = sum(max(x, 0) for x in new)
        fresh = sum(-(-(a + x) // p) - -(-a // p) for a, x in zip(old, new) if x > 0)
        back = sum(-(-a // p) for a, x in zip(old, new) if x < 0)
        # counts in and out, offsets, the slots; an entry of the list of free pages and one of the table for each page that changes hands
        return {"bytes": 4 * (4 * case["streams"] + tokens + 2 * fresh + 2 * back), "flops": 0}
    if op == "write":
        n = case["tokens"] * case["kv_heads"]
        return {"bytes": 2 * n * case["dim"] * (SIZE[case["type"]] + SIZE[case["cache"]]) + 4 * case["tokens"] + (8 * n if case["cache"] == "e4m3" else 0),
                "flops": 0}
    if op == "attend":
        n, q = sum(_kept(case)), case["streams"] * case["heads"]
        kv = 2 * n * case["kv_heads"] * (case["dim"] * SIZE[case["cache"]] + (4 if case["cache"] == "e4m3" else 0))
        return {"bytes": kv + 2 * q * case["dim"] * SIZE[case["type"]] + 4 * q + 4 * n // case["page"] + 4 * case["streams"],
                "flops": 4 * n * case["heads"] * case["dim"]}
    if op == "norm":
        n, s = case["rows"] * case["cols"], SIZE[case["type"]]
        out = (s if case["out"] != "e4m3" else 0) + (1 if case["out"] != "same" else 0)
        return {"bytes": n * (s + (2 * s if case["residual"] else 0) + out) + 4 * case["cols"] + (4 * case["rows"] if case["out"] != "same" else 0), "flops": 5 * n}
    blocks = -(-case["inputs"] // 32)
    rows = case["rows"] * (case["inputs"] * SIZE[case["type"]] + case["outputs"] * SIZE[case["out"]] + (4 if case["type"] == "e4m3" else 0))
    return {"bytes": case["outputs"] * blocks * 17 + rows, "flops": 2 * case["rows"] * case["outputs"] * case["inputs"]}


# ---------------------------------------------------------------------------
# inputs
# ---------------------------------------------------------------------------

_handle = None


def _rh():
    """The one context that a program holds (its own network is not part of these calls)."""
    global _handle
    if _handle is None:
        import numpy as np

        import workloads as wl
        from paper_2407_16990_amd import RH
        net = wl.Net("plain", 4, 2, 2)
        _handle = RH(frame_w=64, frame_h=64, max_frames=1, halo=2, bin_size=32, max_bins=4, net=net,
                     weights=np.asarray(wl.make_weights(net, 0, "fp32")), precision="fp32")
    return _handle


def _gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def _randn(g, *shape, dtype=torch.float32):
    return torch.randn(shape, generator=g, device="cuda", dtype=dtype)


def _i32(v):
    return torch.tensor(v, dtype=torch.int32, device="cuda")


def _paged(g, pages, case, zero=False):
    """One half of a cache: values [page][token][head][dim] in the case's order, and the scales [page][head][token] of an 8-bit one."""
    shape = (pages, case["page"], case["kv_heads"], case["dim"]) if case["order"] == "token" else (pages, case["kv_heads"], case["page"], case["dim"])
    kind, scale = case["cache"], None
    if zero:
        v = torch.zeros(shape, dtype=torch.uint8 if kind == "e4m3" else TYPES[kind], device="cuda")
        v = v.view(E4M3) if kind == "e4m3" else v
    elif kind == "e4m3":
        v = (_randn(g, *shape, dtype=torch.bfloat16) * 140.0).clamp_(-448.0, 448.0).to(E4M3)
    else:
        v = _randn(g, *shape, dtype=TYPES[kind])
    if kind == "e4m3":
        scale = torch.zeros((pages, case["kv_heads"], case["page"]), device="cuda") if zero else \
            torch.rand((pages, case["kv_heads"], case["page"]), generator=g, device="cuda") * 0.008 + 0.004
    return (v if case["order"] == "token" else v.transpose(1, 2)), scale


def prepare(case, seed):
    g, r, op = _gen(seed), random.Random(seed), case["op"]
    s = {"case": case, "rh": _rh() if own else None}
    if op == "plan":
        page, n = case["page"], case["streams"]
        both = list(zip(*_plan_lists(case)))
        r.shuffle(both)
        old, new = [a for a, _ in both], [x for _, x in both]
        have = [-(-a // page) for a in old]
        fresh = sum(-(-(a + x) // page) - h for a, x, h in zip(old, new, have) if x > 0)
        spare = int(fresh * case["room"]) + 1
        pages = sum(have) + spare
        width = -(-(case["history"] + case["chunk"]) // page)
        ids = torch.randperm(pages, generator=g, device="cuda").to(torch.int32)
        table = torch.full((n, width), -1, dtype=torch.int32, device="cuda")
        at = torch.arange(width, device="cuda")[None, :] < _i32(have)[:, None]
        table[at] = ids[: sum(have)]
        free = torch.full((pages,), -1, dtype=torch.int32, device="cuda")
        free[:spare] = ids[sum(have):]
        s.update(n_new=_i32(new), lengths=_i32(old), table=table, free=free, count=_i32([spare]), slots=max(1, sum(max(x, 0) for x in new)))
    elif op == "write":
        h, d, t = case["kv_heads"], case["dim"], case["tokens"]
        pages = -(-(t + t // 3 + 5) // case["page"])
        row = _randn(g, t, 4 * h * d, dtype=TYPES[case["type"]])        # the fused projection: 2*h heads of queries, keys, values
        s["k"], s["v"] = row[:, 2 * h * d:3 * h * d].view(t, h, d), row[:, 3 * h * d:].view(t, h, d)
        slots = torch.randperm(pages * case["page"], generator=g, device="cuda")[:t].to(torch.int32)
        slots[torch.arange(t, device="cuda") % 97 == 13] = -1           # tokens that got no room
        s.update(slots=slots, ck=_paged(g, pages, case, zero=True), cv=_paged(g, pages, case, zero=True))
    elif op == "attend":
        n, page, d = case["streams"], case["page"], case["dim"]
        lens = _lengths(case)
        r.shuffle(lens)
        have = [-(-a // page) for a in lens]
        pages = sum(have) + 1
        ids = torch.randperm(pages, generator=g, device="cuda").to(torch.int32)
        width = max(have)
        table = torch.full((n, width), -1, dtype=torch.int32, device="cuda")
        table[torch.arange(width, device="cuda")[None, :] < _i32(have)[:, None]] = ids[: sum(have)]
        row = _randn(g, n, (case["heads"] + 2 * case["kv_heads"]) * d, dtype=TYPES[case["type"]])
        s.update(q=row[:, : case["heads"] * d].view(n, case["heads"], d), table=table, lengths=_i32(lens), scale=2.0 / math.sqrt(d),
                 ck=_paged(g, pages, case), cv=_paged(g, pages, case))
    elif op == "norm":
        kind = TYPES[case["type"]]
        shape = (case["rows"], case["cols"])
        s["x"] = _randn(g, *shape, dtype=kind)
        s["residual"] = _randn(g, *shape, dtype=kind) * 2 if case["residual"] else None
        s["weight"] = 1.0 + 0.1 * _randn(g, case["cols"])
    else:
        n, k, kind = case["outputs"], case["inputs"], case["type"]
        blocks = -(-k // 32)
        w = torch.zeros((n, blocks * 32), device="cuda")
        w[:, :k] = _randn(g, n, k) / math.sqrt(k)
        w = w.view(n, blocks, 32)
        # weights laid out once: each block of 32 by the power of two that brings its largest to 4..8, nearest code
        e = torch.floor(torch.log2(w.abs().amax(-1).clamp_min(2.0 ** -100))) - 2
        mag = (w * torch.exp2(-e)[..., None]).abs()
        code = torch.bucketize(mag, torch.tensor([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0], device="cuda")).to(torch.uint8)
        code = (code + 8 * (w < 0).to(torch.uint8)).view(n, blocks * 32)
        s["w"] = code[:, 0::2] + 16 * code[:, 1::2]
        s["w_scale"] = (e + 127).to(torch.uint8)
        del w, mag, code
        x = _randn(g, case["rows"], k)
        if kind == "e4m3":
            s["x_scale"] = x.abs().amax(-1).clamp_min(1e-20) / 448.0
            s["x"] = (x / s["x_scale"][:, None]).to(E4M3)
        else:
            s["x_scale"], s["x"] = None, x.to(TYPES[kind])
    return s


# ---------------------------------------------------------------------------
# one pass
# ---------------------------------------------------------------------------

def run(s):
    case = s["case"]
    return (_run_own if own else _PLAIN[case["op"]])(s, case)


def _run_own(s, case):
    rh, op = s["rh"], case["op"]
    if op == "plan":
        slots, off, lengths, count = rh.cache_plan(s["n_new"], s["lengths"], s["table"], s["free"], s["count"], case["page"], s["slots"])
        return {"slots": slots, "off": off, "lengths": lengths, "count": count, "table": s["table"], "free": s["free"]}
    if op in ("write", "attend"):
        from paper_2407_16990_amd import KVCache
        cache = KVCache(s["ck"][0], s["cv"][0], s["ck"][1], s["cv"][1])
    if op == "write":
        rh.cache_write(cache, s["k"], s["v"], s["slots"])
        return {"k": cache.k, "v": cache.v, "k_scale": cache.k_scale, "v_scale": cache.v_scale}
    if op == "attend":
        out, lse = rh.cache_attend(s["q"], cache, s["table"], s["lengths"], scale=s["scale"], window=case["window"], want_lse=True)
        return {"out": out, "lse": lse}
    if op == "norm":
        total, y, y8, scale = rh.norm_residual(s["x"], s["weight"], s["residual"], eps=EPS, outputs=case["out"])
        return {"residual": total, "y": y, "y8": y8, "scale": scale}
    return rh.matvec_packed(s["x"], s["w"], s["w_scale"], x_scale=s["x_scale"], relu=case["relu"], out_dtype=TYPES[case["out"]])


def _plain_plan(s, case):
    n_new, old, page = s["n_new"].long(), s["lengths"].long(), case["page"]
    table, free, have, n = s["table"], s["free"], None, case["streams"]
    width, pages = table.shape[1], free.shape[0]
    have = (old + page - 1) // page
    ended = n_new < 0
    # pages of ended streams go on top of the list, streams in order, pages in order
    back = torch.where(ended, have, 0)
    first = torch.cumsum(back, 0) - back
    col = torch.arange(width, device="cuda")[None, :]
    gives = col < back[:, None]
    top = s["count"].long()
    free[(top + first[:, None] + col)[gives]] = table[gives]
    top = top + back.sum()
    # streams in order take pages while the running sums of what is asked for stay within the list and the slots
    need = torch.where(ended, 0, (old + n_new.clamp_min(0) + page - 1) // page - have)
    fits = ~ended & (have + need <= width)
    need, ask = torch.where(fits, need, 0), torch.where(fits, n_new, 0)
    upto, tokens = torch.cumsum(need, 0), torch.cumsum(ask, 0)
    ok = fits & ((need == 0) | (upto <= top)) & (tokens <= s["slots"])
    got, taken = torch.where(ok, ask, 0), torch.where(ok, need, 0)
    start = torch.cumsum(taken, 0) - taken
    k = col - have[:, None]
    takes = (k >= 0) & (k < taken[:, None])
    table[takes] = free[(top - 1 - start[:, None] - k)[takes]]
    off = torch.zeros(n + 1, dtype=torch.long, device="cuda")
    off[1:] = torch.cumsum(got, 0)
    i = torch.arange(s["slots"], device="cuda")
    b = torch.searchsorted(off[1:], i, right=True).clamp_max(n - 1)
    pos = old[b] + i - off[b]
    slot = table[b, (pos // page).clamp_max(width - 1)].long() * page + pos % page
    slots = torch.where(i < off[n], slot, -1).to(torch.int32)
    lengths = torch.where(ended, 0, old + got).to(torch.int32)
    return {"slots": slots, "off": off.to(torch.int32), "lengths": lengths, "count": (top - taken.sum()).to(torch.int32), "table": table, "free": free}


def _plain_write(s, case):
    page, quant = case["page"], case["cache"] == "e4m3"
    at = s["slots"].long()
    keep = at >= 0
    at = at[keep]
    out = {}
    for name, x, (v, scale) in (("k", s["k"], s["ck"]), ("v", s["v"], s["cv"])):
        x = x[keep].float()
        if quant:
            sc = x.abs().amax(-1).clamp_min(2.0 ** -100) / 448.0
            x = x / sc[..., None]
            scale[at // page, :, at % page] = sc
        if quant:
            v.view(torch.uint8)[at // page, at % page] = x.to(E4M3).view(torch.uint8)
        else:
            v[at // page, at % page] = x.to(v.dtype)
        out[name], out[name + "_scale"] = v, scale
    return out


def _plain_attend(s, case):
    page, h, d, n = case["page"], case["kv_heads"], case["dim"], case["streams"]
    pos = torch.arange(s["table"].shape[1] * page, device="cuda")
    length = s["lengths"].long()[:, None]
    begin = (length - case["window"]).clamp_min(0) if case["window"] else torch.zeros_like(length)
    keep = (pos[None, :] >= begin) & (pos[None, :] < length)
    pages = s["table"].long().clamp_min(0)

    def gathered(v, scale):
        x = v[pages] if scale is None else v.view(torch.uint8)[pages].view(E4M3)
        x = x.reshape(n, -1, h, d).float()
        if scale is not None:
            x = x * scale[pages].transpose(2, 3).reshape(n, -1, h)[..., None]
        return torch.where(keep[:, :, None, None], x, 0.0).transpose(1, 2).contiguous()

    q = s["q"].float().reshape(n, h, -1, d)
    score = torch.matmul(q, gathered(*s["ck"]).transpose(2, 3).contiguous()) * s["scale"]
    score = torch.where(keep[:, None, None, :], score, float("-inf"))
    top = score.amax(-1, keepdim=True)
    p = torch.exp(score - torch.where(torch.isinf(top), 0.0, top))
    total = p.sum(-1, keepdim=True)
    out = torch.matmul(p, gathered(*s["cv"])) / torch.where(total > 0, total, 1.0)
    lse = torch.where(total > 0, top + torch.log(total), float("-inf"))
    return {"out": out.reshape(n, -1, d).to(s["q"].dtype), "lse": lse.reshape(n, -1)}


def _plain_norm(s, case):
    x, kind = s["x"].float(), s["x"].dtype
    got = {"residual": None, "y": None, "y8": None, "scale": None}
    if s["residual"] is not None:
        x = x + s["residual"].float()
        got["residual"] = x.to(kind)
    y = x * torch.rsqrt((x * x).mean(-1, keepdim=True) + EPS) * s["weight"]
    if case["out"] != "e4m3":
        got["y"] = y.to(kind)
    if case["out"] != "same":
        got["scale"] = y.abs().amax(-1).clamp_min(2.0 ** -100) / 448.0
        got["y8"] = (y / got["scale"][:, None]).to(E4M3)
    return got


def _plain_matvec(s, case):
    n, blocks = s["w_scale"].shape
    table = torch.tensor(FP4 + tuple(-v for v in FP4), device="cuda")
    code = torch.stack((s["w"] & 15, s["w"] >> 4), -1).view(n, blocks, 32)
    w = (table[code.int()] * torch.exp2(s["w_scale"].float() - 127)[..., None]).view(n, blocks * 32)[:, : case["inputs"]]
    y = torch.matmul(s["x"].float(), w.t())
    if s["x_scale"] is not None:
        y = y * s["x_scale"][:, None]
    return (torch.relu(y) if case["relu"] else y).to(TYPES[case["out"]])


_PLAIN = {"plan": _plain_plan, "write": _plain_write, "attend": _plain_attend, "norm": _plain_norm, "matvec": _plain_matvec}


# ---------------------------------------------------------------------------
# the definitions in 64 bits
# ---------------------------------------------------------------------------

def exact(case, seed):
    op = case["op"]
    s = prepare(case, seed)
    if op == "plan":
        return None
    if op == "write":
        got = {}
        slot = s["slots"].cpu().tolist()
        rows = torch.tensor([i for i, a in enumerate(slot) if a >= 0], device="cuda", dtype=torch.long)
        page = torch.tensor([a // case["page"] for a in slot if a >= 0], device="cuda", dtype=torch.long)
        line = torch.tensor([a % case["page"] for a in slot if a >= 0], device="cuda", dtype=torch.long)
        for name, x, (v, scale) in (("k", s["k"], s["ck"]), ("v", s["v"], s["cv"])):
            x = x.double()[rows]
            dense = torch.zeros(v.shape, dtype=torch.float64, device="cuda")
            got[name + "_scale"] = None
            if scale is not None:
                most = torch.linalg.vector_norm(x, float("inf"), dim=-1)
                most = torch.maximum(most, torch.full_like(most, 2.0 ** -100)) / 448
                x = x / most.unsqueeze(-1)
                got[name + "_scale"] = torch.zeros(scale.shape, dtype=torch.float64, device="cuda")
                got[name + "_scale"].permute(0, 2, 1)[page, line] = most
            dense[page, line] = x
            got[name] = dense
        return got
    if op == "attend":
        heads, h, d = case["heads"], case["kv_heads"], case["dim"]
        lens = s["lengths"].cpu().tolist()
        out = torch.zeros((len(lens), heads, d), dtype=torch.float64, device="cuda")
        lse = torch.full((len(lens), heads), float("-inf"), dtype=torch.float64, device="cuda")
        for b, n in enumerate(lens):
            if n == 0:
                continue
            lo = max(0, n - case["window"]) if case["window"] else 0
            at = torch.arange(lo, n, device="cuda")
            page, line = s["table"][b].long()[at // case["page"]], at % case["page"]
            for j in range(h):
                both = []
                for v, scale in (s["ck"], s["cv"]):
                    x = (v[page, line, j] if scale is None else v.view(torch.uint8)[page, line, j].view(E4M3)).double()
                    both.append(x if scale is None else x * scale[page, j, line].double()[:, None])
                q = s["q"][b, j * (heads // h):(j + 1) * (heads // h)].double()
                score = (both[0] @ q.t()).t() * s["scale"]
                lse[b, j * (heads // h):(j + 1) * (heads // h)] = torch.logsumexp(score, -1)
                out[b, j * (heads // h):(j + 1) * (heads // h)] = torch.softmax(score, -1) @ both[1]
        return {"out": out, "lse": lse}
    if op == "norm":
        x = s["x"].double()
        got = {"residual": None, "y": None, "y8": None, "scale": None}
        if case["residual"]:
            x = x + s["residual"].double()
            got["residual"] = x
        y = x / (torch.linalg.vector_norm(x, dim=-1, keepdim=True) ** 2 / case["cols"] + EPS).sqrt() * s["weight"].double()
        if case["out"] in ("same", "both"):
            got["y"] = y
        if case["out"] in ("e4m3", "both"):
            most = torch.linalg.vector_norm(y, float("inf"), dim=-1) / 448
            got["scale"] = torch.maximum(most, torch.full_like(most, 2.0 ** -100 / 448))
            got["y8"] = y / got["scale"].unsqueeze(-1)
        return got
    low, high = (s["w"] % 16).long(), (s["w"] // 16).long()
    code = torch.empty((case["outputs"], 2 * low.shape[1]), dtype=torch.long, device="cuda")
    code[:, ::2], code[:, 1::2] = low, high
    mag, e = code % 8, s["w_scale"].double() - 127
    # codes 0 and 1 stand for 0 and 1/2; above, two codes a power of two
    value = torch.where(mag < 2, mag * 0.5, (1 + 0.5 * (mag % 2)) * torch.pow(2.0, (mag // 2 - 1).double()))
    value = torch.where(code >= 8, -value, value.double()) * torch.pow(2.0, e).repeat_interleave(32, 1)
    x = s["x"].double() * (1 if s["x_scale"] is None else s["x_scale"].double()[:, None])
    y = x @ value[:, : case["inputs"]].t().contiguous()
    return y.clamp_min(0) if case["relu"] else y
