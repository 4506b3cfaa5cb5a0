"""The operators of a state-space layer over many live streams, as cases: inputs, one pass, and what a pass cannot do without.

A predictor of macroblock scores that remembers a stream's past in a state of fixed size, in place of a cache that grows with every
frame, runs these: a short causal convolution along the tokens of each stream, a selective scan that carries the stream's state, and a
gated norm whose 8-bit rows go into the next product.  Tokens are frames of a stream, or the macroblocks of one.

Kinds of case
  conv   RH.state_conv: depthwise causal convolution with SiLU; the last inputs of every stream kept in a pool of states
  scan   RH.state_scan: h = exp(delta a) h + delta x b, y = c.h + skip x, times SiLU(gate); h kept in a pool of states
  norm   RH.norm_gated: root-mean-square norm of x * SiLU(gate) over groups of channels, output also in 8 bits

A stream has one token a call where frames arrive live, and many where a chunk of frames, or the macroblocks of one, joins at once: 510 macroblocks for
480 x 272, 920 for 640 x 368, 8 streams, 16 or 30 frames a chunk (workloads/).  Widths are generic.
"""
import math
import random

import torch

own = False

E4M3 = torch.float8_e4m3fn
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
SIZE = {"f32": 4, "bf16": 2}
EPS = 1e-6


def listed():
    return [
        # a frame of each of 8 live streams arrives: nothing but latency
        {"name": "conv_8x1_bf16", "op": "conv", "streams": 8, "longest": 1, "even": True, "channels": 1024, "width": 4, "type": "bf16"},
        # the macroblocks of a frame of each of 30 streams, out of the fused projection's rows
        {"name": "conv_30x920_bf16", "op": "conv", "streams": 30, "longest": 920, "even": True, "channels": 2048, "width": 4, "type": "bf16"},
        # chunks of very different lengths, a width that no vector divides
        {"name": "conv_37x1500_f32", "op": "conv", "streams": 37, "longest": 1500, "even": False, "channels": 515, "width": 3, "type": "f32"},
        # 8 live streams, a small predictor
        {"name": "scan_8x1_bf16", "op": "scan", "streams": 8, "longest": 1, "even": True, "channels": 1024, "n": 16, "groups": 1, "type": "bf16", "gate": True},
        # 512 live streams, a wide one: every state read and written
        {"name": "scan_512x1_bf16", "op": "scan", "streams": 512, "longest": 1, "even": True, "channels": 4096, "n": 16, "groups": 1, "type": "bf16", "gate": True},
        # one stream's past of nine minutes taken in at once: all the work is along one axis
        {"name": "scan_1x16384_bf16", "op": "scan", "streams": 1, "longest": 16384, "even": True, "channels": 1024, "n": 16, "groups": 1, "type": "bf16", "gate": True},
        # the macroblocks of a frame of each of 30 streams: the ordinary large call
        {"name": "scan_30x920_bf16", "op": "scan", "streams": 30, "longest": 920, "even": True, "channels": 2048, "n": 16, "groups": 1, "type": "bf16", "gate": True},
        # chunks of very different lengths, odd widths, no gate
        {"name": "scan_37x2000_f32", "op": "scan", "streams": 37, "longest": 2000, "even": False, "channels": 522, "n": 13, "groups": 2, "type": "f32", "gate": False},
        # a larger state in groups: 64 streams with up to ten seconds of frames
        {"name": "scan_64x300_n64", "op": "scan", "streams": 64, "longest": 300, "even": False, "channels": 512, "n": 64, "groups": 4, "type": "bf16", "gate": True},
        # a row a stream, 8-bit rows for the next product
        {"name": "norm_8x2048_bf16", "op": "norm", "rows": 8, "cols": 2048, "groups": 8, "type": "bf16", "out": "e4m3"},
        # the macroblocks of a frame of each of 30 streams, both outputs
        {"name": "norm_27600x2048_bf16", "op": "norm", "rows": 27600, "cols": 2048, "groups": 8, "type": "bf16", "out": "both"},
        # 16 frames of 920 macroblocks, groups of an odd width
        {"name": "norm_14720x1540_f32", "op": "norm", "rows": 14720, "cols": 1540, "groups": 4, "type": "f32", "out": "same"},
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng: random.Random):
    most = max(work(c)["bytes"] for c in listed())
    most_updates = 27600 * 2048 * 16
    while True:
        op = rng.choice(("conv", "scan", "scan", "scan", "norm"))
        c = {"op": op}
        if op == "norm":
            g = rng.choice((1, 1, 2, 3, 4, 8, 16))
            per = rng.choice((_log(rng, 1, 2048), 64 * rng.randint(1, 32)))
            c.update(rows=_log(rng, 1, 32768), cols=g * per, groups=g, type=rng.choice(("f32", "bf16")), out=rng.choice(("same", "e4m3", "both")))
        else:
            one = rng.random() < 0.4
            c.update(streams=_log(rng, 1, 1024 if one else 128), longest=1 if one else _log(rng, 2, 16384), even=one or rng.random() < 0.4,
                     channels=rng.choice((_log(rng, 1, 8192), 64 * rng.randint(1, 64))))
            if op == "conv":
                c.update(width=rng.randint(2, 5), type=rng.choice(("f32", "bf16")))
            else:
                g = rng.choice((1, 1, 2, 4, 8))
                c["channels"] = max(1, c["channels"] // g) * g
                c.update(n=rng.choice((4, 8, 16, 16, 16, 32, 64, 128, rng.randint(1, 128))), groups=g, type=rng.choice(("f32", "bf16", "bf16")), gate=rng.random() < 0.7)
                if sum(_lengths(c)) * c["channels"] * c["n"] > most_updates:
                    continue
        if work(c)["bytes"] <= most:
            return c


def _lengths(case):
    """Tokens of every stream in this call: the largest first, then one, a stream that has none, the others spread evenly."""
    n, most = case["streams"], case["longest"]
    if case["even"]:
        return [most] * n
    return [most if i == 0 else 1 if i == 1 else 0 if i == 2 else 1 + int((most - 1) * ((i * 0.6180339887498949) % 1.0)) for i in range(n)]


def work(case):
    s = SIZE[case["type"]]
    if case["op"] == "norm":
        n = case["rows"] * case["cols"]
        out = (s if case["out"] != "e4m3" else 0) + (1 if case["out"] != "same" else 0)
        return {"bytes": n * (2 * s + out) + 4 * case["cols"] + (4 * case["rows"] if case["out"] != "same" else 0), "flops": 9 * n}
    rows, d, b = sum(_lengths(case)), case["channels"], case["streams"]
    if case["op"] == "conv":
        w = case["width"]
        return {"bytes": 2 * rows * d * s + 2 * b * (w - 1) * d * s + 4 * d * (w + 1) + 16 * b, "flops": rows * d * (2 * w + 4)}
    n = case["n"]
    return {"bytes": rows * (d * s * (4 if case["gate"] else 3) + 2 * case["groups"] * n * s) + 2 * b * d * n * 4 + 4 * d * (n + 2) + 16 * b, "flops": rows * d * (7 * n + 12)}


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


def _randn(g, *shape, dtype=torch.float32):
    return torch.randn(shape, generator=g, device="cuda", dtype=dtype)


def _i32(v):
    return torch.tensor(v, dtype=torch.int32, device="cuda")


def prepare(case, seed):
    g, r, op, kind = torch.Generator(device="cuda").manual_seed(seed), random.Random(seed), case["op"], TYPES[case["type"]]
    s = {"case": case, "rh": _rh() if own else None}
    if op == "norm":
        rows, d = case["rows"], case["cols"]
        both = _randn(g, rows, 2 * d, dtype=kind)                       # the fused projection's rows: half of them the gate
        s.update(x=_randn(g, rows, d, dtype=kind), gate=both[:, d:], weight=1.0 + 0.1 * _randn(g, d))
        return s
    lens, d, streams = _lengths(case), case["channels"], case["streams"]
    r.shuffle(lens)
    off = [0]
    for n in lens:
        off.append(off[-1] + n)
    rows = off[-1]
    places = r.sample(range(2 * streams + 3), 2 * streams)              # a stream's state before and after: the one before is kept
    s.update(off=None if case["longest"] == 1 and case["even"] else _i32(off), slots=_i32(places[:streams]), into=_i32(places[streams:]),
             past=_i32([0 if r.random() < 0.2 else r.randint(1, 100000) for _ in lens]), lens=lens, begins=off, pool=2 * streams + 3)
    row = _randn(g, rows, 2 * d, dtype=kind)
    s["x"], s["gate"] = row[:, :d], row[:, d:]
    if op == "conv":
        w = case["width"]
        s.update(weight=_randn(g, w, d) / math.sqrt(w), bias=0.1 * _randn(g, d), state=_randn(g, s["pool"], w - 1, d, dtype=kind))
        return s
    n, k = case["n"], case["groups"]
    bc = _randn(g, rows, 2 * k * n, dtype=kind)
    step = torch.exp(torch.rand(d, generator=g, device="cuda") * math.log(100.0) + math.log(0.001))     # steps of 0.001 to 0.1
    s.update(dt=_randn(g, rows, d, dtype=kind) * 0.5, b=bc[:, :k * n].unflatten(1, (k, n)), c=bc[:, k * n:].unflatten(1, (k, n)),
             a=-torch.exp(torch.rand((d, n), generator=g, device="cuda") * math.log(16.0)), dt_bias=step + torch.log(-torch.expm1(-step)),
             skip=1.0 + 0.1 * _randn(g, d), state=_randn(g, s["pool"], d, n))
    if not case["gate"]:
        s["gate"] = None
    return s


# ---------------------------------------------------------------------------
# one pass
# ---------------------------------------------------------------------------

def run(s):
    case = s["case"]
    return (_run_own if own else _PLAIN[case["op"]])(s, case)


def _run_own(s, case):
    rh = s["rh"]
    if case["op"] == "norm":
        y, y8, scale = rh.norm_gated(s["x"], s["gate"], s["weight"], groups=case["groups"], eps=EPS, outputs=case["out"])
        return {"y": y, "y8": y8, "scale": scale}
    if case["op"] == "conv":
        out = rh.state_conv(s["x"], s["weight"], s["state"], s["slots"], bias=s["bias"], offsets=s["off"], past=s["past"], into=s["into"])
    else:
        out = rh.state_scan(s["x"], s["dt"], s["a"], s["b"], s["c"], s["state"], s["slots"], skip=s["skip"], gate=s["gate"], dt_bias=s["dt_bias"],
                            offsets=s["off"], past=s["past"], into=s["into"])
    return {"out": out, "state": s["state"]}


def _rows(s):
    """(stream of every row, first row of every stream, rows of every stream)."""
    streams, rows = s["slots"].shape[0], s["x"].shape[0]
    if s["off"] is None:
        at = torch.arange(rows, device="cuda")
        return at, at, torch.ones_like(at)
    off = s["off"].long()
    return torch.searchsorted(off[1:].contiguous(), torch.arange(rows, device="cuda"), right=True).clamp_max(streams - 1), off[:-1], off[1:] - off[:-1]


def _plain_conv(s, case):
    x, w, state, wide = s["x"].float(), s["weight"], s["state"], case["width"]
    stream, first, count = _rows(s)
    before = torch.where((s["past"] > 0)[:, None, None], state[s["slots"].long()].float(), 0.0)
    place = torch.arange(x.shape[0], device="cuda") - first[stream]
    j = torch.arange(wide, device="cuda") - (wide - 1)
    back = place[:, None] + j[None, :]                                  # below 0: in the state
    at = (first[stream][:, None] + back.clamp_min(0)).clamp_max(x.shape[0] - 1)
    y = s["bias"].expand(x.shape).clone()
    taken = torch.where((back >= 0)[..., None], x[at], before[stream[:, None], (back + wide - 1).clamp_max(wide - 2)])
    y = y + (taken * w[None]).sum(1)
    # the last inputs: of the state what is left of them
    ends = count[:, None] + torch.arange(wide - 1, device="cuda")[None, :] - (wide - 1)
    new = torch.where((ends >= 0)[..., None], x[(first[:, None] + ends.clamp_min(0)).clamp_max(x.shape[0] - 1)],
                      torch.gather(before, 1, (ends + wide - 1).clamp_max(wide - 2)[..., None].expand(-1, -1, x.shape[1])))
    has = count > 0
    state[s["into"].long()[has]] = new[has].to(state.dtype)
    return {"out": (y / (1.0 + torch.exp(-y))).to(s["x"].dtype), "state": state}


def _plain_scan(s, case):
    d, n, k, state = case["channels"], case["n"], case["groups"], s["state"]
    x, dt = s["x"].float(), s["dt"].float() + s["dt_bias"]
    rows = x.shape[0]
    stream, first, count = _rows(s)
    dt = torch.where(dt > 20.0, dt, torch.log1p(torch.exp(dt.clamp_max(20.0))))
    before = torch.where((s["past"] > 0)[:, None, None], state[s["slots"].long()], 0.0)
    spread = (lambda v: v.float()[:, :, None, :].expand(rows, k, d // k, n).reshape(rows, d, n))  # noqa: E731
    fade = torch.exp(dt[..., None] * s["a"])
    h = (dt * x)[..., None] * spread(s["b"])
    has = count > 0
    begin = first[has]
    h[begin] += fade[begin] * before[has]
    # rows t and t - reach, with reach doubled each time; a stream's first row has nothing before it
    fade[begin] = 0.0
    reach = 1
    while reach < case["longest"]:
        h[reach:] += fade[reach:] * h[:-reach].clone()
        fade = torch.cat((fade[:reach], fade[reach:] * fade[:-reach]))
        reach *= 2
    y = (h * spread(s["c"])).sum(-1) + s["skip"] * x
    if s["gate"] is not None:
        z = s["gate"].float()
        y = y * z / (1.0 + torch.exp(-z))
    state[s["into"].long()[has]] = h[(first + count - 1)[has]]
    return {"out": y.to(s["x"].dtype), "state": state}


def _plain_norm(s, case):
    x, z, kind = s["x"].float(), s["gate"].float(), s["x"].dtype
    x = x * z / (1.0 + torch.exp(-z))
    parts = x.unflatten(1, (case["groups"], -1))
    y = (parts * torch.rsqrt((parts * parts).mean(-1, keepdim=True) + EPS)).flatten(1) * s["weight"]
    got = {"y": None, "y8": None, "scale": None}
    if case["out"] != "e4m3":
        got["y"] = y.to(kind)
    if case["out"] != "same":
        got["scale"] = y.abs().amax(-1).clamp_min(2.0 ** -100) / 448.0
        got["y8"] = (y / got["scale"][:, None]).to(E4M3)
    return got


_PLAIN = {"conv": _plain_conv, "scan": _plain_scan, "norm": _plain_norm}


# ---------------------------------------------------------------------------
# the definitions in 64 bits
# ---------------------------------------------------------------------------

def exact(case, seed):
    s, op = prepare(case, seed), case["op"]
    if op == "norm":
        z = s["gate"].double()
        x = s["x"].double() * z * torch.sigmoid(z)
        got = {"y": None, "y8": None, "scale": None}
        y = torch.empty_like(x)
        per = case["cols"] // case["groups"]
        for g in range(0, case["cols"], per):
            part = x[:, g:g + per]
            y[:, g:g + per] = part / (torch.linalg.vector_norm(part, dim=-1, keepdim=True) ** 2 / per + EPS).sqrt() * s["weight"].double()[g:g + per]
        if case["out"] in ("same", "both"):
            got["y"] = y
        if case["out"] in ("e4m3", "both"):
            most = torch.linalg.vector_norm(y, float("inf"), dim=-1)
            got["scale"] = torch.maximum(most, torch.full_like(most, 2.0 ** -100)) / 448
            got["y8"] = y / got["scale"].unsqueeze(-1)
        return got
    x, slots, into, past = s["x"].double(), s["slots"].tolist(), s["into"].tolist(), s["past"].tolist()
    pool, out = s["state"].double(), torch.zeros(x.shape, dtype=torch.float64, device="cuda")
    if op == "conv":
        w, bias, wide = s["weight"].double(), s["bias"].double(), case["width"]
        old = pool.clone()
        if case["longest"] == 1:                                        # a row a stream
            keep = torch.tensor([p > 0 for p in past], device="cuda", dtype=torch.float64)[:, None, None]
            line = torch.cat((old[slots] * keep, x[:, None]), 1)
            y = bias + torch.einsum("bjd,jd->bd", line, w)
            pool[into] = line[:, 1:]
            return {"out": y * torch.sigmoid(y), "state": pool}
        for b, n in enumerate(s["lens"]):
            if n == 0:
                continue
            lo = s["begins"][b]
            line = torch.cat((old[slots[b]] if past[b] > 0 else torch.zeros_like(old[0]), x[lo:lo + n]))
            y = bias + (line.unfold(0, wide, 1) * w.t()).sum(-1)
            out[lo:lo + n] = y * torch.sigmoid(y)
            pool[into[b]] = line[n:]
        return {"out": out, "state": pool}
    step = torch.nn.functional.softplus(s["dt"].double() + s["dt_bias"].double(), threshold=700)
    a, b, c, skip = s["a"].double(), s["b"].double(), s["c"].double(), s["skip"].double()
    per = case["channels"] // case["groups"]
    h = pool[slots]
    for i, p in enumerate(past):
        if p <= 0:
            h[i] = 0
    lens, begins = torch.tensor(s["lens"], device="cuda"), torch.tensor(s["begins"][:-1], device="cuda")
    order = sorted(range(len(past)), key=lambda i: -s["lens"][i])       # the longest first: those that have a t-th token come in front
    h, begins = h[order], begins[order]
    sizes = [s["lens"][i] for i in order]
    live = len(order)
    for t in range(sizes[0]):
        while sizes[live - 1] <= t:
            live -= 1
        at = begins[:live] + t
        now = step[at]
        new = torch.exp(now[..., None] * a) * h[:live] + (now * x[at])[..., None] * b[at].repeat_interleave(per, 1)
        h[:live] = new
        out[at] = (new * c[at].repeat_interleave(per, 1)).sum(-1)
    out += skip * x
    if s["gate"] is not None:
        z = s["gate"].double()
        out *= z * torch.sigmoid(z)
    for i, b_ in enumerate(order):
        if s["lens"][b_] > 0:
            pool[into[b_]] = h[i]
    return {"out": out, "state": pool}
