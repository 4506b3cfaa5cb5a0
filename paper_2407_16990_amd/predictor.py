"""Macroblock importance for live streams, a frame of every stream at a time: a small network that remembers each stream's past, a
transformer in a paged key-value cache or a state-space model in a state of fixed size, on the operators of include/rh_seq.h.  Its scores are what select_regions takes.

One token stands for one frame of one stream: its input is a vector of codec features of the frame's macroblocks (what tells
one frame's place in time from another's has to be among them), its output one score per macroblock.  A layer is
    norm -> queries, keys, values -> attention over the stream's frames -> projection -> residual
    norm -> widening product, ReLU -> narrowing product -> residual
with weights in 4 bits, the residual stream in bf16, and the norms' outputs in 8 bits.  With the mixer "state" attention's place is taken by
    norm -> x and gate -> causal convolution of x -> steps, b and c -> selective scan over the stream's frames -> gated norm -> projection -> residual
which takes the same time and memory however long a stream gets, and many frames of a stream in one call (chunk).

    python -m paper_2407_16990_amd.predictor [--mixer state]       # eight streams through predictor, selection, packing, enhancement and paste
"""
from __future__ import annotations

import argparse
from dataclasses import dataclass

import numpy as np
import torch

from .binding import RH, KVCache, pack_weights


@dataclass(frozen=True)
class PredictorConfig:
    mbw: int                    # macroblock grid of a frame
    mbh: int
    n_features: int             # length of a frame's input vector
    max_streams: int
    hidden: int = 512
    layers: int = 2
    q_heads: int = 8
    kv_heads: int = 2
    dim: int = 64
    widened: int = 2048
    page: int = 16              # frames a page of the cache
    n_pages: int = 4096         # of all streams together
    max_pages: int = 512        # of one stream
    window: int = 0             # frames that attention looks back; 0: all.  Pages behind it are given back, so that a stream goes on for ever where
                                # window + page <= max_pages * page; without a window it has room for max_pages * page frames
    eps: float = 1e-6
    cache_dtype: torch.dtype = torch.bfloat16      # or torch.float8_e4m3fn
    mixer: str = "attention"    # or "state", for which the following count, and of the above neither heads nor what is said of cache, pages and window
    inner: int = 1024           # channels of a state layer
    states: int = 16            # of a channel
    taps: int = 4               # frames that its convolution sees
    groups: int = 8             # of channels, normed apart


_SMALL = ("conv", "a_log")      # matrices that are no products


def weight_shapes(cfg: PredictorConfig) -> dict:
    """Names and shapes of the float weights: [outputs, inputs] of the products, vectors of the norms; of a state layer also
    conv [taps, inner] and conv_bias, dt_bias and skip [inner], a_log [inner, states] with a = -exp(a_log)."""
    h, heads, d, n = cfg.hidden, cfg.q_heads + 2 * cfg.kv_heads, cfg.inner, cfg.states
    shapes = {"in": (h, cfg.n_features), "norm_out": (h,), "out": (cfg.mbw * cfg.mbh, h)}
    for i in range(cfg.layers):
        shapes |= {f"norm_a{i}": (h,)}
        if cfg.mixer == "state":
            shapes |= {f"gate{i}": (2 * d, h), f"conv{i}": (cfg.taps, d), f"conv_bias{i}": (d,), f"select{i}": (d + 2 * n, d), f"dt_bias{i}": (d,), f"a_log{i}": (d, n),
                       f"skip{i}": (d,), f"norm_s{i}": (d,), f"proj{i}": (h, d)}
        else:
            shapes |= {f"qkv{i}": (heads * cfg.dim, h), f"proj{i}": (h, cfg.q_heads * cfg.dim)}
        shapes |= {f"norm_b{i}": (h,), f"wide{i}": (cfg.widened, h), f"narrow{i}": (h, cfg.widened)}
    return shapes


def random_weights(cfg: PredictorConfig, seed: int) -> dict:
    """Weights of that architecture, drawn: products keep the scale of their input, norms near one; steps of 0.001 to 0.1, fading by 1 to 16 times that."""
    rng = np.random.default_rng(seed)

    def draw(name, s):
        kind = name.rstrip("0123456789")
        if kind == "a_log":
            return np.log(rng.uniform(1, 16, s))
        if kind == "dt_bias":
            step = np.exp(rng.uniform(np.log(0.001), np.log(0.1), s))
            return step + np.log(-np.expm1(-step))
        if kind == "conv_bias":
            return 0.1 * rng.standard_normal(s)
        if kind == "conv":
            return rng.standard_normal(s) / np.sqrt(s[0])
        return 1 + 0.1 * rng.standard_normal(s) if len(s) == 1 else rng.standard_normal(s) / np.sqrt(s[1])
    return {name: draw(name, s).astype(np.float32) for name, s in weight_shapes(cfg).items()}


class StreamPredictor:
    """The state of max_streams streams and the step that takes one frame of each.  rh: the context whose stream the work goes
    on, and which is to be torch's current one; other calls of that context must not overlap with a step on another stream, replays included.
    graph: record the step at its second call and replay it from then on (one launch instead of one per operator).
    lengths: frames of each stream that found room since it began (with the mixer "state" every frame does); granted: which streams' frames did in the last step or chunk."""

    def __init__(self, rh: RH, cfg: PredictorConfig, weights: dict, graph: bool = False):
        self.rh, self.cfg, dev = rh, cfg, rh.device
        if cfg.mixer not in ("attention", "state"):
            raise ValueError(f"mixer {cfg.mixer!r}: \"attention\" or \"state\"")
        if cfg.mixer == "state" and (cfg.groups < 1 or cfg.inner % cfg.groups):
            raise ValueError(f"groups {cfg.groups}: they divide inner, {cfg.inner}")
        if cfg.cache_dtype not in (torch.bfloat16, torch.float8_e4m3fn):
            raise ValueError(f"cache_dtype {cfg.cache_dtype}: keys and values are bf16, the cache torch.bfloat16 or torch.float8_e4m3fn")
        for name, shape in weight_shapes(cfg).items():
            if tuple(weights[name].shape) != shape:
                raise ValueError(f"{name}: {tuple(weights[name].shape)}, not {shape}")
        put = lambda a: torch.from_numpy(np.ascontiguousarray(a)).to(dev)  # noqa: E731
        small = lambda n, w: w.ndim == 1 or n.rstrip("0123456789") in _SMALL  # noqa: E731
        self.norms = {n: put(np.asarray(w, dtype=np.float32)) for n, w in weights.items() if small(n, w)}
        self.packed = {n: tuple(put(a) for a in pack_weights(w)) for n, w in weights.items() if not small(n, w)}
        n = cfg.max_streams
        i32 = dict(dtype=torch.int32, device=dev)
        self.lengths = torch.zeros(n, **i32)
        if cfg.mixer == "state":
            # streams' states; what they hold of a stream that has not begun does not matter
            self.states = [(torch.zeros((n, cfg.taps - 1, cfg.inner), dtype=torch.bfloat16, device=dev), torch.zeros((n, cfg.inner, cfg.states), device=dev)) for _ in range(cfg.layers)]
            self.fade = [-torch.exp(self.norms[f"a_log{i}"]) for i in range(cfg.layers)]
            self.every = torch.arange(n, **i32)
        else:
            self._make_caches(dev, i32)
        self.features, self.n_new = torch.zeros((n, cfg.n_features), device=dev), torch.zeros(n, **i32)
        self.want_graph, self.graph, self.outputs, self.calls, self.granted = graph, None, None, 0, None

    def _make_caches(self, dev, i32):
        cfg, n = self.cfg, self.cfg.max_streams
        shape = (cfg.n_pages, cfg.kv_heads, cfg.page, cfg.dim)
        quantised = cfg.cache_dtype == torch.float8_e4m3fn

        def cache():
            kv = [torch.zeros(shape, dtype=torch.uint8, device=dev).view(cfg.cache_dtype) if quantised else
                  torch.zeros(shape, dtype=cfg.cache_dtype, device=dev) for _ in range(2)]
            scales = [torch.zeros(shape[:3], device=dev) if quantised else None for _ in range(2)]
            return KVCache(kv[0].transpose(1, 2), kv[1].transpose(1, 2), *scales)
        self.caches = [cache() for _ in range(cfg.layers)]
        self.table = torch.full((n, cfg.max_pages), -1, **i32)
        # frames in the cache: fewer than a stream has had once pages behind the window are given back
        self.held, self.ended = (torch.zeros(n, **i32), torch.full((n,), -1, **i32)) if cfg.window else (self.lengths, None)
        self.free, self.free_count = torch.arange(cfg.n_pages, **i32), torch.full((1,), cfg.n_pages, **i32)

    def _product(self, name, x, x_scale=None, **kw):
        return self.rh.matvec_packed(x, *self.packed[name], x_scale=x_scale, **kw)

    def _step(self):
        cfg, n = self.cfg, self.cfg.max_streams
        self.n_new.clamp_(-1, 1)                                   # a step has one row a stream: no room is planned for more than it writes
        if cfg.mixer == "state":
            granted = self.n_new > 0
            # a stream without a frame in this step has a row, but keeps its states
            scores = self._layers(self.features, self._state, torch.where(granted, self.every, torch.full_like(self.every, -1)), None)
            self.lengths.add_(granted).masked_fill_(self.n_new < 0, 0)
            return scores, granted
        if cfg.window:
            self._give_back()
        slots, off, _, _ = self.rh.cache_plan(self.n_new, self.held, self.table, self.free, self.free_count, cfg.page, n,
                                              new_lengths=self.held, new_count=self.free_count)
        granted = off[1:] > off[:-1]
        if cfg.window:
            self.lengths.add_(granted).masked_fill_(self.n_new < 0, 0)
        # the plan lists tokens, the rows below are streams: a stream without a token in this step writes nothing
        mine = slots[off[:-1].clamp_max(n - 1).long()]
        return self._layers(self.features, self._attention, torch.where(granted, mine, torch.full_like(mine, -1))), granted

    def _layers(self, features, mix, *args):
        """The network on rows of features; mix: what takes a layer's normed rows to those ahead of its projection."""
        cfg = self.cfg
        x = self._product("in", features, out_dtype=torch.bfloat16)
        h = None
        for i in range(cfg.layers):
            h, _, y, ys = self._norm(f"norm_a{i}", x, h)
            x = self._product(f"proj{i}", *mix(i, y, ys, *args))
            h, _, y, ys = self._norm(f"norm_b{i}", x, h)
            x = self._product(f"narrow{i}", self._product(f"wide{i}", y, ys, relu=True))
        _, _, y, ys = self._norm("norm_out", x, h)
        return self._product("out", y, ys, out_dtype=torch.float32).view(-1, cfg.mbh, cfg.mbw)

    def _attention(self, i, y, ys, slots):
        rh, cfg, cache = self.rh, self.cfg, self.caches[i]
        hq, hk, d = cfg.q_heads, cfg.kv_heads, cfg.dim
        row = self._product(f"qkv{i}", y, ys)
        rh.cache_write(cache, row[:, hq * d:(hq + hk) * d].unflatten(1, (hk, d)), row[:, (hq + hk) * d:].unflatten(1, (hk, d)), slots)
        return rh.cache_attend(row[:, : hq * d].unflatten(1, (hq, d)), cache, self.table, self.held, window=cfg.window).view(-1, hq * d), None

    def _state(self, i, y, ys, slots, offsets):
        rh, d, n, w, kw = self.rh, self.cfg.inner, self.cfg.states, self.norms, dict(offsets=offsets, past=self.lengths)
        conv, state = self.states[i]
        row = self._product(f"gate{i}", y, ys)
        x = rh.state_conv(row[:, :d], w[f"conv{i}"], conv, slots, bias=w[f"conv_bias{i}"], **kw)
        select = self._product(f"select{i}", x)
        b, c = select[:, d:d + n].unflatten(1, (1, n)), select[:, d + n:].unflatten(1, (1, n))
        x = rh.state_scan(x, select[:, :d], self.fade[i], b, c, state, slots, skip=w[f"skip{i}"], dt_bias=w[f"dt_bias{i}"], **kw)
        return rh.norm_gated(x, row[:, d:], w[f"norm_s{i}"], groups=self.cfg.groups, eps=self.cfg.eps, outputs="e4m3")[1:]

    def _give_back(self):
        """The first page of every stream whose frames there all lie behind the window (a step adds one frame, so that one page a step is
        enough): on the free stack as the page of a stream that has ended, and out of the stream's row of the table."""
        cfg = self.cfg
        drop = self.held >= cfg.window + cfg.page
        frames = drop.int() * cfg.page
        self.rh.cache_plan(self.ended, frames, self.table[:, :1].contiguous(), self.free, self.free_count, cfg.page, 1, new_count=self.free_count)
        self.table[:, :-1] = torch.where(drop[:, None], self.table[:, 1:], self.table[:, :-1])
        self.held.sub_(frames)

    def _norm(self, name, x, h):
        """The residual stream with x added to it (x itself begins it), and the norm of it in 8 bits."""
        total, _, y, ys = self.rh.norm_residual(x, self.norms[name], h, eps=self.cfg.eps, outputs="e4m3", sum_out=h)
        return (x if h is None else total), None, y, ys

    def step(self, features: torch.Tensor, n_new: torch.Tensor) -> torch.Tensor:
        """features f32 [max_streams, n_features], n_new int32 [max_streams]: 1 (or more) - a frame of this stream, 0 - none, -1 (or less) - the
        stream has ended -> scores f32 [max_streams, mbh, mbw], of the streams with a frame; a tensor of its own every time.  A stream that got no room in the
        cache (`granted` is False there, its length stays) is scored from the frames that it has: end it and begin it anew, or give the cache more room."""
        self.features.copy_(features)
        self.n_new.copy_(n_new)
        self.calls += 1
        if self.graph is None and self.want_graph and self.calls > 1:
            self._record()
        if self.graph is None:
            scores, self.granted = self._step()
            return scores
        self.graph.replay()
        scores, self.granted = (t.clone() for t in self.outputs)   # the graph's own tensors are the next step's too
        return scores

    def chunk(self, features: torch.Tensor, offsets: torch.Tensor) -> torch.Tensor:
        """Many frames of each stream at once (mixer "state"): features f32 [rows, n_features], rows offsets[b] to offsets[b + 1] (int32 [max_streams + 1], ascending
        from 0 to rows) being the next frames of stream b, which goes on from them -> scores f32 [rows, mbh, mbw].  Not recorded.
        As the operators take them: offsets outside [0, rows] count as its ends, where any descend no stream has a frame, and frames of no stream score 0.  At most
        2048 streams (a step takes any number)."""
        if self.cfg.mixer != "state":
            raise ValueError("chunk: frames of a stream go one at a time through attention")
        rows, streams = features.shape[0], self.cfg.max_streams
        if tuple(offsets.shape) != (streams + 1,) or offsets.dtype != torch.int32:
            raise ValueError(f"chunk: offsets {offsets.dtype} {tuple(offsets.shape)}, not torch.int32 {(streams + 1,)}")
        offsets = offsets.clamp(0, rows)
        begin, end, ends = offsets[:-1], offsets[1:], offsets[::streams]
        offsets.mul_((end >= begin).all())
        scores = self._layers(features, self._state, self.every, offsets)
        # made anew every time: one kept from a call that a caller captures would hold nothing until the graph's replay
        row = torch.arange(rows, dtype=torch.int32, device=offsets.device)
        ahead, behind = (row.view(-1, 1) < ends).unbind(1)          # of the first stream's rows, of the last one's end
        scores.masked_fill_((ahead == behind).view(-1, 1, 1), 0)    # rows that were never written
        frames = end - begin
        self.granted = frames > 0
        self.lengths.add_(frames)
        return scores

    def _record(self):
        rh, main = self.rh, self.rh._stream
        side, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
        rh.set_stream(side)
        try:
            with torch.cuda.graph(graph, stream=side):
                self.outputs = self._step()
        finally:
            rh.set_stream(main)
        self.graph = graph


def residual_features(res_y: torch.Tensor, mbh: int, mbw: int) -> torch.Tensor:
    """Mean magnitude of the codec's luma residual over each macroblock: int16 [n, H, W] -> f32 [n, mbh * mbw]."""
    n, height, width = res_y.shape
    x = torch.zeros((n, mbh * 16, mbw * 16), device=res_y.device)
    x[:, :height, :width] = res_y.abs().float()
    return x.view(n, mbh, 16, mbw, 16).mean((2, 4)).view(n, mbh * mbw)


def main():
    import time

    ap = argparse.ArgumentParser()
    ap.add_argument("--mixer", default="attention", choices=("attention", "state"))
    mixer = ap.parse_args().mixer

    import workloads as wl
    cfg = wl.replace(wl.config(5), n_frames=8)                     # one frame of each of 8 streams of 640 x 368
    streams, frames = cfg.n_frames, 30
    rh = RH(frame_w=cfg.width, frame_h=cfg.height, max_frames=streams, halo=cfg.halo, bin_size=cfg.bin_size, max_bins=256, net=cfg.net,
            weights=wl.make_weights(cfg.net, cfg.weight_seed, cfg.precision), precision=cfg.precision)
    pc = PredictorConfig(mbw=cfg.mbw, mbh=cfg.mbh, n_features=cfg.mbw * cfg.mbh, max_streams=streams, mixer=mixer)
    predictor = StreamPredictor(rh, pc, random_weights(pc, 0), graph=True)
    pixels = torch.from_numpy(wl.make_frames(cfg, streams)).to(rh.device)
    residuals = torch.from_numpy(wl.make_residuals(cfg.width, cfg.height, streams, frames, seed=1)).to(rh.device).view(streams, frames, cfg.height, cfg.width)
    new = torch.ones(streams, dtype=torch.int32, device=rh.device)
    per, k = cfg.mbw * cfg.mbh, int(0.2 * cfg.mbw * cfg.mbh * streams)
    ms = []
    for t in range(frames):
        torch.cuda.synchronize()
        begin = time.perf_counter()
        scores = predictor.step(residual_features(residuals[:, t], cfg.mbh, cfg.mbw), new)
        torch.cuda.synchronize()
        scored = time.perf_counter()
        mask, lst, n_sel = rh.select_regions(scores, [(0, streams, k)])
        po = rh.pack(pixels, scores, mask, lst, n_sel)
        net = rh.enhance(po.bins, n_valid=po.counts[1:2])
        rh.unpack(net, po.places, po.counts[3:4], pixels)
        torch.cuda.synchronize()
        ms.append((1e3 * (scored - begin), 1e3 * (time.perf_counter() - scored)))
    a, b = (sorted(v)[len(v) // 2] for v in zip(*ms))
    print(f"{streams} streams of {cfg.width}x{cfg.height}, {frames} frames each: {a:.3f} ms a frame to score {streams * per} macroblocks, "
          f"{b:.3f} ms to select, pack, enhance and paste {k} of them; {int(predictor.lengths[0])} frames remembered a stream")


if __name__ == "__main__":
    main()
