"""Macroblock importance for live streams, a frame of every stream at a time: a small transformer that remembers each
stream's past in a paged key-value cache, on the operators of include/rh_seq.h.  Its scores are what select_regions takes.

One token stands for one frame of one stream: its input is a vector of codec features of the frame's macroblocks (what tells
one frame's place in time from another's has to be among them), its output one score per macroblock.  A layer is
    norm -> queries, keys, values -> attention over the stream's frames -> projection -> residual
    norm -> widening product, ReLU -> narrowing product -> residual
with weights in 4 bits, the residual stream in bf16, and the norms' outputs in 8 bits.

    python -m paper_2407_16990_amd.predictor        # eight streams through predictor, selection, packing, enhancement and paste
"""
from __future__ import annotations

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


def weight_shapes(cfg: PredictorConfig) -> dict:
    """Names and shapes of the float weights: [outputs, inputs] of the products, [hidden] of the norms."""
    h, heads = cfg.hidden, cfg.q_heads + 2 * cfg.kv_heads
    shapes = {"in": (h, cfg.n_features), "norm_out": (h,), "out": (cfg.mbw * cfg.mbh, h)}
    for i in range(cfg.layers):
        shapes |= {f"norm_a{i}": (h,), f"qkv{i}": (heads * cfg.dim, h), f"proj{i}": (h, cfg.q_heads * cfg.dim),
                   f"norm_b{i}": (h,), f"wide{i}": (cfg.widened, h), f"narrow{i}": (h, cfg.widened)}
    return shapes


def random_weights(cfg: PredictorConfig, seed: int) -> dict:
    """Weights of that architecture, drawn: products keep the scale of their input, norms near one."""
    rng = np.random.default_rng(seed)
    return {name: (1 + 0.1 * rng.standard_normal(s) if len(s) == 1 else rng.standard_normal(s) / np.sqrt(s[1])).astype(np.float32)
            for name, s in weight_shapes(cfg).items()}


class StreamPredictor:
    """The state of max_streams streams and the step that takes one frame of each.  rh: the context whose stream the work goes
    on, and which is to be torch's current one; other calls of that context must not overlap with a step on another stream, replays included.
    graph: record the step at its second call and replay it from then on (one launch instead of one per operator).
    lengths: frames of each stream that found room since it began; granted: which streams' frames did in the last step."""

    def __init__(self, rh: RH, cfg: PredictorConfig, weights: dict, graph: bool = False):
        self.rh, self.cfg, dev = rh, cfg, rh.device
        if cfg.cache_dtype not in (torch.bfloat16, torch.float8_e4m3fn):
            raise ValueError(f"cache_dtype {cfg.cache_dtype}: keys and values are bf16, the cache torch.bfloat16 or torch.float8_e4m3fn")
        for name, shape in weight_shapes(cfg).items():
            if tuple(weights[name].shape) != shape:
                raise ValueError(f"{name}: {tuple(weights[name].shape)}, not {shape}")
        put = lambda a: torch.from_numpy(np.ascontiguousarray(a)).to(dev)  # noqa: E731
        self.norms = {n: put(np.asarray(w, dtype=np.float32)) for n, w in weights.items() if w.ndim == 1}
        self.packed = {n: tuple(put(a) for a in pack_weights(w)) for n, w in weights.items() if w.ndim == 2}
        shape = (cfg.n_pages, cfg.kv_heads, cfg.page, cfg.dim)
        quantised = cfg.cache_dtype == torch.float8_e4m3fn

        def cache():
            kv = [torch.zeros(shape, dtype=torch.uint8, device=dev).view(cfg.cache_dtype) if quantised else
                  torch.zeros(shape, dtype=cfg.cache_dtype, device=dev) for _ in range(2)]
            scales = [torch.zeros(shape[:3], device=dev) if quantised else None for _ in range(2)]
            return KVCache(kv[0].transpose(1, 2), kv[1].transpose(1, 2), *scales)
        self.caches = [cache() for _ in range(cfg.layers)]
        n = cfg.max_streams
        i32 = dict(dtype=torch.int32, device=dev)
        self.lengths, self.table = torch.zeros(n, **i32), torch.full((n, cfg.max_pages), -1, **i32)
        # frames in the cache: fewer than a stream has had once pages behind the window are given back
        self.held, self.ended = (torch.zeros(n, **i32), torch.full((n,), -1, **i32)) if cfg.window else (self.lengths, None)
        self.free, self.free_count = torch.arange(cfg.n_pages, **i32), torch.full((1,), cfg.n_pages, **i32)
        self.features, self.n_new = torch.zeros((n, cfg.n_features), device=dev), torch.zeros(n, **i32)
        self.want_graph, self.graph, self.outputs, self.calls, self.granted = graph, None, None, 0, None

    def _product(self, name, x, x_scale=None, **kw):
        return self.rh.matvec_packed(x, *self.packed[name], x_scale=x_scale, **kw)

    def _step(self):
        rh, cfg = self.rh, self.cfg
        n, hq, hk, d = cfg.max_streams, cfg.q_heads, cfg.kv_heads, cfg.dim
        self.n_new.clamp_(-1, 1)                                   # a step has one row a stream: no room is planned for more than it writes
        if cfg.window:
            self._give_back()
        slots, off, _, _ = rh.cache_plan(self.n_new, self.held, self.table, self.free, self.free_count, cfg.page, n,
                                         new_lengths=self.held, new_count=self.free_count)
        granted = off[1:] > off[:-1]
        if cfg.window:
            self.lengths.add_(granted).masked_fill_(self.n_new < 0, 0)
        # the plan lists tokens, the rows below are streams: a stream without a token in this step writes nothing
        mine = slots[off[:-1].clamp_max(n - 1).long()]
        slots = torch.where(granted, mine, torch.full_like(mine, -1))
        x = self._product("in", self.features, out_dtype=torch.bfloat16)
        h = None
        for i, cache in enumerate(self.caches):
            h, _, y, ys = self._norm(f"norm_a{i}", x, h)
            row = self._product(f"qkv{i}", y, ys)
            rh.cache_write(cache, row[:, hq * d:(hq + hk) * d].unflatten(1, (hk, d)), row[:, (hq + hk) * d:].unflatten(1, (hk, d)), slots)
            a = rh.cache_attend(row[:, : hq * d].unflatten(1, (hq, d)), cache, self.table, self.held, window=cfg.window)
            x = self._product(f"proj{i}", a.view(n, hq * d))
            h, _, y, ys = self._norm(f"norm_b{i}", x, h)
            x = self._product(f"narrow{i}", self._product(f"wide{i}", y, ys, relu=True))
        _, _, y, ys = self._norm("norm_out", x, h)
        return self._product("out", y, ys, out_dtype=torch.float32).view(n, cfg.mbh, cfg.mbw), granted

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

    import workloads as wl
    cfg = wl.replace(wl.config(5), n_frames=8)                     # one frame of each of 8 streams of 640 x 368
    streams, frames = cfg.n_frames, 30
    rh = RH(frame_w=cfg.width, frame_h=cfg.height, max_frames=streams, halo=cfg.halo, bin_size=cfg.bin_size, max_bins=256, net=cfg.net,
            weights=wl.make_weights(cfg.net, cfg.weight_seed, cfg.precision), precision=cfg.precision)
    pc = PredictorConfig(mbw=cfg.mbw, mbh=cfg.mbh, n_features=cfg.mbw * cfg.mbh, max_streams=streams)
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
