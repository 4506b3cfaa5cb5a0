"""The stream predictor (paper_2407_16990_amd/predictor.py) against the same network step by step in 64 bits, with the roundings
that its tensors have (bf16 activations, 8-bit norm outputs, the cache's type) at the same places."""
import numpy as np
import pytest
import torch

import oracle
import workloads as wl
from oracle import sequence as S
from paper_2407_16990_amd import RH, predictor as P

pytestmark = pytest.mark.gpu


def _rh(streams, w=160, h=96):
    net = wl.Net("plain", 4, 2, 2)
    return RH(frame_w=w, frame_h=h, max_frames=streams, halo=2, bin_size=32, max_bins=64, net=net, weights=wl.make_weights(net, 0, "fp32"), precision="fp32")


def _bf16(a):
    return torch.from_numpy(a).to(torch.bfloat16).double().numpy()


def _e4m3(a):
    return torch.from_numpy(a.clip(-448, 448)).float().to(torch.float8_e4m3fn).float().double().numpy()


class Plain:
    """The network on numpy arrays: every stream's keys and values in a list, no pages."""

    def __init__(self, cfg, weights):
        self.cfg = cfg
        self.w = {n: w.astype(np.float64) if w.ndim == 1 else S.unpack_weights(*P.pack_weights(w), w.shape[1]) for n, w in weights.items()}
        self.past = [[[] for _ in range(cfg.max_streams)] for _ in range(cfg.layers)]

    def norm(self, name, s):
        y, sc = S.norm(s, self.w[name], None, self.cfg.eps)[1:]
        return _e4m3(y / sc[:, None]) * sc[:, None]

    def cached(self, a):                                           # [heads, dim]
        if self.cfg.cache_dtype == torch.bfloat16:
            return _bf16(a)
        sc = np.maximum(np.abs(a).max(-1, keepdims=True), S.AMAX_MIN) / 448
        return _e4m3(a / sc) * sc

    def step(self, features, new):
        c, w = self.cfg, self.w
        n = c.max_streams
        x, h = _bf16(features @ w["in"].T), 0.0
        for i in range(c.layers):
            s = x + h                                              # normed before it is rounded
            h = _bf16(s)
            row = _bf16(self.norm(f"norm_a{i}", s) @ w[f"qkv{i}"].T).reshape(n, -1, c.dim)
            a = np.zeros((n, c.q_heads, c.dim))
            for b in range(n):
                past = self.past[i][b]
                if new[b] < 0:
                    past.clear()
                elif new[b] > 0:
                    past.append((self.cached(row[b, c.q_heads:c.q_heads + c.kv_heads]), self.cached(row[b, c.q_heads + c.kv_heads:])))
                seen = past[-c.window:] if c.window else past
                for head in range(c.q_heads if seen else 0):
                    k, v = (np.stack([t[j][head // (c.q_heads // c.kv_heads)] for t in seen]) for j in (0, 1))
                    e = k @ row[b, head] * c.dim ** -0.5
                    e = np.exp(e - e.max())
                    a[b, head] = e @ v / e.sum()
            s = h + _bf16(_bf16(a.reshape(n, -1)) @ w[f"proj{i}"].T)
            h = _bf16(s)
            u = _bf16(np.maximum(self.norm(f"norm_b{i}", s) @ w[f"wide{i}"].T, 0))
            x = _bf16(u @ w[f"narrow{i}"].T)
        return (self.norm("norm_out", x + h) @ w["out"].T).reshape(n, c.mbh, c.mbw)


# Both sides round at the same places, so they differ where a value falls on either side of a tie, and by what follows from that.  Bar: as
# if every rounding were drawn anew on either side: per layer five to bf16 (2^-8 / sqrt 3 = 2.3e-3 of a value at most, uniform) and two to
# e4m3 (2^-4 / sqrt 3 = 3.6e-2), over two layers and the last norm, both sides: sqrt(2 * (10 * 2.3e-3^2 + 5 * 3.6e-2^2)) = 0.115; a wrong
# slot, page or head is an error of the order of one.  Where nothing falls on a tie the difference is that of fp32 sums.
BAR = 0.115


@pytest.mark.parametrize("cache_dtype", [torch.bfloat16, torch.float8_e4m3fn])
@pytest.mark.parametrize("graph", [False, True])
@pytest.mark.parametrize("window", [0, 5])
def test_scores_over_many_frames(cache_dtype, graph, window):
    cfg = P.PredictorConfig(mbw=10, mbh=6, n_features=75, max_streams=5, hidden=160, layers=2, q_heads=6, kv_heads=2, dim=32, widened=288, page=3,
                            n_pages=60, max_pages=12, window=window, cache_dtype=cache_dtype)
    weights = P.random_weights(cfg, 3)
    pred, plain = P.StreamPredictor(_rh(5), cfg, weights, graph=graph), Plain(cfg, weights)
    rng = np.random.default_rng(window)
    for t in range(14):
        f = rng.standard_normal((5, cfg.n_features)).astype(np.float32)
        new = np.array([1, t % 2, -1 if t % 6 == 5 else 1, int(t > 3), 1 if t < 8 else -1 if t == 8 else 0])
        got = pred.step(torch.from_numpy(f).cuda(), torch.from_numpy(new.astype(np.int32)).cuda()).double().cpu().numpy()
        want = plain.step(f.astype(np.float64), new)
        live = [b for b in range(5) if new[b] > 0]
        err = np.linalg.norm(got[live] - want[live]) / np.linalg.norm(want[live])
        assert err <= BAR, (t, err)
        assert pred.lengths.cpu().tolist() == [len(p) for p in plain.past[0]]


def test_scores_feed_the_selection():
    cfg = P.PredictorConfig(mbw=10, mbh=6, n_features=60, max_streams=3, hidden=64, layers=1, q_heads=2, kv_heads=1, dim=32, widened=64, n_pages=8, max_pages=4)
    rh = _rh(3)
    pred = P.StreamPredictor(rh, cfg, P.random_weights(cfg, 1))
    res = torch.from_numpy(wl.make_residuals(160, 96, 3, 1, seed=4)).cuda()
    scores = pred.step(P.residual_features(res, 6, 10), torch.ones(3, dtype=torch.int32, device="cuda"))
    mask, lst, n_sel = rh.select_regions(scores, [(0, 3, 40)])
    o_mask, o_list = oracle.select(scores.cpu().numpy(), np.array([[0, 3, 40]], dtype=np.uint32), "topk", None)
    assert int(n_sel[0]) == 40 and np.array_equal(mask.cpu().numpy(), o_mask) and np.array_equal(lst[:40].cpu().numpy().astype(np.uint32), o_list)


def test_residual_features_of_ragged_frames():
    res = np.arange(2 * 20 * 35, dtype=np.int16).reshape(2, 20, 35) - 500
    got = P.residual_features(torch.from_numpy(res).cuda(), 2, 3).cpu().numpy()
    full = np.zeros((2, 32, 48)); full[:, :20, :35] = np.abs(res)
    assert np.allclose(got, full.reshape(2, 2, 16, 3, 16).mean((2, 4)).reshape(2, 6), rtol=1e-6)


def test_wrong_weights_are_refused():
    cfg = P.PredictorConfig(mbw=10, mbh=6, n_features=60, max_streams=3)
    w = P.random_weights(cfg, 0)
    w["qkv1"] = w["qkv1"][:-1]
    with pytest.raises(ValueError, match="qkv1"):
        P.StreamPredictor(_rh(3), cfg, w)
