"""The stream predictor with state layers (mixer "state") against the same network step by step in 64 bits, with the roundings that its tensors have
(bf16 activations, 8-bit norm outputs) at the same places."""
import numpy as np
import pytest
import torch

import oracle
import workloads as wl
from oracle import sequence as S
from oracle import state as O
from paper_2407_16990_amd import predictor as P
from test_gpu_predictor import _bf16, _e4m3, _rh

pytestmark = pytest.mark.gpu


def _config(**kw):
    return P.PredictorConfig(**{**dict(mbw=10, mbh=6, n_features=75, max_streams=5, hidden=160, layers=2, widened=288, mixer="state", inner=192, states=12, taps=4, groups=3), **kw})


class Plain:
    """The network on numpy arrays: every stream's last inputs and states by themselves, no pool, no slots."""

    def __init__(self, cfg, weights):
        self.cfg, self.w = cfg, {}
        for n, w in weights.items():
            small = w.ndim == 1 or n.rstrip("0123456789") in ("conv", "a_log")
            self.w[n] = w.astype(np.float64) if small else S.unpack_weights(*P.pack_weights(w), w.shape[1])
        self.lengths = np.zeros(cfg.max_streams, int)
        self.conv = np.zeros((cfg.layers, cfg.max_streams, cfg.taps - 1, cfg.inner))
        self.state = np.zeros((cfg.layers, cfg.max_streams, cfg.inner, cfg.states))

    def quantised(self, y):
        sc = np.maximum(np.abs(y).max(-1), S.AMAX_MIN) / S.E4M3_MAX
        return _e4m3(y / sc[:, None]) * sc[:, None]

    def frame(self, b, f):
        """One frame of one stream; the stream goes on."""
        c, w, d = self.cfg, self.w, self.cfg.inner
        if self.lengths[b] == 0:
            self.conv[:, b], self.state[:, b] = 0, 0
        x, h = _bf16(f[None] @ w["in"].T), 0.0
        for i in range(c.layers):
            s = x + h
            h = _bf16(s)
            row = _bf16(self.quantised(S.norm(s, w[f"norm_a{i}"], None, c.eps)[1]) @ w[f"gate{i}"].T)
            u, new = O.conv(row[:, :d], w[f"conv{i}"], self.conv[i], [b], bias=w[f"conv_bias{i}"])
            self.conv[i] = new
            u = _bf16(u)
            sel = _bf16(u @ w[f"select{i}"].T)
            y, new, _ = O.scan(u, sel[:, :d], -np.exp(w[f"a_log{i}"]), sel[:, None, d:d + c.states], sel[:, None, d + c.states:], self.state[i], [b], skip=w[f"skip{i}"],
                               dt_bias=w[f"dt_bias{i}"])
            self.state[i] = new
            g = O.gated_norm(_bf16(y), row[:, d:], w[f"norm_s{i}"], c.groups, c.eps)
            s = h + _bf16(self.quantised(g) @ w[f"proj{i}"].T)
            h = _bf16(s)
            v = _bf16(np.maximum(self.quantised(S.norm(s, w[f"norm_b{i}"], None, c.eps)[1]) @ w[f"wide{i}"].T, 0))
            x = _bf16(v @ w[f"narrow{i}"].T)
        self.lengths[b] += 1
        return (self.quantised(S.norm(x + h, w["norm_out"], None, c.eps)[1]) @ w["out"].T).reshape(c.mbh, c.mbw)


# As if every rounding were drawn anew on either side: per layer seven to bf16 (2^-8 / sqrt 3 = 2.3e-3 of a value at most, uniform) and three to e4m3 (2^-4 / sqrt 3 =
# 3.6e-2), over two layers and the last norm, both sides: sqrt(2 * (14 * 2.3e-3^2 + 7 * 3.6e-2^2)) = 0.135; a wrong slot, stream or gate is an error of the order of one.
BAR = 0.135


def _off(got, want):
    return np.linalg.norm(got - want) / np.linalg.norm(want)


@pytest.mark.parametrize("graph", [False, True])
def test_scores_over_many_frames(graph):
    cfg = _config()
    weights = P.random_weights(cfg, 3)
    pred, plain = P.StreamPredictor(_rh(5), cfg, weights, graph=graph), Plain(cfg, weights)
    rng = np.random.default_rng(0)
    for t in range(14):
        f = rng.standard_normal((5, cfg.n_features)).astype(np.float32)
        new = np.array([1, t % 2, -1 if t % 6 == 5 else 1, int(t > 3), 1 if t < 8 else -1 if t == 8 else 0])
        kept = [s.clone() for pair in pred.states for s in pair]
        got = pred.step(torch.from_numpy(f).cuda(), torch.from_numpy(new.astype(np.int32)).cuda()).double().cpu().numpy()
        for b in range(5):
            if new[b] > 0:
                err = _off(got[b], plain.frame(b, f[b].astype(np.float64)))
                assert err <= BAR, (t, b, err)
            elif new[b] < 0:
                plain.lengths[b] = 0
            if new[b] <= 0:                                        # no frame: the stream's states stay
                assert all(torch.equal(a[b], s[b]) for a, s in zip(kept, [s for pair in pred.states for s in pair]))
        assert pred.lengths.cpu().tolist() == plain.lengths.tolist()
        assert pred.granted.cpu().tolist() == (new > 0).tolist()


@pytest.mark.parametrize("graph", [False, True])
def test_chunks_and_steps_go_on_from_each_other(graph):
    """A chunk of frames of each stream, some of none, between steps: the scores and the states that single steps give."""
    cfg = _config(max_streams=4)
    weights = P.random_weights(cfg, 4)
    a, b = P.StreamPredictor(_rh(4), cfg, weights, graph=graph), P.StreamPredictor(_rh(4), cfg, weights)
    g = torch.Generator(device="cuda").manual_seed(0)
    ones = torch.ones(4, dtype=torch.int32, device="cuda")
    for counts in ([3, 0, 200, 1], [0, 5, 2, 1]):
        f = torch.randn((4, cfg.n_features), generator=g, device="cuda")
        x, y = a.step(f, ones), b.step(f, ones)
        assert _off(x.cpu().numpy(), y.cpu().numpy()) <= BAR
        rows = torch.randn((sum(counts), cfg.n_features), generator=g, device="cuda")
        offsets = np.concatenate(([0], np.cumsum(counts)))
        got = a.chunk(rows, torch.from_numpy(offsets.astype(np.int32)).cuda())
        for t in range(max(counts)):
            live = [s for s in range(4) if t < counts[s]]
            f = torch.zeros((4, cfg.n_features), device="cuda")
            f[live] = rows[[int(offsets[s]) + t for s in live]]
            want = b.step(f, torch.tensor([int(t < n) for n in counts], dtype=torch.int32, device="cuda"))
            for s in live:
                assert _off(got[int(offsets[s]) + t].cpu().numpy(), want[s].cpu().numpy()) <= BAR, (t, s)
        assert torch.equal(a.lengths, b.lengths)
        for (c1, s1), (c2, s2) in zip(a.states, b.states):
            assert _off(c1.double().cpu().numpy(), c2.double().cpu().numpy()) <= BAR and _off(s1.cpu().numpy(), s2.cpu().numpy()) <= BAR


def test_a_stream_begins_with_no_past():
    """What a pool of states holds of streams that have not begun (NaN) does not matter, nor what an ended stream leaves."""
    cfg = _config(max_streams=3)
    weights = P.random_weights(cfg, 5)
    a, b = P.StreamPredictor(_rh(3), cfg, weights), P.StreamPredictor(_rh(3), cfg, weights)
    for conv, state in a.states:
        conv.fill_(float("nan")); state.fill_(float("nan"))
    g = torch.Generator(device="cuda").manual_seed(0)
    ones = torch.ones(3, dtype=torch.int32, device="cuda")
    for t in range(5):
        f = torch.randn((3, cfg.n_features), generator=g, device="cuda")
        assert torch.equal(a.step(f, ones), b.step(f, ones)), t
    ended = torch.tensor([-1, 0, 0], dtype=torch.int32, device="cuda")
    a.step(f, ended)
    fresh = P.StreamPredictor(_rh(3), cfg, weights)
    f = torch.randn((3, cfg.n_features), generator=g, device="cuda")
    assert torch.equal(a.step(f, ones)[0], fresh.step(f, ones)[0])
    assert a.lengths.tolist() == [1, 6, 6]


def test_scores_feed_the_selection():
    cfg = _config(n_features=60, max_streams=3, layers=1, hidden=64, widened=64, inner=64, groups=1)
    rh = _rh(3)
    pred = P.StreamPredictor(rh, cfg, P.random_weights(cfg, 1))
    res = torch.from_numpy(wl.make_residuals(160, 96, 3, 1, seed=4)).cuda()
    scores = pred.step(P.residual_features(res, 6, 10), torch.ones(3, dtype=torch.int32, device="cuda"))
    mask, lst, n_sel = rh.select_regions(scores, [(0, 3, 40)])
    o_mask, o_list = oracle.select(scores.cpu().numpy(), np.array([[0, 3, 40]], dtype=np.uint32), "topk", None)
    assert int(n_sel[0]) == 40 and np.array_equal(mask.cpu().numpy(), o_mask) and np.array_equal(lst[:40].cpu().numpy().astype(np.uint32), o_list)


def test_chunks_need_state_layers():
    cfg = P.PredictorConfig(mbw=10, mbh=6, n_features=60, max_streams=3, hidden=64, layers=1, widened=64, n_pages=8, max_pages=4)
    with pytest.raises(ValueError, match="attention"):
        P.StreamPredictor(_rh(3), cfg, P.random_weights(cfg, 0)).chunk(torch.zeros((3, 60), device="cuda"), torch.arange(4, dtype=torch.int32, device="cuda"))
