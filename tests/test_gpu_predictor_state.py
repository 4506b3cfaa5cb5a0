"""What a StreamPredictor keeps from step to step, and what it hands out."""
import numpy as np
import pytest
import torch

from paper_2407_16990_amd import predictor as P
from test_gpu_predictor import _rh

pytestmark = pytest.mark.gpu


def _config(**kw):
    return P.PredictorConfig(**{**dict(mbw=10, mbh=6, n_features=60, max_streams=4, hidden=64, layers=2, q_heads=2, kv_heads=1, dim=32, widened=96, page=4, n_pages=64,
                                       max_pages=16), **kw})


def _frames(cfg, steps, seed=0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return [torch.randn((cfg.max_streams, cfg.n_features), generator=g, device="cuda") for _ in range(steps)]


def _ones(cfg):
    return torch.ones(cfg.max_streams, dtype=torch.int32, device="cuda")


@pytest.mark.parametrize("graph", [False, True])
def test_scores_of_earlier_frames_stay(graph):
    cfg = _config()
    weights = P.random_weights(cfg, 1)
    kept, plain = P.StreamPredictor(_rh(4), cfg, weights, graph=graph), P.StreamPredictor(_rh(4), cfg, weights)
    frames = _frames(cfg, 7)
    scores = [kept.step(f, _ones(cfg)) for f in frames]
    want = [plain.step(f, _ones(cfg)).cpu() for f in frames]
    assert len({s.data_ptr() for s in scores}) == len(scores)
    for t, (a, b) in enumerate(zip(scores, want)):
        assert torch.equal(a.cpu(), b), t
    assert not np.array_equal(want[0], want[1])
