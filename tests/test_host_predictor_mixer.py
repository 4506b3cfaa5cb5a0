"""What StreamPredictor refuses of a state layer's configuration before it allocates anything, and its weights (no GPU)."""
from types import SimpleNamespace

import numpy as np
import pytest
import torch


@pytest.mark.parametrize("wrong", [dict(mixer="both"), dict(mixer="state", groups=7), dict(mixer="state", groups=0)])
def test_configurations_that_cannot_be_are_refused(wrong):
    from paper_2407_16990_amd import predictor as P
    cfg = P.PredictorConfig(mbw=10, mbh=6, n_features=60, max_streams=3, **wrong)
    with pytest.raises(ValueError, match="mixer|groups"):
        P.StreamPredictor(SimpleNamespace(device=torch.device("cpu")), cfg, {})


def test_weights_have_the_shapes_that_are_asked_for():
    from paper_2407_16990_amd import predictor as P
    for mixer in ("attention", "state"):
        cfg = P.PredictorConfig(mbw=10, mbh=6, n_features=60, max_streams=3, mixer=mixer)
        weights, shapes = P.random_weights(cfg, 0), P.weight_shapes(cfg)
        assert {n: w.shape for n, w in weights.items()} == shapes and all(np.isfinite(w).all() for w in weights.values())
    step = np.log1p(np.exp(weights["dt_bias1"].astype(np.float64)))
    assert (step > 0.00099).all() and (step < 0.101).all() and (np.exp(weights["a_log0"]) <= 16.01).all()


def test_a_missing_matrix_is_refused():
    from paper_2407_16990_amd import predictor as P
    cfg = P.PredictorConfig(mbw=10, mbh=6, n_features=60, max_streams=3, mixer="state")
    weights = P.random_weights(cfg, 0)
    weights["conv1"] = weights["conv1"][:-1]
    with pytest.raises(ValueError, match="conv1"):
        P.StreamPredictor(SimpleNamespace(device=torch.device("cpu")), cfg, weights)
