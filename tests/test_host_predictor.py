"""What StreamPredictor refuses before it allocates anything (no GPU)."""
from types import SimpleNamespace

import pytest
import torch


@pytest.mark.parametrize("dtype", [torch.float32, torch.float16, torch.float8_e5m2])
def test_a_cache_that_the_step_cannot_write_is_refused(dtype):
    from paper_2407_16990_amd import predictor as P
    cfg = P.PredictorConfig(mbw=10, mbh=6, n_features=60, max_streams=3, n_pages=4, cache_dtype=dtype)
    with pytest.raises(ValueError, match="cache_dtype"):
        P.StreamPredictor(SimpleNamespace(device=torch.device("cpu")), cfg, P.random_weights(cfg, 0))
