"""StreamPredictor.chunk on the GPU: offsets that do not fit the rows."""
import pytest
import torch

from paper_2407_16990_amd import predictor as P
from test_gpu_predictor import _rh
from test_gpu_predictor_mixer import BAR, _config, _off

pytestmark = pytest.mark.gpu


def _i32(v):
    return torch.tensor(v, dtype=torch.int32, device="cuda")


def _states(pred):
    return [s.clone() for pair in pred.states for s in pair]


def test_offsets_that_descend_or_leave_the_rows():
    """Descending ones change nothing and score 0; others count as the rows' ends, in scores, states and lengths alike."""
    cfg = _config(max_streams=3)
    weights = P.random_weights(cfg, 6)
    a, b = P.StreamPredictor(_rh(3), cfg, weights), P.StreamPredictor(_rh(3), cfg, weights)
    g = torch.Generator(device="cuda").manual_seed(0)
    for given, taken in (([0, 4, 4, 9], [0, 4, 4, 9]), ([0, 9, 5, 9], None), ([-5, 2, 7, 2 ** 31 - 1], [0, 2, 7, 9]), ([1, 3, 3, 8], [1, 3, 3, 8]), ([9, 6, 3, 0], None)):
        rows = torch.randn((9, cfg.n_features), generator=g, device="cuda")
        before, lengths = _states(a), a.lengths.clone()
        got = a.chunk(rows, _i32(given))
        if taken is None:
            assert bool((got == 0).all()) and torch.equal(a.lengths, lengths) and not bool(a.granted.any())
            assert all(torch.equal(p, q) for p, q in zip(_states(a), before))
            continue
        # the same rows without what no stream has of them
        lo, hi = taken[0], taken[-1]
        want = b.chunk(rows[lo:hi].contiguous(), _i32([v - lo for v in taken]))
        # rows of a product go together in passes, so that other rows beside them may take another order of sums
        assert _off(got[lo:hi].cpu().numpy(), want.cpu().numpy()) <= BAR
        assert bool((got[:lo] == 0).all()) and bool((got[hi:] == 0).all())
        assert torch.equal(a.lengths, b.lengths) and torch.equal(a.granted, b.granted)
        assert all(_off(p.double().cpu().numpy(), q.double().cpu().numpy()) <= BAR for p, q in zip(_states(a), _states(b)))
