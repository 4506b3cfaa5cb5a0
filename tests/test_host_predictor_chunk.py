"""What StreamPredictor.chunk makes of its offsets, ahead of the operators and behind them (no GPU; operators that only make tensors of the right shapes stand in)."""
from types import SimpleNamespace

import pytest
import torch


def _predictor(streams, seen=None):
    """A predictor whose operators write nothing: what they return is NaN, and what offsets they got is in `seen`."""
    from paper_2407_16990_amd import predictor as P

    def nan(*s, dtype=torch.float32):
        return torch.full(s, float("nan"), dtype=dtype)

    def over_streams(x, *a, offsets=None, **kw):
        if seen is not None:
            seen.append(offsets.tolist())
        return nan(*x.shape)
    rh = SimpleNamespace(
        device=torch.device("cpu"), state_conv=over_streams, state_scan=over_streams,
        matvec_packed=lambda x, w, s, **kw: nan(x.shape[0], w.shape[0]),
        norm_residual=lambda x, w, h, **kw: (x if h is None else h, None, x, None), norm_gated=lambda x, *a, **kw: (None, x, None))
    cfg = P.PredictorConfig(mbw=2, mbh=2, n_features=5, max_streams=streams, hidden=32, layers=1, widened=32, mixer="state", inner=32, states=4, groups=1)
    return P.StreamPredictor(rh, cfg, P.random_weights(cfg, 0))


ROWS = 6
# offsets, as the operators take them, frames of each stream
CASES = [([0, 2, 2, 6], [0, 2, 2, 6], [2, 0, 4]), ([1, 2, 4, 5], [1, 2, 4, 5], [1, 2, 1]), ([-9, 2, 4, 2 ** 31 - 1], [0, 2, 4, 6], [2, 2, 2]), ([-2 ** 31, -5, 7, 9], [0, 0, 6, 6], [0, 6, 0]),
         ([0, 4, 2, 6], [0, 0, 0, 0], [0, 0, 0]), ([6, 4, 2, 0], [0, 0, 0, 0], [0, 0, 0]), ([0, 0, 0, 0], [0, 0, 0, 0], [0, 0, 0]), ([0, 6, 6, 5], [0, 0, 0, 0], [0, 0, 0])]


@pytest.mark.parametrize("offsets,taken,frames", CASES)
def test_offsets_count_as_the_operators_take_them(offsets, taken, frames):
    seen = []
    pred = _predictor(3, seen)
    pred.lengths.copy_(torch.tensor([7, 0, 100]))
    pred.granted = torch.ones(3, dtype=torch.bool)
    given = torch.tensor(offsets, dtype=torch.int32)
    scores = pred.chunk(torch.zeros(ROWS, 5), given)
    assert given.tolist() == offsets                                 # the caller's own
    assert seen == [taken, taken]
    assert pred.lengths.tolist() == [n + f for n, f in zip([7, 0, 100], frames)]
    assert pred.granted.tolist() == [f > 0 for f in frames]
    rows = torch.arange(ROWS)
    covered = (rows >= taken[0]) & (rows < taken[-1])
    assert bool(scores[covered].isnan().all()) and bool((scores[~covered] == 0).all())


def test_no_rows():
    pred = _predictor(3)
    assert pred.chunk(torch.zeros(0, 5), torch.tensor([0, 4, 2, 6], dtype=torch.int32)).shape == (0, 2, 2)
    assert pred.lengths.tolist() == [0, 0, 0] and pred.granted.tolist() == [False] * 3


@pytest.mark.parametrize("offsets", [torch.zeros(4, dtype=torch.int64), torch.zeros(4), torch.zeros(3, dtype=torch.int32), torch.zeros(5, dtype=torch.int32), torch.zeros((2, 2), dtype=torch.int32)])
def test_offsets_that_do_not_fit_are_refused(offsets):
    seen = []
    pred = _predictor(3, seen)
    with pytest.raises(ValueError, match="offsets"):
        pred.chunk(torch.zeros(ROWS, 5), offsets)
    assert not seen and pred.lengths.tolist() == [0, 0, 0]
