"""StreamPredictor.chunk on the GPU: offsets that do not fit the rows, and chunks so long that the scan cuts them."""
import numpy as np
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


@pytest.mark.parametrize("counts", [[300, 0, 287], [1, 700, 288]])
def test_chunks_that_are_cut(counts):
    """Streams of 288 frames and more, which the scan takes in pieces side by side: the scores and states that single steps give."""
    cfg = _config(max_streams=3)
    weights = P.random_weights(cfg, 7)
    a, b = P.StreamPredictor(_rh(3), cfg, weights), P.StreamPredictor(_rh(3), cfg, weights, graph=True)
    g = torch.Generator(device="cuda").manual_seed(1)
    for turn in range(2):
        rows = torch.randn((sum(counts), cfg.n_features), generator=g, device="cuda")
        offsets = np.concatenate(([0], np.cumsum(counts))).tolist()
        got = a.chunk(rows, _i32(offsets))
        want = torch.zeros_like(got)
        for t in range(max(counts)):
            live = [s for s in range(3) if t < counts[s]]
            f = torch.zeros((3, cfg.n_features), device="cuda")
            f[live] = rows[[offsets[s] + t for s in live]]
            scores = b.step(f, _i32([int(t < n) for n in counts]))
            for s in live:
                want[offsets[s] + t] = scores[s]
        off = ((got - want).flatten(1).norm(dim=1) / want.flatten(1).norm(dim=1)).cpu().numpy()
        assert off.max() <= BAR, (turn, float(off.max()), int(off.argmax()))
        assert torch.equal(a.lengths, b.lengths)
        for p, q in zip(_states(a), _states(b)):
            assert _off(p.double().cpu().numpy(), q.double().cpu().numpy()) <= BAR


def test_a_caller_may_capture_a_chunk():
    """A chunk in a caller's graph, first of all its calls but one of the context's: replays with new rows and offsets are what the calls give, and so are calls between them."""
    cfg = _config(max_streams=3)
    weights = P.random_weights(cfg, 8)
    rh, other = _rh(3), _rh(3)
    a, b = P.StreamPredictor(rh, cfg, weights), P.StreamPredictor(other, cfg, weights)
    g = torch.Generator(device="cuda").manual_seed(2)
    rows, offsets = torch.zeros((400, cfg.n_features), device="cuda"), _i32([0, 350, 380, 400])
    P.StreamPredictor(rh, cfg, weights).chunk(rows, offsets)        # the context's scratch memory is there
    torch.cuda.synchronize()
    side, main, graph = torch.cuda.Stream(), torch.cuda.current_stream(), torch.cuda.CUDAGraph()
    rh.set_stream(side)
    try:
        with torch.cuda.graph(graph, stream=side):
            scores = a.chunk(rows, offsets)
    finally:
        rh.set_stream(main)
    for given in ([0, 350, 380, 400], [0, 20, 20, 390], [3, 390, 390, 390], [0, 9, 5, 400], [0, 1, 2, 400]):
        new = torch.randn((400, cfg.n_features), generator=g, device="cuda")
        few = torch.randn((5, cfg.n_features), generator=g, device="cuda")
        rows.copy_(new)
        offsets.copy_(_i32(given))
        graph.replay()
        assert torch.equal(scores, b.chunk(new, _i32(given)))
        assert torch.equal(a.chunk(few, _i32([0, 2, 2, 4])), b.chunk(few, _i32([0, 2, 2, 4])))
        assert torch.equal(a.lengths, b.lengths) and all(torch.equal(p, q) for p, q in zip(_states(a), _states(b)))
