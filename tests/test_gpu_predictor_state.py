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


@pytest.mark.parametrize("graph", [False, True])
@pytest.mark.parametrize("cache_dtype", [torch.bfloat16, torch.float8_e4m3fn])
@pytest.mark.parametrize("window,page,max_pages", [(5, 4, 3), (1, 1, 2), (8, 4, 3), (3, 16, 2), (11, 3, 5)])
def test_a_window_goes_on_beyond_the_row_and_the_pool(graph, cache_dtype, window, page, max_pages):
    """Rows of the table and the pool hold a few frames more than the window: after many times as many frames a predictor with
    room for all of them gives the same scores, and no page is lost on the way, streams that end and begin included."""
    pages = -(-(window + page + 1) // page)
    cfg = _config(window=window, page=page, max_pages=max_pages, n_pages=4 * pages, cache_dtype=cache_dtype)
    roomy = _config(window=window, page=page, max_pages=100, n_pages=400, cache_dtype=cache_dtype)
    weights = P.random_weights(cfg, 2)
    small, large = P.StreamPredictor(_rh(4), cfg, weights, graph=graph), P.StreamPredictor(_rh(4), roomy, weights)
    assert max_pages * page >= window + page
    had = np.zeros(4, int)
    for t, f in enumerate(_frames(cfg, 70, window)):
        new = np.array([1, t % 3 > 0, -1 if t % 25 == 24 else 1, 1])
        d_new = torch.from_numpy(new.astype(np.int32)).cuda()
        a, b = small.step(f, d_new), large.step(f, d_new)
        live = new > 0
        assert torch.equal(a[live], b[live]), t
        had = np.where(new < 0, 0, had + live)
        assert small.granted.cpu().numpy().tolist() == live.tolist()
        assert small.lengths.cpu().numpy().tolist() == had.tolist() == large.lengths.cpu().numpy().tolist()
        held = small.held.cpu().numpy()
        assert (held >= np.minimum(had, window)).all() and (held <= window + page).all()
        rows, left = small.table.cpu().numpy(), small.free.cpu().numpy()[:int(small.free_count)]
        assert sorted([p for row, n in zip(rows, held) for p in row[:-(-int(n) // page)]] + left.tolist()) == list(range(cfg.n_pages))


@pytest.mark.parametrize("graph", [False, True])
@pytest.mark.parametrize("max_pages,n_pages", [(2, 64), (16, 9)])
def test_frames_without_room_are_told(graph, max_pages, n_pages):
    """Without a window a stream has room until its row, or the pool, is full; from then on granted says so, until it ends and begins anew."""
    cfg = _config(page=2, max_pages=max_pages, n_pages=n_pages)
    pred = P.StreamPredictor(_rh(4), cfg, P.random_weights(cfg, 3), graph=graph)
    had, seen = np.zeros(4, int), []
    frames = _frames(cfg, 14)
    for f in frames[:8]:
        pred.step(f, _ones(cfg))
        got = pred.granted.cpu().numpy()
        seen.append(pred.granted)
        # streams are served in order: by the row, or by what the pool has left
        need = -(-(had + 1) // 2) - -(-had // 2)
        free = n_pages - int((-(-had // 2)).sum())
        fits = -(-(had + 1) // 2) <= max_pages
        want = fits & ((need == 0) | (np.cumsum(np.where(fits, need, 0)) <= free))
        assert got.tolist() == want.tolist()
        had += want
        assert pred.lengths.cpu().numpy().tolist() == had.tolist()
    assert not got.all() and len({s.data_ptr() for s in seen}) == len(seen)
    ended = _ones(cfg) * 0                                         # no other stream takes the pages that come back
    ended[0] = -1
    pred.step(frames[8], ended)
    pred.step(frames[9], _ones(cfg))
    assert bool(pred.granted[0]) and int(pred.lengths[0]) == 1


@pytest.mark.parametrize("graph", [False, True])
def test_a_step_takes_one_frame_a_stream(graph):
    """Numbers above one count as one: nothing is planned, and later read, that the step does not write."""
    cfg = _config()
    weights = P.random_weights(cfg, 4)
    a, b = P.StreamPredictor(_rh(4), cfg, weights, graph=graph), P.StreamPredictor(_rh(4), cfg, weights)
    for t, f in enumerate(_frames(cfg, 6)):
        many = torch.tensor([1, 2, 7, -3 if t == 3 else 1], dtype=torch.int32, device="cuda")
        x, y = a.step(f, many), b.step(f, many.clamp(-1, 1))
        assert torch.equal(x[many > 0], y[many > 0]) and torch.equal(a.lengths, b.lengths) and torch.equal(a.granted, b.granted)
    assert a.lengths.tolist() == [6, 6, 6, 2]
