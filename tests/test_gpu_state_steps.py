"""rh_state_scan where steps are masked: dt of -inf, or of a type's lowest value, is a step of 0 that leaves the state, bit for bit; an infinite or undefined step is
what the formula makes of it."""
import numpy as np
import pytest
import torch

from test_gpu_state import HALF, TYPES, Streams, _gen, _np, _scan_bounds, _scan_inputs, rh  # noqa: F401  (rh: the fixture)

pytestmark = pytest.mark.gpu

INF = float("inf")
# single rows, streams that stay whole, streams that are cut
LENS = [None, [40, 3, 70], [700, 5, 290]]


def _inputs(s, channels, n, groups, dtype, mask):
    """Inputs in hand, and dt with a value in the masked rows."""
    i = _scan_inputs(_gen(n), s, channels, n, groups, dtype)
    state = i.pop("state")
    # dt + dt_bias of the others stays above -20
    dt = i.pop("dt")
    return i, state, lambda v: torch.where(mask[:, None], torch.tensor(v, device="cuda").to(dtype), dt)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("n,channels,groups", [(4, 70, 2), (13, 34, 1), (16, 64, 1), (128, 20, 1)])
@pytest.mark.parametrize("lens", LENS)
def test_masked_steps_leave_the_state(rh, dtype, n, channels, groups, lens):  # noqa: F811
    """softplus of anything below -104 is 0 in 32 bits: all of them give the same bits as -200, which gives the formula's values; a stream of such rows alone keeps its state's bits."""
    s = Streams(np.random.default_rng(n), lens, 3)
    rng = np.random.default_rng(1)
    masked = rng.random(s.rows) < 0.5
    masked[:s.lens[0]] = True                                        # all of the first stream
    i, state, dt = _inputs(s, channels, n, groups, dtype, torch.tensor(masked, device="cuda"))

    def run(step, **kw):
        mine = state.clone()
        return rh.state_scan(**{**i, **kw}, dt=step, state=mine, slots=s.slots, **s.kw()), mine
    y, new = run(dt(-200.0))
    want, states, y_tol, new_tol = _scan_bounds({**i, "dt": dt(-200.0), "state": state}, True, s, max(s.lens))
    assert (np.abs(_np(y) - want) <= y_tol + HALF[dtype] * (np.abs(want) + y_tol)).all()
    assert (np.abs(_np(new) - states) <= new_tol).all()
    assert torch.equal(new[int(s.into[0])], state[int(s.slots[0])])
    for v in (-INF, torch.finfo(torch.float32).min, torch.finfo(torch.bfloat16).min, -2.4e38, -2.3e38, -1e30, -3000.0):
        got = run(dt(v))
        assert torch.equal(got[0], y) and torch.equal(got[1], new), (v, int((got[0] != y).sum()), int((got[1] != new).sum()))
    # a channel that a bias of -inf freezes, whatever its dt
    frozen = [run(dt(0.0), dt_bias=torch.where(torch.arange(channels, device="cuda") == 2, v, i["dt_bias"])) for v in (-1000.0, -INF)]
    assert torch.equal(frozen[0][0], frozen[1][0]) and torch.equal(frozen[0][1], frozen[1][1])
    for b in range(s.n):
        assert torch.equal(frozen[1][1][int(s.into[b]), 2], state[int(s.slots[b]), 2])


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("n", [13, 16])
@pytest.mark.parametrize("lens", LENS)
def test_infinite_and_undefined_steps(rh, dtype, n, lens):  # noqa: F811
    """A step of +inf puts its row's infinity in the place of the state; one that is no number leaves none in its channel from there on.  Others stay as they are."""
    s = Streams(np.random.default_rng(n), lens, 3)
    channels, at = 20, 1 if lens is None else 30
    one = torch.zeros(s.rows, dtype=torch.bool, device="cuda")
    one[at] = True
    i, state, dt = _inputs(s, channels, n, 1, dtype, one)
    i["gate"] = None
    i["b"], i["c"], i["x"], i["skip"] = i["b"].abs() + 0.1, i["c"].abs() + 0.1, i["x"].abs() + 0.1, i["skip"].abs()
    b = 1 if lens is None else 0                                     # the row's stream
    hit = torch.zeros((s.rows, channels), dtype=torch.bool, device="cuda")
    hit[at:at + 1 if lens is None else s.lens[0], 3] = True

    def run(step):
        mine = state.clone()
        return rh.state_scan(**i, dt=step, state=mine, slots=s.slots, **s.kw()), mine
    base, kept = run(dt(0.0))
    for v, what in ((INF, torch.isposinf), (float("nan"), torch.isnan)):
        step = dt(0.0)
        step[at, 3] = v
        y, new = run(step)
        assert torch.equal(what(y), hit) and torch.equal(y[~hit], base[~hit])
        to = int(s.into[b])
        assert bool(what(new[to, 3]).all())
        new[to, 3] = kept[to, 3]
        assert torch.equal(new, kept)
