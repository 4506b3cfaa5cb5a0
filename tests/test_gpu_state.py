"""The operators that keep a state of fixed size for a stream (rh_state_conv, rh_state_scan, rh_norm_gated) against their plain
implementations in 64 bits (oracle/state.py), within bounds worked out from the arithmetic.

Bounds.  u = 2^-24 is half an ulp of 1 in fp32; a function of the hardware (power of two, logarithm, reciprocal) is off by an ulp, 2 u.
  SiLU   v times the reciprocal of 1 + 2^(-v log2 e): the exponent is rounded (|v| u of the power), then power, sum, reciprocal and product: (|v| + 8) u.
         Its slope is at most 1.1.
  conv   a sum of width products and the bias: (width + 2) u sum|w x|, then SiLU.  The states are inputs: exact.
  scan   delta: dt + dt_bias rounded (u |dt + dt_bias|, at most as much relative to softplus), power, logarithm, quotient: e_d = (|dt + dt_bias| + 16) u.
         A fade exp(delta a) is off by |delta a| (e_d + 4 u) + 2 u.  So an error of the state E becomes
             fade E + (fade |h| (|delta a| (e_d + 4 u) + 4 u) + |delta x b| (e_d + 4 u)) with one more rounding u |h'| of the sum.
         Where a stream is cut into chunks the sum of their deltas, at most `rows` terms, takes the fades' place: `rows` u more on each delta.
         y: sum |c| E + (n + 4) u sum|c h| + 2 u |skip x|, then the gate's SiLU, then half a step of the output.
  norm   products with SiLU; a mean of squares over `per` terms: (per + 2 (|gate| + 8) + 4) u, half of it after the root; four more roundings.
"""
import numpy as np
import pytest
import torch

from oracle import sequence as S
from oracle import state as O
from paper_2407_16990_amd import RhError
from test_gpu_sequence import E4M3, HALF, U, _context, _i32, _np, _refused

pytestmark = pytest.mark.gpu

TINY = 1e-36                          # results below it may be zero
TYPES = [torch.float32, torch.bfloat16]


@pytest.fixture(scope="module")
def rh():
    return _context()


def _gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def _randn(g, *shape, dtype=torch.float32):
    return torch.randn(shape, generator=g, device="cuda").to(dtype)


def _wide(g, rows, cols, dtype, ahead=3, behind=2):
    """A matrix out of the middle of wider rows, at any address; what lies beside it is NaN."""
    w = torch.full((rows, ahead + cols + behind), float("nan"), device="cuda").to(dtype)
    w[:, ahead:ahead + cols] = _randn(g, rows, cols, dtype=dtype)
    return w[:, ahead:ahead + cols]


def _list(t):
    return None if t is None else t.cpu().numpy()


class Streams:
    """lens: rows of each stream (None: one a stream, without offsets).  Some states are zeros (no slot, or no past), some go nowhere; `behind`: rows that no stream has."""

    def __init__(self, rng, lens, n=None, in_place=False, behind=0, ahead=0):
        n = len(lens) if lens is not None else n
        self.n, self.rows = n, (sum(lens) + ahead + behind if lens is not None else n)
        self.lens = lens if lens is not None else [1] * n
        self.offsets = None if lens is None else _i32(ahead + np.concatenate(([0], np.cumsum(lens))))
        self.pool = 2 * n + 3
        at = rng.permutation(self.pool)
        slots, into = at[:n].copy(), at[n:2 * n].copy()
        past = rng.integers(1, 99, n)
        if n > 4:
            slots[1], slots[2], past[3], past[4] = -1, self.pool, 0, -5
            into[n - 1] = -1
            if not in_place:
                into[n - 2] = self.pool + 7
        if in_place:
            into = slots.copy()
        self.slots, self.into, self.past = _i32(slots), None if in_place else _i32(into), _i32(past)
        self.keep = [i for b, m in enumerate(self.lens) for i in range(ahead + sum(self.lens[:b]), ahead + sum(self.lens[:b]) + m)]

    def kw(self):
        return dict(offsets=self.offsets, past=self.past, into=self.into)

    def plain(self):
        return dict(slots=_list(self.slots), offsets=_list(self.offsets), past=_list(self.past), into=_list(self.into))


# ---------------------------------------------------------------------------------------------------- state_conv
def _silu_error(s, e):
    """The error of SiLU(s) where s is off by e."""
    return 1.1 * e + np.abs(O.silu(s)) * (np.abs(s) + 8) * U + TINY


def _check_conv(rh, g, streams, channels, width, dtype, act=True, with_bias=True):
    x = _wide(g, streams.rows, channels, dtype)
    w = _randn(g, width, channels) / width ** 0.5
    bias = _randn(g, channels) if with_bias else None
    state = _randn(g, streams.pool, width - 1, channels, dtype=dtype)
    before = state.clone()
    room = torch.full((streams.rows, channels + 7), 5.0, device="cuda").to(dtype)
    out = room[:, 4:4 + channels]
    got = rh.state_conv(x, w, state, streams.slots, bias=bias, silu=act, out=out, **streams.kw())
    assert got.data_ptr() == out.data_ptr()
    plain = dict(bias=None if bias is None else _np(bias), **streams.plain())
    want, new = O.conv(_np(x), _np(w), _np(before), act=False, **plain)
    most = O.conv(np.abs(_np(x)), np.abs(_np(w)), np.abs(_np(before)), act=False, **{**plain, "bias": None if bias is None else np.abs(_np(bias))})[0]
    assert np.array_equal(_np(state), new)                          # inputs: bit for bit
    k = streams.keep
    tol = (width + 2) * U * most[k]
    y = want[k]
    if act:
        tol, y = _silu_error(y, tol), O.silu(y)
    tol = tol + HALF[dtype] * (np.abs(y) + tol)
    err = np.abs(_np(out)[k] - y)
    assert (err <= tol).all(), float((err / np.maximum(tol, TINY)).max())
    rest = np.setdiff1d(np.arange(streams.rows), k)
    assert (_np(room)[rest] == 5).all() and (_np(room)[:, :4] == 5).all() and (_np(room)[:, 4 + channels:] == 5).all()
    return x, w, bias, before


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("channels", [1, 3, 4, 7, 8, 9, 64, 515, 2048, 2051])
def test_conv_single_rows(rh, dtype, channels):
    for width in (2, 4, 7):
        _check_conv(rh, _gen(channels + width), Streams(np.random.default_rng(channels), None, 9), channels, width, dtype)
    _check_conv(rh, _gen(channels), Streams(np.random.default_rng(channels), None, 9, in_place=True), channels, 3, dtype)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("width", [2, 3, 4, 5, 6, 7, 8])
@pytest.mark.parametrize("channels", [5, 72])
def test_conv_many_rows(rh, dtype, width, channels):
    """Streams of no row, shorter than the window, around runs' ends; rows ahead of the first stream and behind the last stay."""
    lens = [0, 1, 2, 3, 6, 7, 8, 9, 15, 16, 17, 31, 32, 33, 40, 63, 64, 65, 100, 0, 5]
    for in_place in (False, True):
        _check_conv(rh, _gen(width), Streams(np.random.default_rng(width), lens, in_place=in_place, behind=5, ahead=2), channels, width, dtype)


@pytest.mark.parametrize("dtype", TYPES)
def test_conv_without_bias_or_activation(rh, dtype):
    for lens in ([40, 3], None):
        s = Streams(np.random.default_rng(1), lens, 2)
        _check_conv(rh, _gen(1), s, 33, 4, dtype, act=False, with_bias=False)
        _check_conv(rh, _gen(2), s, 33, 4, dtype, act=True, with_bias=False)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("n,longest,channels", [(1, 5000, 1024), (300, 90, 40), (2048, 12, 24), (37, 1500, 515)])
def test_conv_longer_runs_and_many_streams(rh, dtype, n, longest, channels):
    rng = np.random.default_rng(n)
    _check_conv(rh, _gen(n), Streams(rng, rng.integers(0, longest + 1, n).tolist(), in_place=n == 300), channels, 4, dtype)


@pytest.mark.parametrize("dtype", TYPES)
def test_conv_row_by_row_is_the_same(rh, dtype):
    """What a call gives of many rows, calls of a row each give too, bit for bit, and so do calls of any pieces."""
    g, rows, channels, width = _gen(4), 41, 100, 4
    x, w, bias = _randn(g, rows, channels, dtype=dtype), _randn(g, width, channels), _randn(g, channels)
    slot = _i32([1])
    states = [torch.full((3, width - 1, channels), 2.0, device="cuda").to(dtype) for _ in range(3)]
    whole = rh.state_conv(x, w, states[0], slot, bias=bias, offsets=_i32([0, rows]), past=_i32([0]))
    single = torch.cat([rh.state_conv(x[t:t + 1], w, states[1], slot, bias=bias, past=_i32([t])) for t in range(rows)])
    at = [0, 2, 3, 11, 40, 41]
    pieces = torch.cat([rh.state_conv(x[p:q], w, states[2], slot, bias=bias, offsets=_i32([0, q - p]), past=_i32([p])) for p, q in zip(at, at[1:])])
    assert torch.equal(whole, single) and torch.equal(whole, pieces)
    assert torch.equal(states[0], states[1]) and torch.equal(states[0], states[2])


# ---------------------------------------------------------------------------------------------------- state_scan
def _scan_inputs(g, streams, channels, n, groups, dtype, gate=True, skip=True, dt_bias=True, steps=(0.001, 0.1), spread=1.0):
    bc = _wide(g, streams.rows, 2 * groups * n, dtype)
    step = torch.exp(torch.rand(channels, generator=g, device="cuda") * np.log(steps[1] / steps[0]) + np.log(steps[0]))
    return dict(x=_wide(g, streams.rows, channels, dtype) , dt=_wide(g, streams.rows, channels, dtype, 1, 4) * spread,
                a=-torch.exp(torch.rand((channels, n), generator=g, device="cuda") * np.log(16.0)),
                b=bc[:, :groups * n].unflatten(1, (groups, n)), c=bc[:, groups * n:].unflatten(1, (groups, n)),
                state=_randn(g, streams.pool, channels, n), skip=_randn(g, channels) if skip else None,
                gate=_wide(g, streams.rows, channels, dtype) if gate else None, dt_bias=step + torch.log(-torch.expm1(-step)) if dt_bias else None)


def _scan_bounds(i, soft, streams, cut_rows):
    """The oracle's y and states, and how far off they may be (the recursion of the docstring)."""
    p = {k: None if v is None else _np(v) for k, v in i.items()}
    plain = streams.plain()
    y, new, most = O.scan(**p, soft=soft, **plain)
    y_tol, new_tol = np.zeros(y.shape), np.zeros(new.shape)
    offsets, slots, past, into = (plain[k] for k in ("offsets", "slots", "past", "into"))
    per = p["x"].shape[1] // p["b"].shape[1]
    for begin, end, old, to in O._streams(offsets, slots, past, into, p["state"].shape[0], p["x"].shape[0]):
        h = np.zeros(p["state"].shape[1:]) if old is None else np.array(p["state"][old])
        e = np.zeros(h.shape)
        for t in range(begin, end):
            raw = p["dt"][t] + (0 if p["dt_bias"] is None else p["dt_bias"])
            d = O.softplus(raw) if soft else raw
            e_d = ((np.abs(raw)[:, None] + 16) if soft else 2) * U + cut_rows * U
            power = np.abs(d[:, None] * p["a"])
            fade, add = np.exp(d[:, None] * p["a"]), (d * p["x"][t])[:, None] * np.repeat(p["b"][t], per, 0)
            e = fade * e + fade * np.abs(h) * (power * (e_d + 4 * U) + 4 * U) + np.abs(add) * (e_d + 4 * U)
            h = fade * h + add
            e += U * np.abs(h)
            c = np.repeat(p["c"][t], per, 0)
            tol = (np.abs(c) * e).sum(1) + (h.shape[1] + 4) * U * most[t]
            plain_y = (c * h).sum(1)
            if p["skip"] is not None:
                plain_y = plain_y + p["skip"] * p["x"][t]
                tol += 2 * U * np.abs(p["skip"] * p["x"][t]) + U * np.abs(plain_y)
            if p["gate"] is not None:
                z = p["gate"][t]
                tol = tol * np.abs(O.silu(z)) + np.abs(y[t]) * (np.abs(z) + 10) * U
            y_tol[t] = tol + TINY
        if to is not None:
            new_tol[to] = e + TINY
    return y, new, y_tol, new_tol


def _check_scan(rh, g, streams, channels, n, groups, dtype, soft=True, cut_rows=0, **kw):
    i = _scan_inputs(g, streams, channels, n, groups, dtype, **kw)
    y, new, y_tol, new_tol = _scan_bounds(i, soft, streams, cut_rows)
    room = torch.full((streams.rows, channels + 6), 5.0, device="cuda").to(dtype)
    out, state = room[:, 5:5 + channels], i.pop("state")
    before = state.clone()
    got = rh.state_scan(**i, state=state, slots=streams.slots, softplus=soft, out=out, **streams.kw())
    assert got.data_ptr() == out.data_ptr()
    k = streams.keep
    tol = y_tol[k] + HALF[dtype] * (np.abs(y[k]) + y_tol[k])
    err = np.abs(_np(out)[k] - y[k])
    assert (err <= tol).all(), ("y", float((err / tol).max()), np.argwhere(err > tol)[:4].tolist())
    err = np.abs(_np(state) - new)
    assert (err <= new_tol).all(), ("state", float((err / np.maximum(new_tol, TINY)).max()), np.argwhere(err > new_tol)[:4].tolist())
    rest = np.setdiff1d(np.arange(streams.rows), k)
    assert (_np(room)[rest] == 5).all() and (_np(room)[:, :5] == 5).all() and (_np(room)[:, 5 + channels:] == 5).all()
    return i, before, out, state


SIZES = [1, 3, 4, 5, 8, 13, 16, 20, 32, 33, 64, 100, 128]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("n", SIZES)
def test_scan_single_rows(rh, dtype, n):
    for channels, groups, in_place in ((1, 1, False), (66, 2, True), (300, 3, False)):
        _check_scan(rh, _gen(n), Streams(np.random.default_rng(n), None, 11, in_place=in_place), channels, n, groups, dtype)


@pytest.mark.parametrize("dtype", TYPES)
def test_scan_single_rows_of_many_streams(rh, dtype):
    for count in (1, 2, 3, 5, 3000):                                # several streams a thread, and what is left of them
        _check_scan(rh, _gen(count), Streams(np.random.default_rng(count), None, count), 520 if count == 3000 else 4500, 16, 1, dtype)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("n", SIZES)
def test_scan_many_rows(rh, dtype, n):
    """Streams of no row, of one, around stages' and fours' ends; rows of no stream stay."""
    lens = [0, 1, 2, 3, 4, 5, 7, 8, 9, 15, 16, 17, 31, 32, 33, 63, 64, 65, 0, 97]
    for channels, groups, in_place in ((5, 1, False), (150, 2, True)):
        _check_scan(rh, _gen(n), Streams(np.random.default_rng(n), lens, in_place=in_place, behind=4, ahead=3), channels, n, groups, dtype, cut_rows=0 if n <= 64 else 97)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("channels,groups", [(1, 1), (7, 7), (8, 1), (127, 1), (128, 1), (129, 1), (390, 3), (1032, 8)])
def test_scan_channel_layouts(rh, dtype, channels, groups):
    _check_scan(rh, _gen(channels), Streams(np.random.default_rng(channels), [33, 1, 70]), channels, 16, groups, dtype)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("lens,channels,n", [([2500], 40, 16), ([191], 12, 16), ([192], 12, 16), ([193], 12, 16), ([700, 1, 0, 300, 513, 40], 130, 16), ([1800, 5], 20, 64), ([3000], 9, 4),
                                             ([900, 1200], 20, 7), ([1500], 33, 128), ([4000], 6, 1)])
def test_scan_streams_that_are_cut(rh, dtype, lens, channels, n):
    """Chunks side by side: the same as one after the other, and the same bits on every run; in place too."""
    for in_place in (False, True):
        streams = Streams(np.random.default_rng(len(lens)), lens, in_place=in_place)
        i, before, out, state = _check_scan(rh, _gen(channels), streams, channels, n, 1, dtype, cut_rows=max(lens))
        first, after = out.clone(), state.clone()
        for _ in range(3):
            state.copy_(before)
            again = rh.state_scan(**i, state=state, slots=streams.slots, **streams.kw())
            assert torch.equal(again[streams.keep], first[streams.keep]) and torch.equal(state, after)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("n_streams,longest", [(64, 400), (65, 400), (700, 60), (2048, 20)])
def test_scan_many_streams(rh, dtype, n_streams, longest):
    rng = np.random.default_rng(n_streams)
    lens = rng.integers(0, longest + 1, n_streams)
    lens[n_streams // 2] = 5 * longest                               # one that is cut
    _check_scan(rh, _gen(n_streams), Streams(rng, lens.tolist()), 24, 16, 2, dtype, cut_rows=5 * longest)


@pytest.mark.parametrize("dtype", TYPES)
def test_scan_optional_inputs(rh, dtype):
    for lens in ([40, 300], None):
        s = Streams(np.random.default_rng(1), lens, 2)
        for gate in (False, True):
            for skip in (False, True):
                _check_scan(rh, _gen(1), s, 20, 16, 1, dtype, gate=gate, skip=skip, dt_bias=gate, cut_rows=300)
        _check_scan(rh, _gen(2), s, 20, 16, 1, dtype, soft=False, spread=0.05, dt_bias=False, cut_rows=300)      # steps of either sign as they are


@pytest.mark.parametrize("dtype", TYPES)
def test_scan_steps_of_any_size(rh, dtype):
    """dt from far below zero, where softplus is its exponential, to above 20, where it is the identity; states that fade at once, and not at all."""
    for lens in ([60, 250], None):
        s = Streams(np.random.default_rng(3), lens, 2)
        for spread, steps in ((30.0, (0.5, 2.0)), (0.1, (1e-6, 1e-4)), (3.0, (1e-3, 10.0))):
            _check_scan(rh, _gen(5), s, 30, 16, 1, dtype, spread=spread, steps=steps, cut_rows=250)


def test_scan_softplus_is_exact_over_its_range(rh):
    """y of one row from a state of zeros, x = b = c = 1, is softplus(dt): within e_d of the bounds, three roundings more."""
    dt = torch.cat((torch.linspace(-85, 90, 70001, device="cuda"), torch.linspace(-1e-3, 1e-3, 3001, device="cuda"), torch.linspace(19.9, 20.1, 2001, device="cuda"),
                    torch.linspace(-17.5, -16, 2001, device="cuda")))
    rows = dt.numel()
    one = torch.ones((rows, 1), device="cuda")
    y = rh.state_scan(one, dt[:, None].contiguous(), torch.zeros((1, 1), device="cuda"), one[:, None], one[:, None], torch.zeros((0, 1, 1), device="cuda"),
                      torch.full((rows,), -1, dtype=torch.int32, device="cuda"))
    want = O.softplus(_np(dt))
    err = np.abs(_np(y)[:, 0] - want) / want
    # dt is exact here: of e_d what the power, the logarithm, the quotient and the rounding of |dt| log2(e) take
    assert err.max() <= 19 * U, (err.max() / U, float(dt[int(err.argmax())]))


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("n", [13, 16])
def test_scan_infinities_are_what_the_formula_makes_of_them(rh, dtype, n):
    """An infinite input gives the infinity that the definition gives; it stays with its channel and its stream."""
    g, channels = _gen(9), 20
    for lens, at in (([30, 30, 300], 5), (None, 0)):
        s = Streams(np.random.default_rng(0), lens, 3)
        i = _scan_inputs(g, s, channels, n, 1, dtype)
        i = {k: v if v is None else v.clone() for k, v in i.items()}
        i["b"], i["c"] = i["b"].abs() + 0.1, i["c"].abs() + 0.1
        i["gate"] = None
        i["skip"] = i["skip"].abs() + 0.1
        i["x"][at, 3] = float("inf")
        rows = [at] if lens is None else list(range(at, 30))
        state = i.pop("state")
        y = rh.state_scan(**i, state=state, slots=s.slots, **s.kw())
        bad = torch.isposinf(y.float())
        want = torch.zeros_like(bad)
        want[rows, 3] = True
        # one row on, the skip's infinity is gone and the state's stays
        assert torch.equal(bad, want) and bool(torch.isfinite(y.float()[~want]).all())
        kept = (s.slots if s.into is None else s.into).tolist()
        assert bool(torch.isposinf(state[kept[0], 3]).all()) and int((~torch.isfinite(state)).sum()) == n


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("n", [5, 13, 16, 100])
def test_scan_infinities_reach_the_chunks_behind(rh, dtype, n):
    """In a stream that is cut, also where a chunk fades to nothing: the state and every later row are infinite, as step by step; other channels stay finite."""
    channels, rows, at = 9, 1500, 40
    s = Streams(np.random.default_rng(0), [rows])
    i = _scan_inputs(_gen(9), s, channels, n, 1, dtype, gate=False, skip=False, steps=(0.05, 2.0), spread=0.1)
    i = {k: v if v is None else v.clone() for k, v in i.items()}
    i["b"], i["c"] = i["b"].abs() + 0.1, i["c"].abs() + 0.1
    i["x"][at, 3] = float("inf")
    state = i.pop("state")
    y = rh.state_scan(**i, state=state, slots=s.slots, **s.kw()).float()
    assert bool(torch.isposinf(y[at:, 3]).all()) and bool(torch.isfinite(y[:at, 3]).all())
    assert bool(torch.isfinite(y[:, [c for c in range(channels) if c != 3]]).all())
    kept = state[int(s.into[0])]
    assert bool(torch.isposinf(kept[3]).all()) and int((~torch.isfinite(kept)).sum()) == n


@pytest.mark.parametrize("dtype", TYPES)
def test_scan_row_by_row_is_the_same(rh, dtype):
    """Rows in one call, in calls of pieces and of a row each: within the bounds of each other."""
    rows, channels, n = 90, 70, 16
    s = Streams(np.random.default_rng(0), [rows])
    i = _scan_inputs(_gen(3), s, channels, n, 1, dtype)
    y, new, y_tol, new_tol = _scan_bounds(i, True, s, 0)
    state, slot, into = i.pop("state"), s.slots, s.into
    parts = {k: i[k] for k in ("x", "dt", "b", "c", "gate")}
    rest = {k: v for k, v in i.items() if k not in parts}
    for at in (list(range(rows + 1)), [0, 1, 4, 33, 64, 90]):
        mine, got = state.clone(), []
        for p, q in zip(at, at[1:]):
            one = dict(offsets=None) if q - p == 1 and len(at) > 10 else dict(offsets=_i32([0, q - p]))
            got.append(rh.state_scan(**{k: v[p:q] for k, v in parts.items()}, **rest, state=mine, slots=slot if p == 0 else into, into=into, **one))
        err = np.abs(_np(torch.cat(got)) - y)
        assert (err <= y_tol + HALF[dtype] * (np.abs(y) + y_tol)).all()
        k = int(into[0])
        assert (np.abs(_np(mine[k]) - new[k]) <= new_tol[k]).all()


# ---------------------------------------------------------------------------------------------------- norm_gated
def _check_gated(rh, x, z, w, groups, eps, outputs):
    want = O.gated_norm(_np(x), _np(z), _np(w), groups, eps)
    want_sc = np.maximum(np.abs(want).max(-1), S.AMAX_MIN) / 448
    y, y8, sc = rh.norm_gated(x, z, w, groups=groups, eps=eps, outputs=outputs)
    per = x.shape[1] // groups
    rel = (per / 2 + 2 * (np.abs(_np(z)).max() + 8) + 8) * U
    bar = rel * np.abs(want) + TINY
    assert (y is None) == (outputs == "e4m3") and (y8 is None) == (sc is None) == (outputs == "same")
    if outputs != "e4m3":
        assert (np.abs(_np(y) - want) <= bar + HALF[x.dtype] * np.abs(want) * (1 + 1e-4)).all()
    if outputs != "same":
        assert (np.abs(_np(sc) - want_sc) <= (rel + 6 * U) * want_sc).all()
        q = want / want_sc[:, None]
        # half a step of the code, of a quotient that is off by that much: a step more where it lies at a tie
        tol = np.maximum(np.abs(q) * 2.0 ** -4, 2.0 ** -10) * (1 + 1e-3) + 448 * (2 * rel + 8 * U)
        assert (np.abs(_np(y8) - q) <= tol).all()
        assert (np.abs(_np(y8)).max(-1) == 448)[np.abs(want).max(-1) > 1e-20].all()        # of a row of zeros nothing is 448


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,cols,groups", [(1, 1, 1), (5, 6, 6), (3, 6, 2), (4, 64, 1), (7, 60, 4), (9, 2048, 8), (3, 2048, 1), (300, 96, 3), (5, 1540, 4), (2, 1023, 33), (2, 1024, 1024), (2, 32768, 1),
                                              (2, 32768, 2), (2, 32768, 4), (2, 32768, 32), (2, 32768, 64), (2, 32768, 128), (2, 32768, 1024), (2, 32767, 7), (2, 32767, 151), (2, 32760, 3), (2, 16384, 32),
                                              (2, 2145, 33), (2, 16384, 1), (2, 16384, 2), (2, 16384, 64), (2, 513, 1), (3, 4097, 1), (3, 5000, 5), (1000, 24, 2)])
def test_gated_norm(rh, dtype, rows, cols, groups):
    g = _gen(cols + groups)
    x, z, w = _wide(g, rows, cols, dtype), _wide(g, rows, cols, dtype, 6, 1), 1 + 0.2 * _randn(g, cols)
    for outputs in ("same", "e4m3", "both"):
        _check_gated(rh, x, z, w, groups, 1e-6, outputs)


def test_gated_norm_extreme_rows(rh):
    g = _gen(1)
    x, z, w = _randn(g, 6, 96), _randn(g, 6, 96), torch.ones(96, device="cuda")
    x[0] = 0                                                         # zeros
    z[1] = -60.0                                                     # a gate that is all but shut: products of 1e-24, below eps
    x[2] *= 1e15
    x[3, 5] = float("nan")
    y, y8, sc = rh.norm_gated(x, z, w, groups=3, outputs="both")
    assert bool((y[0] == 0).all()) and bool((y8[0].float() == 0).all())
    ok = [0, 1, 2, 4, 5]
    _check_gated(rh, x[ok], z[ok], w, 3, 1e-6, "both")
    assert bool(y[3, :32].isnan().all()) and bool(torch.isfinite(y[3, 32:]).all())       # its group
    assert bool(sc[3].isnan()) and bool(y8[3].float().isnan().all())                     # and its row's scale


# ---------------------------------------------------------------------------------------------------- sizes, streams, graphs, refusals
def test_offsets_past_32_bits(rh):
    """States and rows whose elements lie beyond 2^32 bytes and 2^31 elements."""
    g, channels, n = _gen(0), 4096, 128
    pool = 2 ** 31 // (channels * n) + 3
    state = torch.zeros((pool, channels, n), device="cuda")
    conv_pool = 2 ** 31 // (3 * channels) + 3
    conv_state = torch.zeros((conv_pool, 3, channels), dtype=torch.bfloat16, device="cuda")
    wide = 2 ** 31 // 3 + 64
    rows = torch.zeros(3 * wide + channels, dtype=torch.bfloat16, device="cuda").as_strided((4, channels), (wide, 1))
    rows.copy_(_randn(g, 4, channels))
    near = rows.clone()
    i = _scan_inputs(g, Streams(np.random.default_rng(0), [4]), channels, n, 1, torch.bfloat16, gate=False)
    small = torch.zeros((2, channels, n), device="cuda")
    small[0] = state[pool - 2] = _randn(g, channels, n)
    args = {k: i[k] for k in ("dt", "a", "b", "c", "skip", "dt_bias")}
    for offsets, m in ((_i32([0, 4]), 1), (None, 4)):
        slots = [pool - 2] * m
        into = [pool - 1] + [-1] * (m - 1)
        far = rh.state_scan(rows, state=state, slots=_i32(slots), into=_i32(into), offsets=offsets, **args)
        want = rh.state_scan(near, state=small, slots=_i32([0] * m), into=_i32([1] + [-1] * (m - 1)), offsets=offsets, **args)
        assert torch.equal(far, want) and torch.equal(state[pool - 1], small[1])
    w = _randn(g, 4, channels)
    kept = torch.zeros((2, 3, channels), dtype=torch.bfloat16, device="cuda")
    kept[0] = conv_state[conv_pool - 2] = _randn(g, 3, channels).to(torch.bfloat16)
    for offsets, m in ((_i32([0, 4]), 1), (None, 4)):
        far = rh.state_conv(rows, w, conv_state, _i32([conv_pool - 2] * m), into=_i32([conv_pool - 1] + [-1] * (m - 1)), offsets=offsets)
        want = rh.state_conv(near, w, kept, _i32([0] * m), into=_i32([1] + [-1] * (m - 1)), offsets=offsets)
        assert torch.equal(far, want) and torch.equal(conv_state[conv_pool - 1], kept[1])
    ones = torch.ones(channels, device="cuda")
    assert torch.equal(rh.norm_gated(rows, rows, ones)[0], rh.norm_gated(near, near, ones)[0])


@pytest.mark.parametrize("n_streams", [3, 100])
def test_offsets_that_descend(n_streams):
    """They write nothing, not the counters between workgroups either: a stream that is cut in a call after them comes out right.  Offsets beyond the rows count as their ends."""
    rh, fresh = _context(), _context()
    g, channels, rows = _gen(0), 24, 2000
    guard = torch.full((rows + 20, channels), 5.0, device="cuda")
    out = guard[10:10 + rows]
    x, w, state = _randn(g, rows, channels), _randn(g, 4, channels), torch.full((n_streams, 3, channels), 3.0, device="cuda")
    s = Streams(np.random.default_rng(0), [rows])
    i = _scan_inputs(g, s, channels, 16, 1, torch.float32)
    i["state"] = torch.full((n_streams, channels, 16), 3.0, device="cuda")
    rng, slots = np.random.default_rng(1), _i32(np.arange(n_streams))
    for k in range(6):
        offsets = rng.integers(-2 ** 31, 2 ** 31 - 1, n_streams + 1) if k < 2 else rng.integers(-50, rows + 50, n_streams + 1)
        if k == 4:
            offsets = np.array([0, rows] * (n_streams // 2 + 1))[:n_streams + 1]         # every other stream has all rows
        if k == 5:
            offsets = np.concatenate((np.arange(n_streams), [0]))                        # the last one alone
        offsets[-2:] = np.clip(offsets[-2:], 1, rows)
        offsets[-1] = offsets[-2] - 1                                                    # some descend for certain
        print("offsets", k, offsets[:4].tolist(), flush=True)
        rh.state_conv(x, w, state, slots, offsets=_i32(offsets), out=out)
        rh.state_scan(**i, slots=slots, offsets=_i32(offsets), out=out)
        torch.cuda.synchronize()
        assert bool((guard == 5).all()) and bool((state == 3).all()) and bool((i["state"] == 3).all())
    offsets = np.zeros(n_streams + 1, int)
    offsets[0], offsets[1:] = -7, rows + 9                                               # the first stream has all, from below the first row to behind the last
    want = np.zeros(n_streams + 1, int)
    want[1:] = rows
    for c in (rh, fresh):
        c.state_scan(**i, slots=_i32(np.full(n_streams, -1)), offsets=_i32(want))        # the scratch memory is there
    a = rh.state_scan(**i, slots=_i32(np.full(n_streams, -1)), offsets=_i32(offsets)), rh.state_conv(x, w, state, _i32(np.full(n_streams, -1)), offsets=_i32(offsets))
    b = fresh.state_scan(**i, slots=_i32(np.full(n_streams, -1)), offsets=_i32(want)), fresh.state_conv(x, w, state, _i32(np.full(n_streams, -1)), offsets=_i32(want))
    assert all(torch.equal(p, q) for p, q in zip(a, b))


def _layer(rh, g, channels, n, dtype):
    """A layer's three calls together on rows in hand; -> step(x, gate, dt, b, c, states, slots, offsets, past)."""
    w, bias = _randn(g, 4, channels) / 2, _randn(g, channels)
    a, skip, weight = -torch.exp(_randn(g, channels, n)), _randn(g, channels), torch.ones(channels, device="cuda")

    def step(t, conv_state, state, slots, **kw):
        x = rh.state_conv(t["x"], w, conv_state, slots, bias=bias, **kw)
        y = rh.state_scan(x, t["dt"], a, t["b"], t["c"], state, slots, skip=skip, **kw)
        return rh.norm_gated(y, t["gate"], weight, groups=2, outputs="both")
    return step


def _layer_inputs(g, rows, channels, n, dtype):
    return dict(x=_randn(g, rows, channels, dtype=dtype), gate=_randn(g, rows, channels, dtype=dtype), dt=_randn(g, rows, channels, dtype=dtype),
                b=_randn(g, rows, 1, n, dtype=dtype), c=_randn(g, rows, 1, n, dtype=dtype))


@pytest.mark.parametrize("lens", [None, [300, 2, 70]])
def test_a_captured_layer_replays_what_the_calls_give(rh, lens):
    channels, n, dtype, streams = 96, 16, torch.bfloat16, 3
    g = _gen(0)
    step = _layer(rh, g, channels, n, dtype)
    rows = sum(lens) if lens else streams
    kw = dict(offsets=_i32(np.concatenate(([0], np.cumsum(lens)))) if lens else None)
    slots = _i32([2, 0, 3])
    side, main = torch.cuda.Stream(), torch.cuda.current_stream()
    state = lambda: (torch.zeros((4, 3, channels), dtype=dtype, device="cuda"), torch.zeros((4, channels, n), device="cuda"))  # noqa: E731
    eager, cap, past, fixed = state(), state(), _i32([0, 0, 0]), _layer_inputs(g, rows, channels, n, dtype)
    step(fixed, *state(), slots, past=past, **kw)                    # the scratch memory is there
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    rh.set_stream(side)
    try:
        with torch.cuda.graph(graph, stream=side):
            got = step(fixed, *cap, slots, past=past, **kw)
    finally:
        rh.set_stream(main)
    for k in range(5):
        new = _layer_inputs(g, rows, channels, n, dtype)
        for key, t in fixed.items():
            t.copy_(new[key])
        past.fill_(k)
        graph.replay()
        want = step(new, *eager, slots, past=past, **kw)
        torch.cuda.synchronize()
        assert all(torch.equal(p.view(torch.uint8), q.view(torch.uint8)) for p, q in zip(got, want)), k
        assert all(torch.equal(p, q) for p, q in zip(cap, eager)), k


def test_the_first_call_that_cuts_a_stream_allocates(rh):
    """In a capture it is refused; the calls that need no memory are recorded."""
    fresh, side, main = _context(), torch.cuda.Stream(), torch.cuda.current_stream()
    g = _gen(0)
    t = _layer_inputs(g, 900, 96, 16, torch.bfloat16)
    state, a = torch.zeros((1, 96, 16), device="cuda"), -torch.ones((96, 16), device="cuda")
    call = lambda rows: fresh.state_scan(t["x"][:rows], t["dt"][:rows], a, t["b"][:rows], t["c"][:rows], state, _i32_at, offsets=offsets, past=_zero)  # noqa: E731
    _i32_at, offsets, _zero = _i32([0]), _i32([0, 900]), _i32([0])
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    fresh.set_stream(side)
    try:
        with torch.cuda.graph(graph, stream=side):
            short = call(100)
            with pytest.raises(RhError, match="capture") as e:
                call(900)
            assert e.value.status == 6
    finally:
        fresh.set_stream(main)
    graph.replay()
    want = call(100)
    torch.cuda.synchronize()
    assert torch.equal(short, want)
    assert bool(torch.isfinite(call(900).float()).all())


def test_on_another_stream_and_in_turn():
    side = torch.cuda.Stream()
    other, here = _context(stream=side), _context()
    g = _gen(0)
    t = _layer_inputs(g, 700, 96, 16, torch.bfloat16)
    slots, kw = _i32([0, 1]), dict(offsets=_i32([0, 500, 700]))
    state = lambda: (torch.zeros((2, 3, 96), dtype=torch.bfloat16, device="cuda"), torch.zeros((2, 96, 16), device="cuda"))  # noqa: E731
    p, q = state(), state()
    steps = [_layer(c, _gen(7), 96, 16, torch.bfloat16) for c in (other, here)]
    torch.cuda.synchronize()
    got = [steps[0](t, *p, slots, **kw) for _ in range(3)]           # its own calls follow each other
    want = [steps[1](t, *q, slots, **kw) for _ in range(3)]
    torch.cuda.synchronize()
    for a, b in zip(got, want):
        assert all(torch.equal(x.view(torch.uint8), y.view(torch.uint8)) for x, y in zip(a, b))
    assert all(torch.equal(a, b) for a, b in zip(p, q))


def test_empty_calls(rh):
    z = lambda *s: torch.zeros(s, device="cuda")  # noqa: E731
    none = torch.zeros(0, dtype=torch.int32, device="cuda")
    state, conv_state = torch.full((2, 8, 4), 3.0, device="cuda"), torch.full((2, 3, 8), 3.0, device="cuda")
    assert rh.state_conv(z(0, 8), z(4, 8), conv_state, none).shape == (0, 8)
    assert rh.state_scan(z(0, 8), z(0, 8), z(8, 4), z(0, 1, 4), z(0, 1, 4), state, none).shape == (0, 8)
    assert rh.norm_gated(z(0, 8), z(0, 8), z(8))[0].shape == (0, 8)
    # streams without rows keep their states, those without a past too
    rh.state_conv(z(0, 8), z(4, 8), conv_state, _i32([0, 1]), offsets=_i32([0, 0, 0]), past=_i32([0, 1]))
    rh.state_scan(z(0, 8), z(0, 8), z(8, 4), z(0, 1, 4), z(0, 1, 4), state, _i32([0, 1]), offsets=_i32([0, 0, 0]), past=_i32([0, 1]))
    assert bool((state == 3).all()) and bool((conv_state == 3).all())


def test_refusals(rh):
    INVALID, SHAPE, CAPACITY = 1, 2, 3
    z = lambda *s, dtype=torch.float32: torch.zeros(s, dtype=dtype, device="cuda")  # noqa: E731
    slots = _i32([0, 1])
    conv = lambda x=z(2, 8), w=z(4, 8), state=z(2, 3, 8), **kw: rh.state_conv(x, w, state, kw.pop("slots", slots), **kw)  # noqa: E731
    conv()
    _refused(SHAPE, conv, w=z(1, 8), state=z(2, 0, 8))
    _refused(SHAPE, conv, w=z(9, 8), state=z(2, 8, 8))
    _refused(SHAPE, conv, x=z(1, 8).expand(2, 8))
    _refused(INVALID, conv, x=z(2, 8).to(E4M3), state=z(2, 3, 8).to(E4M3))
    many = _i32(np.zeros(2049))
    _refused(CAPACITY, conv, x=z(3, 8), slots=many, offsets=_i32(np.zeros(2050)))

    def scan(x=z(2, 8), dt=z(2, 8), a=z(8, 4), b=z(2, 1, 4), c=z(2, 1, 4), state=z(2, 8, 4), **kw):
        return rh.state_scan(x, dt, a, b, c, state, kw.pop("slots", slots), **kw)
    scan()
    _refused(SHAPE, scan, b=z(2, 3, 4), c=z(2, 3, 4))
    _refused(SHAPE, scan, a=z(8, 0), b=z(2, 1, 0), c=z(2, 1, 0), state=z(2, 8, 0))
    _refused(SHAPE, scan, a=z(8, 129), b=z(2, 1, 129), c=z(2, 1, 129), state=z(2, 8, 129))
    _refused(SHAPE, scan, x=z(1, 8).expand(2, 8))
    _refused(SHAPE, scan, b=z(1, 1, 4).expand(2, 1, 4))
    _refused(INVALID, scan, x=z(2, 8).to(E4M3), dt=z(2, 8).to(E4M3), b=z(2, 1, 4).to(E4M3), c=z(2, 1, 4).to(E4M3))
    _refused(CAPACITY, scan, x=z(3, 8), dt=z(3, 8), b=z(3, 1, 4), c=z(3, 1, 4), slots=many, offsets=_i32(np.zeros(2050)))
    wide = 65537
    _refused(SHAPE, scan, x=z(2, wide), dt=z(2, wide), a=z(wide, 4), state=z(2, wide, 4))
    gated = lambda x=z(2, 12), gate=z(2, 12), w=z(12), **kw: rh.norm_gated(x, gate, w, **kw)  # noqa: E731
    gated()
    _refused(SHAPE, gated, groups=5)
    _refused(SHAPE, gated, groups=0)
    _refused(SHAPE, gated, groups=2 ** 40)
    _refused(SHAPE, gated, x=z(1, 32769), gate=z(1, 32769), w=z(32769))
    _refused(SHAPE, gated, x=z(1, 2050), gate=z(1, 2050), w=z(2050), groups=1025)
    _refused(SHAPE, gated, gate=z(1, 12).expand(2, 12))
    _refused(INVALID, gated, eps=-1.0)
    _refused(INVALID, gated, eps=float("nan"))
    _refused(INVALID, gated, x=z(2, 12).to(E4M3), gate=z(2, 12).to(E4M3))


class Neither:
    def __bool__(self):
        raise KeyError("neither")


def test_tensors_that_do_not_fit_are_refused_in_the_binding(rh):
    z = lambda *s, dtype=torch.float32: torch.zeros(s, dtype=dtype, device="cuda")  # noqa: E731
    slots, bf = _i32([0, 1]), torch.bfloat16
    x, w, cs, a, b, hs = z(2, 8), z(4, 8), z(2, 3, 8), z(8, 4), z(2, 1, 4), z(2, 8, 4)
    row = z(2, 24)
    out = torch.full((2, 8), 5.0, device="cuda")
    conv = lambda *v, **kw: rh.state_conv(*v, **{"out": out, **kw})  # noqa: E731
    scan = lambda *v, **kw: rh.state_scan(*v, **{"out": out, **kw})  # noqa: E731
    calls = [
        lambda: conv(x.cpu(), w, cs, slots), lambda: conv(x.t(), w, cs, slots), lambda: conv(x, w.to(bf), cs, slots), lambda: conv(x, w[:, :7], cs, slots),
        lambda: conv(x, w, cs.to(bf), slots), lambda: conv(x, w, cs[:, :2], slots), lambda: conv(x, w, z(2, 8, 3).transpose(1, 2), slots), lambda: conv(x, w, cs, slots.long()),
        lambda: conv(x, w, cs, slots[:1]), lambda: conv(x, w, cs, slots, bias=z(7)), lambda: conv(x, w, cs, slots, offsets=slots), lambda: conv(x, w, cs, slots, past=slots[:1]),
        lambda: conv(x, w, cs, slots, into=slots.long()), lambda: conv(x, w, cs, slots, out=out.to(bf)), lambda: conv(x, w, cs, slots, out=out[:1]), lambda: conv(x, w, cs, slots, out=x), lambda: conv(x, w, cs, slots, out=cs.view(-1)[16:32].view(2, 8)),
        lambda: conv(row[:, :8], w, cs, slots, out=row[:, 7:15]), lambda: conv([1.0], w, cs, slots),
        lambda: scan(x, x.to(bf), a, b, b, hs, slots), lambda: scan(x, x, a[:7], b, b, hs, slots), lambda: scan(x, x, a, b[:1], b, hs, slots), lambda: scan(x, x, a, b, b[..., :3], hs, slots),
        lambda: scan(x, x, a, b.to(bf), b.to(bf), hs, slots), lambda: scan(x, x, a, b[:, 0], b[:, 0], hs, slots), lambda: scan(x, x, a, b, b, hs.to(bf), slots), lambda: scan(x, x, a, b, b, hs[..., :3], slots),
        lambda: scan(x, x, a, z(2, 4, 1).transpose(1, 2)[..., :4].expand(2, 1, 4)[:, :, ::2], b, hs, slots), lambda: scan(x, x, a, b, b, hs, slots[:1]), lambda: scan(x, x, a, b, b, hs, slots, skip=z(7)),
        lambda: scan(x, x, a, b, b, hs, slots, gate=x[:1]), lambda: scan(x, x, a, b, b, hs, slots, dt_bias=z(8, dtype=bf)), lambda: scan(x, x, a, b, b, hs, slots, out=x), lambda: scan(x, x, a, row[:, 4:8].unflatten(1, (1, 4)), b, hs, slots, out=row[:, :8]),
        lambda: scan(x, x, a, b, row[:, 7:11].unflatten(1, (1, 4)), hs, slots, out=row[:, :8]), lambda: scan(x, x, a, b, b, hs, slots, out=hs.view(-1)[8:24].view(2, 8)),
        lambda: scan(x, z(2, 8), a, b, b, hs, slots, gate=row[:, :8], out=row[:, 4:12]), lambda: scan(x, x, a, b, b, hs, slots, offsets=_i32([0, 1])),
        lambda: rh.norm_gated(x, x[:1], z(8)), lambda: rh.norm_gated(x, x.to(bf), z(8)), lambda: rh.norm_gated(x, x, z(7)), lambda: rh.norm_gated(x, x, z(8), outputs="bf16"), lambda: rh.norm_gated(x.t(), x.t(), z(2)),
    ]
    for k, call in enumerate(calls):
        with pytest.raises(AssertionError):
            call()
            print("call", k, "was taken")
    with pytest.raises(TypeError):
        rh.norm_gated(x, x, z(8), eps="1")
    with pytest.raises(KeyError):
        conv(x, w, cs, slots, silu=Neither())
    with pytest.raises(KeyError):
        scan(x, x, a, b, b, hs, slots, softplus=Neither())
    handle, device = rh._ctx
    rh._ctx = (handle, device + 1)
    for call in (lambda: conv(x, w, cs, slots), lambda: scan(x, x, a, b, b, hs, slots), lambda: rh.norm_gated(x, x, z(8))):
        with pytest.raises(AssertionError, match="another device"):
            call()
    rh._ctx = (handle, device)
    torch.cuda.synchronize()
    assert bool((out == 5).all())
    # columns of the same rows side by side are apart
    side = rh.state_conv(row[:, :8], w, cs, slots, out=row[:, 8:16])
    assert side.data_ptr() == row[:, 8:16].data_ptr()
    side = rh.state_scan(row[:, :8], x, a, row[:, 16:20].unflatten(1, (1, 4)), row[:, 20:].unflatten(1, (1, 4)), hs, slots, out=row[:, 8:16])
    assert side.data_ptr() == row[:, 8:16].data_ptr()


def test_results_do_not_change_from_run_to_run(rh):
    g = _gen(2)
    t = _layer_inputs(g, 3000, 200, 16, torch.bfloat16)
    step, slots, kw = _layer(rh, g, 200, 16, torch.bfloat16), _i32([0, 1, 2]), dict(offsets=_i32([0, 2500, 2501, 3000]), past=_i32([0, 0, 0]))
    runs = []
    for _ in range(4):
        states = torch.zeros((3, 3, 200), dtype=torch.bfloat16, device="cuda"), torch.zeros((3, 200, 16), device="cuda")
        runs.append([v.clone().view(torch.uint8) for v in (*step(t, *states, slots, **kw), *states)])
    assert all(torch.equal(p, q) for r in runs[1:] for p, q in zip(runs[0], r))


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("n", [5, 16])
def test_scan_decays_of_the_largest_size(rh, dtype, n):
    """a of -3e38: a step of 0 leaves the state, one of 1 leaves nothing of it; rows behind a stream's last are no steps."""
    channels, low = 6, -3e38
    for lens in ([5, 2, 301], [801], None):
        s = Streams(np.random.default_rng(2), lens, 3)
        i = _scan_inputs(_gen(4), s, channels, n, 1, dtype, dt_bias=False, gate=False, skip=False)
        i = {k: v if v is None else v.clone() for k, v in i.items()}
        i["a"] = torch.full_like(i["a"], low)
        i["dt"] = (torch.rand(i["dt"].shape, generator=_gen(6), device="cuda") < 0.2).to(dtype)
        state = i.pop("state")
        p = {k: None if v is None else _np(v) for k, v in i.items()}
        want, new, most = O.scan(**p, state=_np(state), soft=False, **s.plain())
        y = rh.state_scan(**i, state=state, slots=s.slots, softplus=False, **s.kw())
        k = s.keep
        # the state is a product rounded once or what it was: U; n products and sums of y, and its own rounding
        assert (np.abs(_np(y)[k] - want[k]) <= (n + 4) * U * most[k] + HALF[dtype] * np.abs(want[k]) * (1 + 2 * n * U) + 2 * n * U * most[k] + TINY).all()
        assert (np.abs(_np(state) - new) <= 2 * U * np.abs(new) + TINY).all()


@pytest.mark.parametrize("n", [5, 16])
def test_scan_states_that_grow_past_the_powers(rh, n):
    """a above 0 over chunks whose power passes 2^128: a state of zeros stays so until something is added, a small one grows to what it is step by step."""
    channels, rows = 3, 400                                          # chunks of 64 rows; exp(2 * 60) passes 2^128
    s = Streams(np.random.default_rng(2), [rows])
    i = _scan_inputs(_gen(4), s, channels, n, 1, torch.float32, dt_bias=False, gate=False, skip=False)
    i = {k: v if v is None else v.clone() for k, v in i.items()}
    i["a"] = torch.full_like(i["a"], 1.0)
    i["dt"] = torch.zeros_like(i["dt"])
    i["dt"][:60, 0], i["dt"][:, 1], i["dt"][:, 2] = 2.0, 2.0, 0.0
    i["x"][:-1] = 0
    state = torch.zeros_like(i.pop("state"))
    state[int(s.slots[0]), 0] = 1e-30
    p = {k: None if v is None else _np(v) for k, v in i.items()}
    want, new, most = O.scan(**p, state=_np(state), soft=False, **s.plain())
    assert np.isfinite(want).all()
    y = rh.state_scan(**i, state=state, slots=s.slots, softplus=False, **s.kw())
    # a step's power: its argument, 2 log2(e), rounded with log2(e) and as a product, 4 U of the power; 2 U from the power, 1 as it is multiplied.  A chunk's: its sum is exact, the
    # argument of a half 60 log2(e), 120 U of it, twice.  8 a step are above either.
    assert (np.abs(_np(y) - want) <= (60 * 8 + n + 4) * U * most + TINY).all()
    assert (np.abs(_np(state) - new) <= (60 * 8 + 4) * U * np.abs(new) + TINY).all()
