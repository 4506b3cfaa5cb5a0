"""What the entry points of rh_state_conv, rh_state_scan and rh_norm_gated do on the host: null arguments, refusals, launches, allocations, captures, a lost launch (no GPU; the
recording stand-in of test_host_calls takes the place of the HIP runtime)."""
import numpy as np
import pytest

from oracle import state as O
from test_host_capture import run_child  # noqa: F401  (the fixture, whose stream says whether it is being captured)

SETUP = '''
class Rows(C.Structure):
    _fields_ = [("offsets", C.c_void_p), ("slots", C.c_void_p), ("into", C.c_void_p), ("past", C.c_void_p), ("n_streams", C.c_int32), ("n_rows", C.c_int32), ("n_slots", C.c_int32)]
class Scan(C.Structure):
    _fields_ = [(k, C.c_void_p) for k in ("x", "dt", "gate", "b", "c")] + [(k + "_stride", C.c_int64) for k in ("x", "dt", "gate", "b", "c")] + \\
               [(k, C.c_void_p) for k in ("a", "dt_bias", "skip")] + [(k, C.c_int32) for k in ("type", "channels", "groups", "n", "softplus")]
L.rh_state_conv.argtypes = [C.c_void_p, C.c_void_p, C.c_void_p, C.c_int64, C.c_void_p, C.c_void_p, C.c_int32, C.c_int32, C.c_int32, C.c_int32, C.c_void_p, C.c_void_p, C.c_int64]
L.rh_state_scan.argtypes = [C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p, C.c_int64]
L.rh_norm_gated.argtypes = [C.c_void_p, C.c_void_p, C.c_int64, C.c_void_p, C.c_int64, C.c_void_p, C.c_int32, C.c_int32, C.c_int32, C.c_int32, C.c_float, C.c_void_p, C.c_void_p, C.c_void_p]
def rows(n=8, m=None, **kw):
    return Rows(**{**dict(offsets=None if m is None else 9 << 24, slots=1 << 24, into=None, past=None, n_streams=n, n_rows=n if m is None else m, n_slots=20), **kw})
def inputs(**kw):
    return Scan(**{**dict(x=2 << 24, dt=3 << 24, gate=4 << 24, b=5 << 24, c=6 << 24, x_stride=96, dt_stride=96, gate_stride=96, b_stride=32, c_stride=32, a=7 << 24, dt_bias=None, skip=None,
                          type=1, channels=96, groups=2, n=16, softplus=1), **kw})
conv = lambda r=None, t=1, ch=96, w=4, xs=96, ys=96, x=P(2), y=P(5), weight=P(3), state=P(4): L.rh_state_conv(ctx, C.byref(r or rows()), x, xs, weight, None, t, ch, w, 1, state, y, ys)
scan = lambda r=None, i=None, ys=96, state=P(8), y=P(10): L.rh_state_scan(ctx, C.byref(r or rows()), C.byref(i or inputs()), state, y, ys)
long = lambda: scan(rows(3, 5000))
gated = lambda t=1, n=8, cols=96, groups=2, eps=1e-6, xs=96, zs=96, y=P(4), y8=P(5), sc=P(6): L.rh_norm_gated(ctx, P(1), xs, P(2), zs, P(3), t, n, cols, groups, eps, y, y8, sc)
'''


def test_null_contexts_are_rejected():
    import paper_2407_16990_amd as pkg
    lib = pkg.load_library()
    assert lib.rh_state_conv(None, None, None, 1, None, None, 0, 1, 2, 0, None, None, 1) == 1
    assert lib.rh_state_scan(None, None, None, None, None, 1) == 1
    assert lib.rh_norm_gated(None, None, 1, None, 1, None, 0, 1, 1, 1, 0.0, None, None, None) == 1


def test_refusals_launch_nothing(run_child):  # noqa: F811
    run_child(SETUP + '''
INVALID, SHAPE, CAPACITY = 1, 2, 3
ok = [lambda: conv(), lambda: conv(rows(8, 100)), lambda: scan(), lambda: scan(rows(8, 100)), lambda: gated(), lambda: gated(y=None), lambda: gated(y8=None, sc=None),
      lambda: conv(rows(n_slots=0), state=None), lambda: scan(rows(n_slots=0), state=None), lambda: conv(rows(0)), lambda: scan(rows(0)), lambda: gated(n=0),
      lambda: scan(rows(5000)), lambda: conv(rows(5000)), lambda: scan(rows(2048, 100)), lambda: scan(i=inputs(gate=None, gate_stride=0)),
      lambda: L.rh_state_scan(ctx, C.byref(rows(0, 0)), C.byref(inputs(x=None)), None, None, 96)]
for k, f in enumerate(ok): assert f() == 0, (k, L.rh_last_error(ctx))
bad = [(INVALID, lambda: L.rh_state_conv(ctx, None, P(2), 96, P(3), None, 1, 96, 4, 1, P(4), P(5), 96)), (INVALID, lambda: conv(x=None)), (INVALID, lambda: conv(y=None)), (INVALID, lambda: conv(weight=None)),
       (INVALID, lambda: conv(state=None)), (INVALID, lambda: conv(rows(slots=None))), (INVALID, lambda: conv(t=2)), (INVALID, lambda: conv(t=7)), (SHAPE, lambda: conv(ch=0)), (SHAPE, lambda: conv(w=1)),
       (SHAPE, lambda: conv(w=9)), (SHAPE, lambda: conv(xs=95)), (SHAPE, lambda: conv(ys=95)), (SHAPE, lambda: conv(rows(8, n_rows=9))), (SHAPE, lambda: conv(rows(-1))), (SHAPE, lambda: conv(rows(n_slots=-1))),
       (CAPACITY, lambda: conv(rows(2049, 5000))), (SHAPE, lambda: conv(rows(2, 0x7FFF0001), ch=1)), (SHAPE, lambda: scan(rows(2, 0x7FFF0001))), (SHAPE, lambda: conv(rows(2 ** 31 - 1), ch=2 ** 20, xs=2 ** 20, ys=2 ** 20)), (SHAPE, lambda: conv(rows(8, -1))),
       (INVALID, lambda: L.rh_state_scan(ctx, None, C.byref(inputs()), P(8), P(10), 96)), (INVALID, lambda: L.rh_state_scan(ctx, C.byref(rows()), None, P(8), P(10), 96)),
       *[(INVALID, lambda k=k: scan(i=inputs(**{k: None}))) for k in ("x", "dt", "b", "c", "a")], (INVALID, lambda: scan(y=None)), (INVALID, lambda: scan(state=None)), (INVALID, lambda: scan(rows(slots=None))),
       (INVALID, lambda: scan(i=inputs(type=2))), (SHAPE, lambda: scan(i=inputs(channels=0))), (SHAPE, lambda: scan(i=inputs(channels=65537))), (SHAPE, lambda: scan(i=inputs(groups=0))),
       (SHAPE, lambda: scan(i=inputs(groups=5))), (SHAPE, lambda: scan(i=inputs(n=0))), (SHAPE, lambda: scan(i=inputs(n=129, b_stride=999, c_stride=999))), (SHAPE, lambda: scan(ys=95)),
       *[(SHAPE, lambda k=k: scan(i=inputs(**{k: 31 if k in ("b_stride", "c_stride") else 95}))) for k in ("x_stride", "dt_stride", "gate_stride", "b_stride", "c_stride")],
       (CAPACITY, lambda: scan(rows(2049, 5000))), (SHAPE, lambda: scan(rows(2 ** 31 - 1), inputs(channels=65536, x_stride=65536, dt_stride=65536, gate_stride=65536), 65536)),
       (INVALID, lambda: gated(t=2)), (SHAPE, lambda: gated(cols=0)), (SHAPE, lambda: gated(n=-1)), (SHAPE, lambda: gated(cols=32769, groups=1, xs=40000, zs=40000)), (SHAPE, lambda: gated(groups=0)),
       (SHAPE, lambda: gated(groups=7)), (SHAPE, lambda: gated(n=2 ** 31 - 1, cols=2048, groups=1, xs=2048, zs=2048)), (SHAPE, lambda: gated(cols=2050, groups=1025, xs=2050, zs=2050)), (SHAPE, lambda: gated(xs=95)), (SHAPE, lambda: gated(zs=95)), (INVALID, lambda: gated(eps=-1.0)),
       (INVALID, lambda: gated(eps=float("nan"))), (INVALID, lambda: gated(y8=None)), (INVALID, lambda: gated(sc=None)), (INVALID, lambda: gated(y=None, y8=None, sc=None))]
for k, (st, f) in enumerate(bad):
    rec.rec_reset()
    got = f()
    assert got == st and len(L.rh_last_error(ctx)) > 20 and not names(), (k, got, st, L.rh_last_error(ctx), names())
''')


def test_launches_and_memory(run_child):  # noqa: F811
    run_child(SETUP + '''
live = rec.rec_live()
rec.rec_reset()
for f in (conv, lambda: conv(rows(8, 5000)), scan, lambda: scan(rows(8, 100)), gated): assert f() == 0
assert len(names()) == 5 and rec.rec_mallocs() == 0 and rec.rec_syncs() == 0         # a launch a call, no memory
rec.rec_reset()
assert long() == 0 and rec.rec_mallocs() == 2 and len(names()) == 3 and "k_seq_zero" in names()[0], names()          # rows enough for a stream to be cut: scratch memory and counters
for again in range(2):
    rec.rec_reset()
    assert long() == 0 and scan(rows(700, 200000), inputs(channels=4096, groups=1, x_stride=4096, dt_stride=4096, gate_stride=4096), 4096) == 0 and attend() == 0
    assert rec.rec_mallocs() == 0 and rec.rec_syncs() == 0 and len(names()) == 5, names()
L.rh_destroy(ctx)
st, ctx = create(PLAIN, 4, 2, 2, 0)
L.rh_destroy(ctx)
assert rec.rec_live() == 0
''')


def test_a_captured_call_does_not_allocate(run_child):  # noqa: F811
    run_child(SETUP + '''
for status in (1, 2, -1):
    st, ctx = create(PLAIN, 4, 2, 2, 0)
    rec.rec_capture(status)
    rec.rec_reset()
    assert long() == 6 and b"capture" in L.rh_last_error(ctx) and not names() and rec.rec_mallocs() == 0
    for f in (conv, scan, gated, lambda: scan(rows(8, 100))): assert f() == 0
    rec.rec_capture(0)
    assert long() == 0
    rec.rec_capture(status)
    rec.rec_reset()
    assert long() == 0 and rec.rec_mallocs() == 0 and rec.rec_syncs() == 0
    rec.rec_capture(0)
''')


def test_a_lost_launch_is_reported_and_the_next_call_goes_on(run_child):  # noqa: F811
    run_child(SETUP + '''
assert long() == 0                                           # the counters are there
for f, n in ((conv, 1), (lambda: conv(rows(8, 500)), 1), (scan, 1), (long, 2), (gated, 1)):
    for k in range(n):
        rec.rec_reset(); rec.rec_fail_launch(k)
        assert f() == 4 and len(names()) == k and L.rh_last_error(ctx), (k, names())
    rec.rec_reset()
    assert f() == 0 and len(names()) == n
''')


def test_the_binding_looks_at_its_tensors():
    import torch

    from paper_2407_16990_amd import binding
    x, i = torch.zeros(2, 64), torch.zeros(2, dtype=torch.int32)
    for call in (lambda: binding._seq.state_conv((1, 0), x, x, x, i, None, None, None, None, True, None), lambda: binding._seq.state_conv(0, x),
                 lambda: binding._seq.state_scan((1, 0), x, x, x, x, x, x, i, None, None, None, True, None, None, None, None), lambda: binding._seq.norm_gated((1, 0), x, x, x[0], 1, 1e-6, "same"),
                 lambda: binding._seq.norm_gated((1, 0), x)):
        with pytest.raises(AssertionError):
            call()


# ---------------------------------------------------------------------------------------------------- the plain implementations themselves
def test_plain_conv_is_a_convolution():
    rng = np.random.default_rng(0)
    x, w, state = rng.standard_normal((9, 3)), rng.standard_normal((4, 3)), rng.standard_normal((2, 3, 3))
    y, new = O.conv(x, w, state, [1], bias=np.array([1.0, 2, 3]), offsets=[0, 9], act=False)
    for c in range(3):
        line = np.concatenate((state[1, :, c], x[:, c]))
        assert np.allclose(y[:, c], np.convolve(line, w[::-1, c], "valid") + c + 1)
    assert np.array_equal(new[1], x[-3:]) and np.array_equal(new[0], state[0])


def test_plain_scan_is_the_sum_it_stands_for():
    """h_t = sum_s exp(a sum of delta over (s, t]) delta_s x_s b_s, written out; a past of zeros, and one that counts."""
    rng = np.random.default_rng(1)
    T, D, N, G = 7, 4, 3, 2
    x, dt, b, c = rng.standard_normal((T, D)), rng.standard_normal((T, D)), rng.standard_normal((T, G, N)), rng.standard_normal((T, G, N))
    a, skip, gate, state = -rng.random((D, N)), rng.standard_normal(D), rng.standard_normal((T, D)), rng.standard_normal((1, D, N))
    for past in (0, 1):
        y, new, most = O.scan(x, dt, a, b, c, state, [0], skip=skip, gate=gate, offsets=[0, T], past=[past])
        d = np.log1p(np.exp(dt))
        total = np.cumsum(d, 0)
        for ch in range(D):
            for t in range(T):
                h = past * np.exp(a[ch] * total[t, ch]) * state[0, ch] + sum(np.exp(a[ch] * (total[t, ch] - total[s, ch])) * d[s, ch] * x[s, ch] * b[s, ch // 2] for s in range(t + 1))
                want = ((c[t, ch // 2] * h).sum() + skip[ch] * x[t, ch]) * gate[t, ch] / (1 + np.exp(-gate[t, ch]))
                assert abs(y[t, ch] - want) <= 1e-12 * (1 + most[t, ch])
            assert np.allclose(new[0, ch], h, rtol=1e-12)


def test_plain_streams_keep_to_their_slots():
    x, w, state = np.ones((5, 1)), np.ones((2, 1)), np.arange(4.0).reshape(4, 1, 1)
    y, new = O.conv(x, w, state, [3, 2, -1], offsets=[1, 3, 3, 4], past=[0, 1, 1], into=[0, 1, 2], act=False)
    assert np.isnan(y[[0, 4]]).all() and y[1:4, 0].tolist() == [1, 2, 1]
    assert new[:, 0, 0].tolist() == [1, 1, 1, 3]             # the second stream has no rows: its place stays


def test_plain_gated_norm():
    rng = np.random.default_rng(2)
    x, z, w = rng.standard_normal((3, 6)), rng.standard_normal((3, 6)), rng.standard_normal(6)
    y = O.gated_norm(x, z, w, 2, 0.5)
    s = x * z / (1 + np.exp(-z))
    for g in (slice(0, 3), slice(3, 6)):
        assert np.allclose(y[:, g], s[:, g] / np.sqrt((s[:, g] ** 2).sum(1, keepdims=True) / 3 + 0.5) * w[g])
