"""The largest calls of rh_state_scan, rh_state_conv and rh_norm_gated that one launch takes, and the next larger ones, which are refused before any work (no GPU; the recording
stand-in of test_host_calls takes the place of the HIP runtime, so nothing runs)."""
from test_host_capture import run_child  # noqa: F401  (the fixture)
from test_host_state import SETUP

WIDE = SETUP + '''
SHAPE, MOST = 2, 2 ** 24 - 1
def wide(ch, n, groups=1, **kw):
    return inputs(channels=ch, n=n, groups=groups, x_stride=ch, dt_stride=ch, gate_stride=ch, b_stride=groups * n, c_stride=groups * n, **kw)
def taken(f):
    rec.rec_reset()
    st = f()
    assert (st == 0) == (len(names()) > 0), (st, names())                # all of a call's work or none
    assert st in (0, SHAPE), (st, L.rh_last_error(ctx))
    if st: assert len(L.rh_last_error(ctx)) > 20
    return st == 0
'''


def test_single_rows(run_child):  # noqa: F811
    """Four streams a workgroup, of 1024 / m channels (8 of more than 64 states)."""
    run_child(WIDE + '''
assert taken(lambda: scan(rows(8192), wide(8192, 16), 8192))
assert taken(lambda: scan(rows(16384), wide(4096, 16), 4096))
for n, per in ((1, 256), (4, 256), (5, 128), (16, 64), (17, 32), (64, 16), (65, 8), (128, 8)):
    for ch in (65536, 65535, 4096):
        blocks = -(-ch // per)
        most = MOST // blocks * 4
        assert taken(lambda: scan(rows(most), wide(ch, n), ch)), (n, ch, most)
        assert not taken(lambda: scan(rows(most + 1), wide(ch, n), ch)), (n, ch, most)
''')


def test_many_rows(run_child):  # noqa: F811
    """A stream and a group's channels a workgroup; rows beyond the streams count where streams may be cut."""
    run_child(WIDE + '''
assert taken(lambda: scan(rows(2048, 2048), wide(65536, 1), 65536)) and taken(lambda: scan(rows(2048, 2 ** 31 - 2 ** 16), wide(65536, 16), 65536))
assert taken(lambda: scan(rows(1, 2 ** 31 - 2 ** 16), wide(1, 16), 1))
for groups, blocks in ((65536, 65536), (32768, 32768), (1, 4096)):
    most = min(2048, MOST // blocks)
    assert taken(lambda: scan(rows(most, 5000), wide(65536, 128, groups), 65536)), groups
    if most < 2048: assert not taken(lambda: scan(rows(most + 1, 5000), wide(65536, 128, groups), 65536)), groups
''')


def test_convolution_and_norm(run_child):  # noqa: F811
    run_child(WIDE + '''
ch = 8192                                                                # 1024 pieces of bf16
most = (2 ** 31 - 2 ** 12) // 1024
assert taken(lambda: conv(rows(most), ch=ch, xs=ch, ys=ch)) and not taken(lambda: conv(rows(most + 1), ch=ch, xs=ch, ys=ch))
assert taken(lambda: conv(rows(5, most * 16 - 80), ch=ch, xs=ch, ys=ch)) and not taken(lambda: conv(rows(5, most * 16 - 64), ch=ch, xs=ch, ys=ch))
most = (2 ** 32 - 1) // 1024                                             # 8192 columns of bf16 in a group: 512 lanes with two pieces
assert taken(lambda: gated(n=2 * most, cols=ch, groups=1, xs=ch, zs=ch)) and not taken(lambda: gated(n=2 * most + 2, cols=ch, groups=1, xs=ch, zs=ch))
''')
