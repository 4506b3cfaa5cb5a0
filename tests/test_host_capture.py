"""The sequence operators' own memory and stream capture: what a captured call may not allocate is refused, and what it may use is there and
cleared before any call counts on it (no GPU; the recording stand-in takes the place of the HIP runtime, here with a stream that says
whether it is being captured)."""
import subprocess
import sys

import pytest

from test_host_calls import HERE, PRELUDE
from test_host_sequence import SETUP

CAPTURE = '''
#include "recording_hip.cpp"
static int g_capture;
extern "C" {
void rec_capture(int status) { g_capture = status; }     // 0 none, 1 active, 2 invalidated, -1: a legacy stream beside another's capture
err_t hipStreamIsCapturing(void*, int* status) { *status = g_capture < 0 ? 0 : g_capture; return g_capture < 0 ? 906 : OK; }
}
'''


@pytest.fixture(scope="module")
def run_child(tmp_path_factory):
    from paper_2407_16990_amd import binding
    binding.load_library()
    d = tmp_path_factory.mktemp("rec")
    (d / "capture.cpp").write_text(CAPTURE)
    lib = str(d / "librecording_hip.so")
    subprocess.check_call(["g++", "-O1", "-std=c++17", "-Wall", "-shared", "-fPIC", "-I" + HERE, "-o", lib, str(d / "capture.cpp")])

    def run(body):
        r = subprocess.run([sys.executable, "-c", PRELUDE + SETUP + body + "\nprint('DONE')", lib, binding.lib_path()], capture_output=True, text=True, timeout=300)
        assert r.returncode == 0 and r.stdout.strip().endswith("DONE"), r.stdout[-2000:] + r.stderr[-3000:]
    return run


IN_PLACE = '''
in_place = lambda: L.rh_cache_plan(ctx, P(1), P(2), 8, 16, 100, 6, P(3), P(4), P(5), P(6), 100000, P(7), P(2), P(5))
'''


@pytest.mark.parametrize("status", [1, 2, -1])
def test_a_captured_call_does_not_allocate(run_child, status):
    run_child(IN_PLACE + f'''
rec.rec_capture({status})
for f in (attend, matvec, in_place):
    rec.rec_reset()
    assert f() == 6 and b"capture" in L.rh_last_error(ctx)               # RH_E_STATE
    assert not names() and rec.rec_mallocs() == 0 and rec.rec_syncs() == 0
for f in (plan, write, norm):                                            # these have no memory of their own
    assert f() == 0
rec.rec_capture(0)
for f in (attend, matvec, in_place): assert f() == 0
rec.rec_capture({status})
rec.rec_reset()
for f in (plan, write, attend, norm, matvec, in_place): assert f() == 0
assert rec.rec_mallocs() == 0 and rec.rec_syncs() == 0 and len(names()) == 6
''')


def test_counters_are_cleared_before_the_context_has_them(run_child):
    """The fill is waited for, so that a call on another stream finds it done; one that is lost leaves no counters behind."""
    run_child(IN_PLACE + '''
for f in (attend, matvec, in_place):
    st, ctx = create(PLAIN, 4, 2, 2, 0)
    live = rec.rec_live()
    rec.rec_reset(); rec.rec_fail_launch(0)
    assert f() == 4 and not names() and rec.rec_live() == live
    rec.rec_reset()
    assert f() == 0
    assert "k_seq_zero" in names()[0] and len(names()) == 2 and rec.rec_syncs() == 1, (names(), rec.rec_syncs())
    rec.rec_reset()
    assert f() == 0 and rec.rec_syncs() == 0 and len(names()) == 1
''')
