"""What the sequence operators' entry points do on the host: null arguments, launches, allocations, a lost launch (no GPU; the
recording stand-in of test_host_calls takes the place of the HIP runtime)."""
from test_host_calls import run_child  # noqa: F401  (the fixture)

SETUP = '''
class KV(C.Structure):
    _fields_ = [("p", C.c_void_p * 4), ("ks", C.c_int64 * 3), ("vs", C.c_int64 * 3), ("type", C.c_int32), ("n_pages", C.c_int32),
                ("page", C.c_int32), ("heads", C.c_int32), ("dim", C.c_int32)]
V = lambda *v: (C.c_void_p * len(v))(*v)
kv = KV((C.c_void_p * 4)(1 << 24, 2 << 24, None, None), (16 * 128, 128, 64), (16 * 128, 128, 64), 1, 10, 16, 2, 64)
S2 = lambda a, b: (C.c_int64 * 2)(a, b)
st, ctx = create(PLAIN, 4, 2, 2, 0)
assert st == 0
L.rh_norm_residual.argtypes = [C.c_void_p, C.c_void_p, C.c_int64, C.c_void_p, C.c_int64, C.c_void_p, C.c_int32, C.c_int32, C.c_int32, C.c_float,
                               C.c_void_p, C.c_int64, C.c_void_p, C.c_void_p, C.c_void_p]
L.rh_cache_attend.argtypes = [C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p, C.c_int32, C.c_int32, C.c_void_p, C.c_int32, C.c_void_p, C.c_int32,
                              C.c_float, C.c_int32, C.c_void_p, C.c_void_p]
L.rh_matvec_packed.argtypes = [C.c_void_p, C.c_void_p, C.c_int32, C.c_int64, C.c_void_p, C.c_void_p, C.c_void_p, C.c_int32, C.c_int32, C.c_int32,
                               C.c_int32, C.c_void_p, C.c_int32, C.c_int64]
plan = lambda n=8, slots=8: L.rh_cache_plan(ctx, P(1), P(2), n, 16, 100, 6, P(3), P(4), P(5), P(6), slots, P(7), P(8), P(9))
write = lambda n=8: L.rh_cache_write(ctx, C.byref(kv), P(1), S2(512, 64), P(2), S2(512, 64), 1, P(3), n)
attend = lambda n=8, heads=8: L.rh_cache_attend(ctx, C.byref(kv), P(1), S2(512, 64), 1, heads, P(2), 6, P(3), n, 0.125, 0, P(4), P(5))
norm = lambda: L.rh_norm_residual(ctx, P(1), 512, P(2), 512, P(3), 1, 8, 512, 1e-6, P(4), 512, P(5), P(6), P(7))
matvec = lambda: L.rh_matvec_packed(ctx, P(1), 1, 512, None, P(2), P(3), 8, 100, 512, 0, P(4), 1, 100)
'''


def test_null_contexts_are_rejected():
    import paper_2407_16990_amd as pkg
    lib = pkg.load_library()
    assert lib.rh_cache_plan(None, None, None, 1, 1, 1, 1, None, None, None, None, 1, None, None, None) == 1
    assert lib.rh_cache_write(None, None, None, None, None, None, 0, None, 1) == 1
    assert lib.rh_cache_attend(None, None, None, None, 0, 1, None, 1, None, 1, 1.0, 0, None, None) == 1
    assert lib.rh_norm_residual(None, None, 1, None, 1, None, 0, 1, 1, 0.0, None, 1, None, None, None) == 1
    assert lib.rh_matvec_packed(None, None, 0, 1, None, None, None, 1, 1, 1, 0, None, 0, 1) == 1


def test_null_arguments_are_rejected_one_by_one(run_child):  # noqa: F811
    run_child(SETUP + '''
from itertools import product
calls = {
    "plan": (L.rh_cache_plan, [ctx, P(1), P(2), 8, 16, 100, 6, P(3), P(4), P(5), P(6), 8, P(7), P(8), P(9)], [1, 2, 7, 8, 9, 10, 12, 13, 14]),
    "write": (L.rh_cache_write, [ctx, C.byref(kv), P(1), S2(512, 64), P(2), S2(512, 64), 1, P(3), 8], [1, 2, 3, 4, 5, 7]),
    "attend": (L.rh_cache_attend, [ctx, C.byref(kv), P(1), S2(512, 64), 1, 8, P(2), 6, P(3), 8, 0.125, 0, P(4), P(5)], [1, 2, 3, 6, 8, 12]),
    "norm": (L.rh_norm_residual, [ctx, P(1), 512, P(2), 512, P(3), 1, 8, 512, 1e-6, P(4), 512, P(5), P(6), P(7)], [1, 5, 13, 14]),
    "matvec": (L.rh_matvec_packed, [ctx, P(1), 1, 512, None, P(2), P(3), 8, 100, 512, 0, P(4), 1, 100], [1, 5, 6, 11]),
}
for name, (f, args, required) in calls.items():
    rec.rec_reset()
    assert f(*args) == 0, (name, L.rh_last_error(ctx))
    assert len(names()) >= 1
    for i in required:
        rec.rec_reset()
        bad = list(args); bad[i] = None
        assert f(*bad) == 1 and len(L.rh_last_error(ctx)) > 10, (name, i)
        assert not names(), (name, i)
assert L.rh_norm_residual(ctx, P(1), 512, P(2), 512, P(3), 1, 8, 512, 1e-6, None, 512, None, None, None) == 1     # no output at all
''')


def test_scratch_memory_grows_once_and_is_freed(run_child):  # noqa: F811
    run_child(SETUP + '''
live = rec.rec_live()
for f in (plan, write, attend, norm, matvec): assert f() == 0
for again in range(2):
    rec.rec_reset()
    for f in (plan, write, attend, norm, matvec): assert f() == 0
    assert rec.rec_mallocs() == 0 and rec.rec_syncs() == 0, (rec.rec_mallocs(), rec.rec_syncs())
    assert len(names()) == 5, names()                        # a launch a call
rec.rec_reset(); assert attend(2000, 32) == 0 and attend(8) == 0 and plan(2048, 100000) == 0
first = rec.rec_mallocs()
assert attend(2000, 32) == 0 and rec.rec_mallocs() == first
L.rh_destroy(ctx)
st, ctx2 = create(PLAIN, 4, 2, 2, 0)
L.rh_destroy(ctx2)
assert rec.rec_live() == 0
''')


def test_a_lost_launch_is_reported_and_the_next_call_goes_on(run_child):  # noqa: F811
    run_child(SETUP + '''
for f in (plan, write, attend, norm, matvec):
    st, ctx = create(PLAIN, 4, 2, 2, 0)
    k = 0
    while True:                                              # the first call: also the launches that clear scratch memory
        rec.rec_reset(); rec.rec_fail_launch(k)
        st = f()
        if st == 0: break
        assert st == 4 and len(names()) == k, (st, names())
        k += 1
        assert k < 5
    assert k >= 1
    rec.rec_reset(); rec.rec_fail_launch(0)
    assert f() == 4 and L.rh_last_error(ctx)
    rec.rec_reset(); assert f() == 0 and len(names()) == 1
''')


def test_the_binding_looks_at_its_tensors():
    """What the library cannot see of a tensor is refused in the binding: where it lies, its type, its shape (no GPU: nothing passes here)."""
    import pytest
    import torch
    from paper_2407_16990_amd import KVCache, binding, load_library
    load_library()
    x, w, s = torch.zeros(2, 64), torch.zeros((8, 32), dtype=torch.uint8), torch.zeros((8, 2), dtype=torch.uint8)
    calls = [lambda: binding._seq.matvec_packed(0, x, w, s, None, False, None, None), lambda: binding._seq.norm_residual(0, x, x[0], None, 1e-6, "same", None),
             lambda: binding._seq.norm_residual(0, [1.0], x[0], None, 1e-6, "same", None), lambda: binding._seq.matvec_packed(0, x),
             lambda: binding._seq.cache_plan(0, *[torch.zeros(4, dtype=torch.int32)] * 5, 16, 4, None, None), lambda: binding._seq.cache_write(0, b"", x, x, x),
             lambda: binding._seq.cache_attend(0, b"no cache", x, x, x, None, 0, None, True), lambda: KVCache(torch.zeros(1, 1, 1, 32), torch.zeros(1, 1, 1, 32))]
    for call in calls:
        with pytest.raises(AssertionError):
            call()
