"""Sizes at which rh_cache_plan's 32-bit positions would not do (no GPU; the recording stand-in of test_host_calls takes the place of the HIP runtime)."""
from test_host_calls import run_child  # noqa: F401  (the fixture)
from test_host_sequence import SETUP


def test_tables_and_stacks_past_32_bits_are_refused(run_child):  # noqa: F811
    """All streams may end at lengths that claim whole rows: the pages they give back, on top of the stack, have to be countable."""
    run_child(SETUP + '''
call = lambda n, page, n_pages, width: L.rh_cache_plan(ctx, P(1), P(2), n, page, n_pages, width, P(3), P(4), P(5), P(6), 8, P(7), P(8), P(9))
for n, page, n_pages, width in ((2048, 1, 1, 1 << 20), (2048, 16, 2048, (1 << 20) - 1), (1, 1, (1 << 31) - 8, 1000), (1024, 1, 1 << 30, 1 << 20)):
    rec.rec_reset()
    assert call(n, page, n_pages, width) == 2 and b"entries" in L.rh_last_error(ctx), (n, page, n_pages, width)          # RH_E_SHAPE
    assert not names()
for n, page, n_pages, width in ((2048, 1, 1000, (1 << 20) - 1), (2047, 16, (1 << 20) - 1, 1 << 20), (1, 1, (1 << 31) - 1008, 1000)):
    rec.rec_reset()
    assert call(n, page, n_pages, width) == 0, (n, page, n_pages, width, L.rh_last_error(ctx))
    assert len(names()) == 1
''')
