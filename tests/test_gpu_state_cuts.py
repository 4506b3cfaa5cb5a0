"""rh_state_scan at the borders of the rule by which streams are cut into chunks (288 rows, one and a half chunks, whole stages), against its plain implementation in 64 bits."""
import numpy as np
import pytest
import torch

from test_gpu_state import TYPES, Streams, _check_scan, _gen, rh  # noqa: F401  (rh: the fixture)

pytestmark = pytest.mark.gpu

CUT = 288                                                            # rows from which on a stream may be cut


def _longest_cut(lens):
    return max([n for n in lens if n >= CUT], default=0)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("n", [13, 16, 128])
@pytest.mark.parametrize("lens", [[286], [287], [288], [289], [290], [319], [320], [321], [383], [384], [385], [287, 288, 289], [288, 0, 288, 1, 287]])
def test_lengths_around_the_first_cut(rh, dtype, n, lens):  # noqa: F811
    """Few rows, so that chunks have 64: from 288 on streams are cut, into whole stages and what is left."""
    for in_place in (False, True):
        _check_scan(rh, _gen(n), Streams(np.random.default_rng(n), lens, in_place=in_place), 12, n, 1, dtype, cut_rows=_longest_cut(lens))


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("n", [5, 16])
def test_lengths_around_one_and_a_half_chunks(rh, dtype, n):  # noqa: F811
    """64 groups of a channel on a card of 256 compute units: of 3840 rows chunks have 320, and streams of 480 rows are the shortest that are cut; 640, 641 and 960, 961: two and three chunks, and one more."""
    for lens in ([479, 480, 481, 0, 2000, 1, 399], [640, 641, 960, 961, 638], [3840]):
        assert sum(lens) == 3840
        _check_scan(rh, _gen(n), Streams(np.random.default_rng(n), lens), 64, n, 64, dtype, cut_rows=max(lens))


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("n_streams,long", [(64, 288), (65, 288), (2048, 600)])
def test_one_of_many_streams_is_cut(rh, dtype, n_streams, long):  # noqa: F811
    rng = np.random.default_rng(n_streams)
    lens = rng.integers(0, 8, n_streams)
    for at in (0, n_streams // 2, n_streams - 3):                   # the last ones of Streams are not kept
        some = lens.copy()
        some[at] = long
        _check_scan(rh, _gen(n_streams), Streams(rng, some.tolist()), 10, 16, 1, dtype, cut_rows=long)


@pytest.mark.parametrize("dtype", TYPES)
def test_steps_of_any_size_in_a_stream_that_is_cut(rh, dtype):  # noqa: F811
    """dt from far below zero to above 20; states that fade at once, and not at all, over whole chunks."""
    s = Streams(np.random.default_rng(3), [60, 700], 2)
    for spread, steps in ((30.0, (0.5, 2.0)), (0.1, (1e-6, 1e-4)), (3.0, (1e-3, 10.0))):
        _check_scan(rh, _gen(5), s, 30, 16, 1, dtype, spread=spread, steps=steps, cut_rows=700)
    _check_scan(rh, _gen(2), s, 20, 16, 1, dtype, soft=False, spread=0.05, dt_bias=False, cut_rows=700)


@pytest.mark.parametrize("dtype", TYPES)
def test_a_stream_that_is_not_cut_is_as_exact_beside_one_that_is(rh, dtype):  # noqa: F811
    """287 rows: within the bounds of rows one after the other, without what a chunk's sum of steps adds."""
    _check_scan(rh, _gen(6), Streams(np.random.default_rng(6), [287, 250, 100]), 30, 16, 1, dtype, spread=30.0, steps=(0.5, 2.0))
