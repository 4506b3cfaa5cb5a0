"""Infinite values, scales and inputs of the sequence operators: the outputs that the formula gives - infinities of the right sign, NaN where
infinities of both signs or nothing times an infinity meet - and no other output touched."""
import numpy as np
import pytest
import torch

from oracle import sequence as S
from test_gpu_sequence import E4M3, KINDS, _attend_inputs, _np, _values, _weights, rh  # noqa: F401  (the fixture)

pytestmark = pytest.mark.gpu


def _attend_both(rh, q, cache, table, lengths, scale=0.125):
    out, lse = rh.cache_attend(q, cache, table, lengths, scale=scale, want_lse=True)
    with np.errstate(invalid="ignore"):
        want, w_lse = S.attend(_np(q), _values(cache.k, cache.k_scale), _values(cache.v, cache.v_scale), table.cpu().numpy(), lengths.cpu().numpy(), cache.page, scale)
    return _np(out), _np(lse), want, w_lse


def _same_where_not_finite(got, want):
    bad = ~np.isfinite(want)
    assert np.array_equal(got[bad], want[bad], equal_nan=True), (got[bad][:8], want[bad][:8])
    assert np.isfinite(got[~bad]).all()
    return bad


@pytest.mark.parametrize("q_dtype,c_dtype", KINDS[:2])
@pytest.mark.parametrize("heads,group,dim", [(1, 1, 64), (2, 5, 32), (1, 20, 128), (2, 3, 96)])
def test_infinite_values(rh, q_dtype, c_dtype, heads, group, dim):  # noqa: F811
    """Every token of short streams in turn, some of long ones: whatever the bits of its weight, one included."""
    lens = [1, 2, 7, 33, 60, 700, 5000]
    q, cache, table, lengths = _attend_inputs(dim + group, lens, heads, group, dim, 16, q_dtype, c_dtype)
    clean = rh.cache_attend(q, cache, table, lengths, scale=0.125)
    t = table.cpu().numpy()
    for step in range(8):
        old = cache.v.clone()
        for b, n in enumerate(lens):
            for d, sign in ((step, 1), (dim - 1 - step, -1)):
                pos = (step * 977 + d) % n
                cache.v[int(t[b, pos // 16]), pos % 16, :, d] = sign * float("inf")
        out, _, want, _ = _attend_both(rh, q, cache, table, lengths)
        bad = _same_where_not_finite(out, want)
        assert bad.sum() == len(lens) * heads * group * 2 and np.isinf(want[bad]).all()
        assert np.array_equal(out[~bad], _np(clean)[~bad])
        cache.v.copy_(old)


@pytest.mark.parametrize("q_dtype,c_dtype", KINDS[:2])
def test_infinities_of_both_signs(rh, q_dtype, c_dtype):  # noqa: F811
    q, cache, table, lengths = _attend_inputs(5, [40, 300], 1, 3, 64, 16, q_dtype, c_dtype)
    for b in range(2):
        p = int(table[b, 1])
        cache.v[p, 2, 0, 7], cache.v[p, 3, 0, 7] = float("inf"), float("-inf")
    out, _, want, _ = _attend_both(rh, q, cache, table, lengths)
    assert np.isnan(want[..., 7]).all()
    _same_where_not_finite(out, want)


@pytest.mark.parametrize("q_dtype,c_dtype", KINDS[:2])
def test_keys_that_make_a_score_minus_infinity(rh, q_dtype, c_dtype):  # noqa: F811
    """Such a token has no weight: the others' mean is left, and their log-sum-exp."""
    q, cache, table, lengths = _attend_inputs(6, [33, 200], 1, 2, 64, 16, q_dtype, c_dtype)
    q[..., 5] = q[..., 5].abs() + 0.25
    p, page = [int(table[b, 1]) for b in range(2)], cache.page
    for at in p:
        cache.k[at, 4, 0, 5] = float("-inf")
    out, lse, want, w_lse = _attend_both(rh, q, cache, table, lengths)
    assert np.isfinite(want).all() and np.isfinite(w_lse).all() and page == 16
    # scores of some units: errors of 1e-5 in fp32, outputs rounded to bf16 besides
    assert np.abs(out - want).max() <= (1e-5 if q_dtype == torch.float32 else 2.0 ** -8 * np.abs(want).max() + 1e-5) and np.abs(lse - w_lse).max() <= 1e-5


def test_infinite_scales_of_values(rh):  # noqa: F811
    q, cache, table, lengths = _attend_inputs(7, [1, 5, 90, 1000], 2, 4, 64, 16, torch.bfloat16, E4M3)
    code = cache.v.view(torch.uint8)
    for b, n in enumerate([1, 5, 90, 1000]):
        pos = n // 2
        p, line = int(table[b, pos // 16]), pos % 16
        cache.v_scale[p, :, line] = float("inf")
        code[p, line, :, 3], code[p, line, :, 4], code[p, line, :, 5] = 0x01, 0x81, 0x00        # the smallest numbers of either sign, and none
    out, _, want, _ = _attend_both(rh, q, cache, table, lengths)
    assert np.isposinf(want[..., 3]).all() and np.isneginf(want[..., 4]).all() and np.isnan(want[..., 5]).all()
    _same_where_not_finite(out, want)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("rows,n_in", [(1, 64), (16, 700), (33, 2048), (16, 16384)])
def test_infinite_inputs_of_products(rh, dtype, rows, n_in):  # noqa: F811
    g = torch.Generator(device="cuda").manual_seed(n_in)
    w, sc = _weights(g, 90, n_in)
    x = torch.randn((rows, n_in), generator=g, device="cuda").to(dtype)
    clean = _np(rh.matvec_packed(x, w, sc, out_dtype=torch.float32))
    x[0, n_in // 3] = float("inf")
    x[rows // 2, n_in - 1] = float("-inf")
    got = _np(rh.matvec_packed(x, w, sc, out_dtype=torch.float32))
    with np.errstate(invalid="ignore"):
        want = np.stack([(row * S.unpack_weights(w.cpu().numpy(), sc.cpu().numpy(), n_in)).sum(-1) for row in _np(x)])
    bad = ~np.isfinite(want)
    assert bad.any() and np.array_equal(got[bad], want[bad], equal_nan=True) and np.array_equal(got[~bad], clean[~bad])
