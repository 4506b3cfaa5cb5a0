"""Attention over scores that lie far apart, with bounds that wrong weights do not pass: queries and keys are small whole numbers, so that 32 bits hold
every score, and what is left of an error is the exponent's: u |s| for a score in powers of two (rounded twice: with the scale and as a product), the same
for the top, 2 u for the function, and the sums of n weights, all relative: e = 8 u max|s| + (16 + n / 16) u.  An output is a mean of values with such weights,
numerator and denominator: 2 e max|v|, and half an ulp of its type."""
import numpy as np
import pytest
import torch

from oracle import sequence as S
from test_gpu_sequence import E4M3, HALF, KINDS, U, _attend_inputs, _np, _values, rh  # noqa: F401  (the fixture)

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("q_dtype,c_dtype", KINDS)
@pytest.mark.parametrize("heads,group,dim", [(2, 4, 64), (1, 17, 128), (3, 1, 32), (1, 2, 224)])
def test_scores_hundreds_apart(rh, q_dtype, c_dtype, heads, group, dim):  # noqa: F811
    lens = [500, 77, 1, 2, 260, 0, 6000]
    q, cache, table, lengths = _attend_inputs(dim, lens, heads, group, dim, 16, q_dtype, c_dtype, poison=False)
    g = torch.Generator(device="cuda").manual_seed(dim)
    q = torch.randint(-3, 4, q.shape, generator=g, device="cuda").to(q_dtype)
    cache.k.copy_(torch.randint(-3, 4, cache.k.shape, generator=g, device="cuda").float().to(c_dtype))
    if c_dtype == E4M3:
        cache.k_scale.copy_(torch.tensor([0.5, 1.0, 2.0], device="cuda")[torch.randint(0, 3, cache.k_scale.shape, generator=g, device="cuda")])
    k, v, t = _values(cache.k, cache.k_scale), _values(cache.v, cache.v_scale), table.cpu().numpy()
    for scale, window in ((1.0, 0), (0.25, 0), (0.0, 0), (-0.5, 0), (1.0, 50)):
        out, lse = rh.cache_attend(q, cache, table, lengths, scale=scale, window=window, want_lse=True)
        w_out, w_lse = S.attend(_np(q), k, v, t, lens, 16, scale, window)
        out, lse = _np(out), _np(lse)
        for b, n in enumerate(lens):
            if n == 0:
                assert (out[b] == 0).all() and np.isneginf(lse[b]).all()
                continue
            pos = np.arange(max(0, n - window) if window else 0, n)
            p, line = t[b][pos // 16], pos % 16
            for h in range(q.shape[1]):
                most = np.abs(k[p, line, h // group] @ _np(q)[b, h] * scale).max()
                e = 8 * U * most + (16 + len(pos) / 16) * U
                bar = 2 * e * np.abs(v[p, line, h // group]).max() + HALF[q.dtype] * np.abs(w_out[b, h]) * (1 + 1e-6)
                assert (np.abs(out[b, h] - w_out[b, h]) <= bar).all(), (scale, window, b, h)
                assert abs(lse[b, h] - w_lse[b, h]) <= e + 2 * U * abs(w_lse[b, h]), (scale, window, b, h)
