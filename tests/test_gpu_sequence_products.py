"""Products with 4-bit weights on inputs whose result is known bit for bit: sums that 32 bits hold whatever their order, single products at every
scale; and rows of 8 bits with bf16 outputs at every number of rows and length."""
import numpy as np
import pytest
import torch

from oracle import sequence as S
from test_gpu_sequence import E4M3, TYPES, _check_matvec, _rows, _weights, rh  # noqa: F401  (the fixture)

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,n_out,n_in", [(1, 70, 64), (1, 40, 512), (16, 100, 1000), (17, 300, 512), (32, 64, 4096), (33, 50, 1500), (64, 200, 2048), (70, 33, 8192), (16, 4100, 700)])
def test_what_is_left_when_large_terms_cancel(rh, dtype, rows, n_out, n_in):  # noqa: F811
    """Every row has two pairs of +-448 under the same code, far apart, and small whole multiples of 2^-9 elsewhere.  All terms are multiples of 2^-10 and every
    partial sum stays below 2 * 448 * 6 + 8192 * 6 * 2^-6 < 2^13: 32 bits hold each of them, in any order, so that the result is exact."""
    rng = np.random.default_rng(rows * 9 + n_in)
    g = torch.Generator(device="cuda").manual_seed(rows + n_in)
    w, _ = _weights(g, n_out, n_in)
    sc = torch.full((n_out, (n_in + 31) // 32), 127, dtype=torch.uint8, device="cuda")
    x = rng.integers(-8, 9, (rows, n_in)) * 2.0 ** -9
    pairs = rng.permutation(n_in)[:4]
    for a, b in (pairs[:2], pairs[2:]):
        x[:, a], x[:, b] = 448, -448
        code = w[:, a // 2] >> (4 * (a % 2)) & 15
        keep = w[:, b // 2] & (0xF0 if b % 2 == 0 else 0x0F)
        w[:, b // 2] = keep | code << (4 * (b % 2))
    t = torch.from_numpy(x).float().to(dtype).cuda()
    assert np.array_equal(t.double().cpu().numpy() if dtype != E4M3 else S.e4m3_values()[t.view(torch.uint8).cpu().numpy()], x)
    want = torch.from_numpy(S.matvec(x, w.cpu().numpy(), sc.cpu().numpy()))
    assert torch.equal(want.float().double(), want)
    for out in (torch.float32, torch.bfloat16):
        assert torch.equal(rh.matvec_packed(t, w, sc, out_dtype=out).cpu(), want.to(out)), out


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,n_in", [(1, 512), (16, 1000), (17, 512), (32, 700), (33, 2048), (64, 1024)])
def test_every_code_at_every_scale_along_a_long_row(rh, dtype, rows, n_in):  # noqa: F811
    """Rows with a single one among zeros: the outputs are the weights under it, of every code at every scale byte; 255 is not a number."""
    rng = np.random.default_rng(n_in + rows)
    at = rng.integers(0, n_in, rows)
    n = np.arange(4096)
    w = torch.from_numpy(np.repeat((n % 16 * 17).astype(np.uint8)[:, None], 16 * ((n_in + 31) // 32), axis=1)).cuda()
    sc = torch.from_numpy(np.repeat((n // 16).astype(np.uint8)[:, None], (n_in + 31) // 32, axis=1)).cuda()
    x = torch.zeros((rows, n_in), device="cuda")
    x[torch.arange(rows), torch.from_numpy(at)] = 1
    real = S.unpack_weights(w.cpu().numpy()[:, :16], sc.cpu().numpy()[:, :1], 1)[:, 0]
    for out in (torch.float32, torch.bfloat16):
        y = rh.matvec_packed(x.to(dtype), w, sc, out_dtype=out).float().cpu().numpy()
        with np.errstate(over="ignore"):
            want = torch.from_numpy(real.astype(np.float32)).to(out).float().numpy()
        assert np.isnan(y[:, 4080:]).all()
        # numbers below the normal ones may come out as zeros
        ok = (y == want) | ((np.abs(want) < 2.0 ** -126) & (np.abs(y) < 2.0 ** -126))
        assert ok[:, :4080].all(), (out, np.argwhere(~ok[:, :4080])[:5])


@pytest.mark.parametrize("rows,n_out,n_in", [(1, 60, 512), (16, 200, 1024), (17, 100, 1000), (32, 64, 4096), (33, 130, 600), (64, 300, 2048), (64, 40, 8192)])
def test_rows_of_8_bits_with_bf16_outputs(rh, rows, n_out, n_in):  # noqa: F811
    g = torch.Generator(device="cuda").manual_seed(n_in + rows)
    x = _rows(g, rows, n_in, E4M3)
    xs = torch.rand(rows, generator=g, device="cuda") * 0.1
    for wide in (False, True):
        w, sc = _weights(g, n_out, n_in, wide=wide)
        y = _check_matvec(rh, x, w, sc, None if wide else xs, False, torch.bfloat16)
    # a NaN of a row stays in that row's outputs
    w, sc = _weights(g, n_out, n_in)
    y = rh.matvec_packed(x, w, sc)
    bad = x.clone()
    bad.view(torch.uint8)[rows // 2, n_in // 3] = 0x7F
    z = rh.matvec_packed(bad, w, sc)
    assert bool(z[rows // 2].isnan().all())
    z[rows // 2] = y[rows // 2]
    assert torch.equal(z, y)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,n_out,n_in", [(1, 48, 32), (2, 100, 130), (17, 90, 512), (33, 64, 700), (64, 200, 2048), (16, 60, 16384)])
def test_outputs_of_scales_far_apart_side_by_side(rh, dtype, rows, n_out, n_in):  # noqa: F811
    """Neighbouring outputs whose blocks have the smallest scales, the largest and others: each comes out as it would alone.  Rows of two sizes, for the
    large scales and for the small ones (8-bit rows cannot be that far apart)."""
    rng = np.random.default_rng(n_in + rows)
    g = torch.Generator(device="cuda").manual_seed(n_in)
    w, _ = _weights(g, n_out, n_in)
    blocks = (n_in + 31) // 32
    scales = np.array([2, 3, 8, 9, 60, 127, 200, 251, 252, 253, 254], dtype=np.uint8)
    small, large = 2.0 ** -20, 2.0 ** 60
    for mixed in (False, True):
        # one scale an output, or two a row: the small beside the large of the same output
        sc = np.repeat(rng.choice(scales, (n_out, 1)), blocks, axis=1)
        if mixed:
            sc = np.where(rng.random((n_out, blocks)) < 0.5, sc, rng.choice(scales, (n_out, blocks)))
        x = rng.standard_normal((rows, n_in)) * (small if dtype != E4M3 else 2.0 ** -4)
        if dtype != E4M3:
            x[1::2] *= large / small
        t = torch.from_numpy(x).float().to(dtype).cuda()
        xn = t.double().cpu().numpy() if dtype != E4M3 else S.e4m3_values()[t.view(torch.uint8).cpu().numpy()]
        d_sc = torch.from_numpy(sc.astype(np.uint8)).cuda()
        real = S.unpack_weights(w.cpu().numpy(), sc.astype(np.uint8), n_in)
        want, most = xn @ real.T, np.abs(xn) @ np.abs(real).T
        y = rh.matvec_packed(t, w, d_sc, out_dtype=torch.float32).double().cpu().numpy()
        held = most < 2.0 ** 127                                   # others' partial sums may pass fp32
        tol = (n_in + 8) * 2.0 ** -24 * most + 2.0 ** -24 * np.abs(want) + n_in * 2.0 ** -149
        assert mixed or held.any()
        assert (np.abs(y - want)[held] <= tol[held]).all(), np.argwhere(held & ~(np.abs(y - want) <= tol))[:5]


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("rows,n_in", [(1, 32), (18, 512), (33, 600)])
def test_infinite_inputs_beside_the_largest_scales(rh, dtype, rows, n_in):  # noqa: F811
    g = torch.Generator(device="cuda").manual_seed(rows)
    w, _ = _weights(g, 64, n_in)
    blocks = (n_in + 31) // 32
    sc = torch.full((64, blocks), 120, dtype=torch.uint8, device="cuda")
    sc[5], sc[20, blocks // 2], sc[41] = 253, 254, 3
    x = (torch.randn((rows, n_in), generator=g, device="cuda") * 2.0 ** -20).to(dtype)
    x[rows // 2, n_in // 2] = float("inf")
    y = rh.matvec_packed(x, w, sc, out_dtype=torch.float32).double().cpu().numpy()
    with np.errstate(invalid="ignore"):
        want = np.stack([(row * S.unpack_weights(w.cpu().numpy(), sc.cpu().numpy(), n_in)).sum(-1) for row in x.double().cpu().numpy()])
    bad = ~np.isfinite(want)
    assert bad.sum() == 64 and np.array_equal(y[bad], want[bad], equal_nan=True) and np.isfinite(y[~bad]).all()
