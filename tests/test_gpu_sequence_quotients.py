"""8-bit outputs of the sequence operators bit for bit: scale = max(largest magnitude, 2^-100) * (1/448) and element = value / scale, 1/448, product and quotient
each rounded to fp32, the element then to e4m3 (nearest, ties to even).  No tolerance: the same steps in numpy and torch on the CPU give the same codes."""
import numpy as np
import pytest
import torch

from test_gpu_sequence import E4M3, _empty_cache, rh  # noqa: F401  (the fixture)

pytestmark = pytest.mark.gpu


def _codes(v):
    """v f32 [rows, n] -> (codes uint8 [rows, n], scales f32 [rows])."""
    v = v.astype(np.float32)
    scale = np.maximum(np.abs(v).max(-1), np.float32(2.0 ** -100)) * (np.float32(1) / np.float32(448))
    assert scale.dtype == np.float32
    return torch.from_numpy(v / scale[:, None]).to(E4M3).view(torch.uint8).numpy(), scale


def _values(rng, rows, n):
    """Few significant bits, so that many quotients lie at a tie between two codes or next to one; rows of every size, tiny ones too."""
    v = rng.integers(-40, 41, (rows, n)) * np.exp2(rng.integers(-6, 1, (rows, n)))
    v[:, 0] = rng.integers(30, 60, rows)
    size = np.exp2(rng.integers(-120, 100, rows).astype(np.float64))
    size[: rows // 2] = 1
    return (v * size[:, None]).astype(np.float32)


@pytest.mark.parametrize("src", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("n,heads,dim", [(1, 1, 32), (300, 3, 96), (500, 4, 128), (200, 1, 256)])
def test_write_gives_the_codes_of_the_quotients(rh, src, n, heads, dim):  # noqa: F811
    rng = np.random.default_rng(dim)
    page, pages = 16, n // 16 + 2
    k, v = (torch.from_numpy(_values(rng, n * heads, dim)).to(src).view(n, heads, dim) for _ in range(2))
    cache = _empty_cache(pages, page, heads, dim, E4M3, "head")
    slots = torch.from_numpy(rng.permutation(pages * page)[:n].astype(np.int32))
    rh.cache_write(cache, k.cuda(), v.cuda(), slots.cuda())
    p, line = slots.numpy() // page, slots.numpy() % page
    for x, c, sc in ((k, cache.k, cache.k_scale), (v, cache.v, cache.v_scale)):
        codes, scales = _codes(x.float().numpy().reshape(n * heads, dim))
        assert np.array_equal(sc.cpu().numpy()[p, :, line].reshape(-1), scales)
        got = c.view(torch.uint8).cpu().numpy()[p, line].reshape(n * heads, dim)
        assert np.array_equal(got, codes), int((got != codes).sum())


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("rows,cols", [(5, 16), (9, 256), (4, 1024), (3, 4096)])
def test_norm_gives_the_codes_of_the_quotients(rh, dtype, rows, cols):  # noqa: F811
    """A row of ones of either sign (eps 0) is normed to itself exactly, and the weight brings few-bit values of many sizes."""
    rng = np.random.default_rng(cols)
    for most in range(41, 64, 2):
        sign = rng.choice([-1.0, 1.0], (rows, cols)).astype(np.float32)
        weight = (rng.integers(1, 41, cols) * np.exp2(rng.integers(-6, 1, cols))).astype(np.float32)
        weight[0] = most
        weight *= np.float32(2.0 ** float(rng.choice([0, 0, -115, 90])))
        x = torch.from_numpy(sign).to(dtype).cuda()
        _, y, y8, sc = rh.norm_residual(x, torch.from_numpy(weight).cuda(), eps=0.0, outputs="both")
        assert dtype == torch.bfloat16 or np.array_equal(y.cpu().numpy(), sign * weight)
        codes, scales = _codes(sign * weight)
        assert np.array_equal(sc.cpu().numpy(), scales)
        got = y8.view(torch.uint8).cpu().numpy()
        assert np.array_equal(got, codes), (most, int((got != codes).sum()))


def test_write_and_norm_are_torchs_formula_on_the_gpu(rh):  # noqa: F811
    """The formula in torch's operations on the same device gives the same bits: t / 448.0 is a product with 1/448 there."""
    g = torch.Generator(device="cuda").manual_seed(0)
    x = torch.randn((500, 4, 96), generator=g, device="cuda").to(torch.bfloat16)
    cache = _empty_cache(40, 16, 4, 96, E4M3, "token")
    rh.cache_write(cache, x, x, torch.arange(500, dtype=torch.int32, device="cuda"))
    scale = x.float().abs().amax(-1).clamp_min(2.0 ** -100) / 448.0
    codes = (x.float() / scale[..., None]).to(E4M3).view(torch.uint8)
    got = cache.k.view(torch.uint8).reshape(-1, 4, 96)[:500], cache.k_scale.transpose(1, 2).reshape(-1, 4)[:500]
    assert torch.equal(got[0], codes) and torch.equal(got[1], scale)
    y = torch.randn((300, 700), generator=g, device="cuda")
    _, n, n8, sc = rh.norm_residual(y, torch.ones(700, device="cuda"), outputs="both")
    scale = n.abs().amax(-1).clamp_min(2.0 ** -100) / 448.0
    assert torch.equal(sc, scale) and torch.equal(n8.view(torch.uint8), (n / scale[:, None]).to(E4M3).view(torch.uint8))
