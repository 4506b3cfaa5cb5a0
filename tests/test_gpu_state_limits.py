"""rh_state_scan at sizes that need many workgroups: 8192 single rows of 8192 channels, 2048 streams of 65536 channels; against the formula in 64 bits on the GPU."""
import pytest
import torch

from test_gpu_state import HALF, TINY, U, _gen, _i32, _randn, rh  # noqa: F401  (rh: the fixture)

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("streams,channels,offsets", [(8192, 8192, False), (2048, 65536, True)])
def test_many_workgroups(rh, streams, channels, offsets):  # noqa: F811
    """A state of one element a channel, steps as they are given."""
    g, bf = _gen(1), torch.bfloat16
    x, b, c = _randn(g, streams, channels, dtype=bf), _randn(g, streams, 1, 1, dtype=bf), _randn(g, streams, 1, 1, dtype=bf)
    dt = (torch.rand((streams, channels), generator=g, device="cuda") * 0.5).to(bf)
    a = -torch.rand((channels, 1), generator=g, device="cuda") - 0.5
    state = _randn(g, 4, channels, 1)
    slots = _i32([k % 3 for k in range(streams)])                    # streams may share what they read
    into = _i32([3 if k == streams - 1 else -1 for k in range(streams)])
    before = state.clone()
    y = rh.state_scan(x, dt, a, b, c, state, slots, softplus=False, into=into, offsets=_i32(range(streams + 1)) if offsets else None)
    assert torch.equal(state[:3], before[:3])
    for k in range(0, streams, 512):
        d = dt[k:k + 512].double()
        old = before[slots[k:k + 512].long(), :, 0].double() * torch.exp(d * a[:, 0].double())
        h = old + d * x[k:k + 512].double() * b[k:k + 512, 0].double()
        want = h * c[k:k + 512, 0].double()
        # of the power: 2 for itself, 0.75 log2(e) for its argument and for the product's rounding; of the two products of delta x b 2, of the sum 1, the product with c 1
        tol = (8 * old.abs() + 3 * (h - old).abs()) * c[k:k + 512, 0].double().abs() * U + 2 * U * want.abs()
        err = (y[k:k + 512].double() - want).abs()
        assert bool((err <= tol + HALF[bf] * (want.abs() + tol) + TINY).all()), (k, float((err / want.abs().clamp_min(1e-3)).max()))
    assert bool(((state[3, :, 0].double() - h[-1]).abs() <= U * (8 * old[-1].abs() + 3 * (h - old)[-1].abs() + h[-1].abs()) + TINY).all())
