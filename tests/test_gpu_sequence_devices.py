"""Sequence operators take tensors of their context's device only.  One device is here: the context is said to be another's, so that every tensor
is the wrong one; nothing may be launched then."""
import pytest
import torch

from test_gpu_sequence import _attend_inputs, _context, _i32

pytestmark = pytest.mark.gpu


def test_tensors_of_another_device_are_refused():
    rh = _context()
    q, cache, table, lengths = _attend_inputs(1, [30, 5], 2, 4, 64, 16, torch.bfloat16, torch.bfloat16)
    x, weight = torch.randn((2, 64), device="cuda"), torch.ones(64, device="cuda")
    w, sc = torch.ones((8, 32), dtype=torch.uint8, device="cuda"), torch.full((8, 2), 127, dtype=torch.uint8, device="cuda")
    slots, free = _i32([0, 1]), torch.arange(10, dtype=torch.int32, device="cuda")
    out = torch.full((2, 8), 5.0, device="cuda")
    calls = [lambda: rh.cache_plan(_i32([1, 1]), lengths.clone(), table.clone(), free, _i32([4]), 16, 4), lambda: rh.cache_write(cache, q[:, :2], q[:, 2:4], slots),
             lambda: rh.cache_attend(q, cache, table, lengths), lambda: rh.norm_residual(x, weight, outputs="both"), lambda: rh.matvec_packed(x, w, sc, out=out)]
    handle, device = rh._ctx
    assert device == 0
    before = cache.k.clone()
    rh._ctx = (handle, 1)
    for call in calls:
        with pytest.raises(AssertionError, match="another device"):
            call()
    torch.cuda.synchronize()
    assert torch.equal(cache.k.view(torch.uint8), before.view(torch.uint8)) and bool((out == 5).all())
    rh._ctx = (handle, 0)
    for call in calls:
        call()
    # codes 1 at even and 0 at odd inputs, scale one: halves of the even inputs' sum; 32 terms of a few units in fp32
    assert torch.allclose(out, (x[:, 0::2] * 0.5).sum(1, keepdim=True).expand(2, 8), rtol=0, atol=1e-4)
