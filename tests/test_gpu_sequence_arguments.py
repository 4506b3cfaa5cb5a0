"""Arguments of the sequence operators that are no truth values: what they raise comes through, and nothing has been computed."""
import pytest
import torch

from test_gpu_sequence import _attend_inputs, rh  # noqa: F401  (the fixture)

pytestmark = pytest.mark.gpu


class Neither:
    def __bool__(self):
        raise KeyError("neither")


def test_what_is_no_truth_value(rh):  # noqa: F811
    q, cache, table, lengths = _attend_inputs(1, [30, 5], 2, 4, 64, 16, torch.bfloat16, torch.bfloat16)
    x = torch.randn((2, 64), device="cuda")
    w, sc = torch.ones((8, 32), dtype=torch.uint8, device="cuda"), torch.full((8, 2), 127, dtype=torch.uint8, device="cuda")
    out = torch.full((2, 8), 5.0, device="cuda")
    with pytest.raises(KeyError):
        rh.matvec_packed(x, w, sc, relu=Neither(), out=out)
    attended = torch.full((2, 8, 64), 5.0, dtype=torch.bfloat16, device="cuda")
    with pytest.raises(KeyError):
        rh.cache_attend(q, cache, table, lengths, want_lse=Neither(), out=attended)
    torch.cuda.synchronize()
    assert bool((out == 5).all()) and bool((attended == 5).all())
    assert torch.equal(rh.matvec_packed(x, w, sc, relu=1), rh.matvec_packed(x, w, sc, relu=True)) and len(rh.cache_attend(q, cache, table, lengths, want_lse=1)) == 2
