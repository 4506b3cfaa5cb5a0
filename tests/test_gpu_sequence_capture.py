"""The first call that wants the sequence operators' memory, inside a stream capture and on another stream than the next."""
import pytest
import torch

from paper_2407_16990_amd import RhError
from test_gpu_sequence import _attend_inputs, _context, _weights

pytestmark = pytest.mark.gpu


def _inputs():
    g = torch.Generator(device="cuda").manual_seed(0)
    w, sc = _weights(g, 300, 16384)
    return torch.randn((16, 16384), generator=g, device="cuda"), w, sc, _attend_inputs(1, [3000, 5, 90], 2, 4, 64, 16, torch.bfloat16, torch.bfloat16)


def test_a_first_call_in_a_capture_is_refused():
    x, w, sc, (q, cache, table, lengths) = _inputs()
    rh, ref = _context(), _context()
    want = ref.matvec_packed(x, w, sc), ref.cache_attend(q, cache, table, lengths)
    torch.cuda.synchronize()
    side, weight = torch.cuda.Stream(), torch.ones(16384, device="cuda")

    def record(calls):
        graph = torch.cuda.CUDAGraph()
        rh.set_stream(side)
        try:
            with torch.cuda.graph(graph, stream=side):
                got = calls()
        finally:
            rh.set_stream(torch.cuda.current_stream())
        return graph, got

    def refused():
        out = rh.norm_residual(x, weight)                          # needs no memory of its own
        for call in (lambda: rh.matvec_packed(x, w, sc), lambda: rh.cache_attend(q, cache, table, lengths)):
            with pytest.raises(RhError, match="capture") as e:
                call()
            assert e.value.status == 6
        return out

    record(refused)
    # the context goes on: eager calls, and from then on captured ones
    for _ in range(2):
        assert torch.equal(rh.matvec_packed(x, w, sc), want[0]) and torch.equal(rh.cache_attend(q, cache, table, lengths), want[1])
    graph, got = record(lambda: (rh.matvec_packed(x, w, sc), rh.cache_attend(q, cache, table, lengths)))
    for _ in range(3):
        for t in got:
            t.fill_(7)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, want))
        assert torch.equal(rh.matvec_packed(x, w, sc), want[0])
        torch.cuda.synchronize()


def test_the_next_call_may_be_on_another_stream():
    x, w, sc, (q, cache, table, lengths) = _inputs()
    ref = _context()
    want = ref.matvec_packed(x, w, sc), ref.cache_attend(q, cache, table, lengths)
    torch.cuda.synchronize()
    for _ in range(3):
        first, second = torch.cuda.Stream(), torch.cuda.Stream()
        rh = _context(stream=first)
        rh.matvec_packed(x[:1, :64].contiguous(), w[:, :32].contiguous(), sc[:, :2].contiguous())      # the first call; uses no counter
        rh.set_stream(second)
        got = rh.matvec_packed(x, w, sc), rh.cache_attend(q, cache, table, lengths)
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, want))
