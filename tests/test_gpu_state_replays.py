"""A captured scan and convolution whose offsets change between replays: streams that are cut in one and not in the next, empty ones, offsets that descend."""
import numpy as np
import pytest
import torch

from test_gpu_state import _gen, _i32, _layer_inputs, _randn, rh  # noqa: F401  (rh: the fixture)

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("streams", [4, 70])
def test_offsets_that_change_between_replays(rh, streams):  # noqa: F811
    """The launches go by rows and streams alone; what is cut is found on the GPU.  Every replay is what the call gives, also behind one that wrote nothing."""
    channels, n, rows, g = 40, 16, 1200, _gen(0)
    t = _layer_inputs(g, rows, channels, n, torch.bfloat16)
    w, a, slots = _randn(g, 4, channels) / 2, -torch.exp(_randn(g, channels, n)), _i32(np.arange(streams))

    def lay(*ends):
        return np.concatenate((ends, np.full(streams + 1 - len(ends), ends[-1])))
    lists = [lay(0, rows), lay(0, 100, 500, 500, rows), lay(0, 287, 575, 864, rows), lay(0, 900, 600, rows), lay(0, 0, 0, 0, rows), lay(0, 640, 0), lay(0, 1, 2, 3, 4), lay(0, 100, 500, 500, rows),
             np.linspace(0, rows, streams + 1).astype(int), lay(5, 5), lay(0, rows)]
    state = lambda: (torch.zeros((streams, 3, channels), dtype=torch.bfloat16, device="cuda"), torch.zeros((streams, channels, n), device="cuda"))  # noqa: E731
    out = lambda: [torch.zeros((rows, channels), dtype=torch.bfloat16, device="cuda") for _ in range(2)]  # noqa: E731
    offsets, cap, eager, got, want = _i32(lists[0]), state(), state(), out(), out()

    def call(s, o, where):
        rh.state_conv(t["x"], w, s[0], slots, offsets=where, out=o[0])
        rh.state_scan(o[0], t["dt"], a, t["b"], t["c"], s[1], slots, gate=t["gate"], offsets=where, out=o[1])
    call(state(), out(), offsets)                                    # the scratch memory is there
    torch.cuda.synchronize()
    side, main, graph = torch.cuda.Stream(), torch.cuda.current_stream(), torch.cuda.CUDAGraph()
    rh.set_stream(side)
    try:
        with torch.cuda.graph(graph, stream=side):
            call(cap, got, offsets)
    finally:
        rh.set_stream(main)
    for k, where in enumerate(lists):
        before = [v.clone() for v in (*cap, *got)]
        offsets.copy_(_i32(where))
        graph.replay()
        call(eager, want, _i32(where))
        torch.cuda.synchronize()
        assert all(torch.equal(p, q) for p, q in zip((*cap, *got), (*eager, *want))), k
        if (np.diff(where) < 0).any():
            assert all(torch.equal(p, q) for p, q in zip((*cap, *got), before)), k
        assert all(bool(torch.isfinite(v.float()).all()) for v in (*cap, *got)), k
