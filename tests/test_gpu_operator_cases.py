"""The calls of perf/operators.py as a program on another stream makes them."""
import pytest

pytestmark = pytest.mark.gpu


def test_cases_run_on_the_stream_that_is_current(lib):
    """A context is bound to the stream it was made on: a case that is run on another stream, or captured there, has its launches
    there, behind what that stream did before."""
    import torch
    import perf.operators as ops
    case = {"name": "t", "op": "evict", "dtype": "bf16", "shape": "wide_g2", "batch": 2, "cached": 900, "ragged": 0.2, "keep": 0.5, "lead": 1, "recent": 16}
    before = ops.own
    ops.own = True
    try:
        st = ops.prepare(case, 3)
        k, v = st["k"].clone(), st["v"].clone()

        def restore():
            st["k"].copy_(k)
            st["v"].copy_(v)
            torch.cuda.synchronize()
        want = [x.clone() for x in ops.run(st).values()]
        first = ops._context(st)[1]
        assert first.stream == torch.cuda.current_stream().cuda_stream
        side = torch.cuda.Stream()
        restore()
        with torch.cuda.stream(side):
            ctx = ops._context(st)[1]
            assert ctx.stream == side.cuda_stream and ctx is not first
            got = ops.run(st)
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(want, got.values()))
        graph = torch.cuda.CUDAGraph()
        restore()
        with torch.cuda.graph(graph, stream=side):
            ops.run(st)
        for _ in range(3):
            restore()
            st["meta"].zero_()
            torch.cuda.synchronize()
            graph.replay()
            torch.cuda.synchronize()
            assert all(torch.equal(a, b) for a, b in zip(want, got.values()))
        assert ops._context(st)[1] is first
    finally:
        ops.own = before
        for c in ops._CONTEXTS.values():
            c.close()
        ops._CONTEXTS.clear()
