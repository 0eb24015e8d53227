"""Gated units, passes one behind the other: kernels that begin beside their predecessors see what those leave, and nobody takes memory that is still in use."""
import pytest


@pytest.mark.gpu
@pytest.mark.parametrize("captured", [False, True])
@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("shape", [(16, 5, 512, 512), (9, 21, 333, 129), (5, 301, 501, 515), (4, 256, 512, 512), (1, 200, 1024, 512), (30, 90, 256, 136)], ids=str)
def test_passes_without_a_pause_are_those_with_one(shape, dtype, captured):
    """Steps that update inputs and weights in place and give their results' memory back at once, enqueued without a pause (or replayed from a graph): the same
    bits as with a synchronisation behind every call."""
    import torch
    import paper_1711_09846_b200 as pbt
    m, rows, width, hidden = shape
    dt = getattr(torch, dtype)

    def run(pause):
        gen = torch.Generator().manual_seed(7)
        w = torch.randn(m, 2 * hidden, width, generator=gen).mul_(width ** -0.5).to(dt).cuda()
        x, dh = (torch.randn(m, rows, n, generator=gen).to(dt).cuda() for n in (width, hidden))
        step = torch.zeros(m, dtype=torch.int64, device="cuda")
        unit, drop = pbt.GatedUnit(w, "silu"), pbt.Dropout(0.1, 5, step)
        sums = torch.zeros(m, 3, device="cuda")

        def steps():
            for keep in (True, False, True, True):
                h = unit.forward(x, dropout=drop, keep=keep)
                h, kept = h if keep else (h, None)
                pause()
                dx, dw = unit.backward(dh, x, kept, dropout=drop)
                pause()
                x.mul_(0.75).add_(dx, alpha=0.25)
                w.add_(dw, alpha=-1.0 / 1024)
                dh.mul_(0.5).add_(h, alpha=0.125)
                sums.add_(torch.stack([t.float().abs().amax((1, 2)) for t in (h, dx, dw)], 1))
                step.add_(1)
                del h, kept, dx, dw
                pause()
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            steps()
        side.synchronize()
        if captured and pause is none:
            graph = torch.cuda.CUDAGraph()
            with torch.cuda.graph(graph):
                steps()
            for _ in range(3):
                graph.replay()
        else:
            for _ in range(3):
                steps()
        unit.check()
        return [t.clone() for t in (x, w, dh, sums)]

    def none():
        pass
    expected = run(torch.cuda.synchronize)
    assert all(bool(t.isfinite().all()) for t in expected)
    for _ in range(3):
        for a, b in zip(run(none), expected):
            assert torch.equal(a, b)
