"""The workspace that device.Layer keeps: a captured call goes on writing to the one it was captured with, whatever is called after it."""
import pytest
import torch

from paper_2603_30033_amd import workloads as wl
from paper_2603_30033_amd.device import Layer, to_device
from test_gpu_forward_paged import Server, inputs

pytestmark = pytest.mark.gpu


def test_a_workspace_that_a_graph_uses_outlives_a_larger_one():
    w, inp, _ = inputs(wl.scaled(wl.WORKLOADS["tiny_f32"], dtype="bf16", seed=91), B=2, N=700)
    with Layer(w, inp, max_positions=700) as layer:
        X = [to_device(inp["X"][b], w.dtype) for b in range(2)]
        s = Server(w, layer, 2, 16, pages=100)
        s.step(X, [1, 1])
        batch = s.batch([1, 1])
        x = torch.stack([X[0][1], X[1][1]])
        y = torch.empty_like(x)
        layer.forward_paged(x, s.pools, batch, Y=y)
        want = y.clone()
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            layer.forward_paged(x, s.pools, batch, Y=y)
        first = layer._ws
        at, size = first.data_ptr(), first.numel()
        del first
        s2 = Server(w, layer, 2, 16, pages=100)
        s2.step(X, [699, 699])                                    # a larger workspace
        assert layer._ws.numel() > size
        # nothing else is given the memory that the graph writes to
        others = [torch.full((size,), 7, dtype=torch.uint8, device="cuda") for _ in range(8)]
        torch.cuda.synchronize()
        assert all(t.data_ptr() + t.numel() <= at or at + size <= t.data_ptr() for t in others + [layer._ws])
        for _ in range(3):
            y.zero_()
            graph.replay()
            torch.cuda.synchronize()
            assert torch.equal(y, want) and all((t == 7).all() for t in others)
