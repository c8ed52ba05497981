"""A captured route of logits that a graph recorded on another stream holds."""

import pytest
import torch

import ops_ref as ref
import paper_2609_25442_amd as wb

pytestmark = pytest.mark.gpu


def test_a_captured_route_of_a_living_graph_s_leaf_is_refused():
    z = ref.randn(20, 8, seed=1).cuda().requires_grad_()
    alive = wb.route(z, 2)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        with pytest.raises(wb.WbError, match="another stream"):
            wb.route(z, 2)
        gates = wb.route(z.detach(), 2).gates
    for _ in range(3):
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(gates, alive.gates)
    # without one it is captured, gradient and all
    d = ref.randn(20, 2, seed=2).cuda()
    del alive
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        wb.route(z, 2).gates.backward(d)
    torch.cuda.current_stream().wait_stream(side)
    want, z.grad = z.grad.clone(), None
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        wb.route(z, 2).gates.backward(d)
    for _ in range(3):
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(z.grad, want)
