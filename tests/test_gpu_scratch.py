"""Replays of captured calls after larger calls on the same stream, which the scratch memory of both must survive."""
import pytest
import torch

from paper_2304_13134_amd import binding as lb
from gpu_util import announce

pytestmark = pytest.mark.gpu


def test_replays_after_larger_calls_on_the_same_stream():
    announce("replays after larger calls")
    g = torch.Generator(device="cuda").manual_seed(2)

    def operands(rows, N, K):
        return [torch.randn(n, generator=g, device="cuda").bfloat16() for n in ((rows, N), (rows, K), (N, K))]

    def step(dy, x, w):
        # shares of a long reduction, operands laid out, sums over workgroups: all three are in scratch memory
        s, gain = x[:, :64].contiguous(), torch.ones(64, device="cuda")
        inv = torch.ones(x.shape[0], device="cuda")
        return [*lb.last_product_grad_weight(dy, x), lb.last_product(x, w)[0], lb.last_product_grad_input(dy, w),
                *lb.last_residual_norm_grad(s, s, gain, inv)]

    small, large = operands(3000, 33, 65), operands(20000, 129, 257)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        lb.release_workspaces()
        want = [t.clone() for t in step(*small)]
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            got = step(*small)
        step(*large)                                                # outgrows the buffer that is kept for this stream
        side.synchronize()
        fillers = [torch.full((1 << k,), 7.0, device="cuda") for k in range(10, 23)]
        for k in range(3):
            for t in got:
                t.zero_()
            graph.replay()
            side.synchronize()
            assert all(torch.equal(a, b) for a, b in zip(got, want)), k
            assert all(bool((f == 7.0).all()) for f in fillers), k
        again = step(*small)
        side.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(again, want))
