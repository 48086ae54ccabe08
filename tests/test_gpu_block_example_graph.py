"""The expert-block example's gradients, captured into a graph."""
import pytest
import torch

from tests.helpers import require_gpu

pytestmark = pytest.mark.gpu


def test_gradients_in_a_graph():
    """Replays give the eager call's bits at the step counter's present value
    and for the inputs' present contents, with eager work between them."""
    require_gpu()
    from examples import expert_block
    m = expert_block.ExpertBlocks(50, 7, blocks=2, width=80, hidden=96, experts=5, k=2, rate=0.25, seed=3)
    g = torch.Generator().manual_seed(2)
    x = torch.randn(64, 50, generator=g).to(m.dtype).cuda()
    labels = torch.randint(0, 7, (64,), generator=g).cuda()
    offsets = m._all_rows(64)
    assert m._all_rows(64) is offsets and offsets.tolist() == [0, 64] and m._all_rows(65).tolist() == [0, 65]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        m.gradients(x, labels)
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        loss, grads = m.gradients(x, labels)
    seen = []
    for step in (0, 4, 8, 4):
        m.steps_done.fill_(step)
        x.mul_(1.125)
        graph.replay()
        torch.cuda.synchronize()
        want_loss, want = m.gradients(x, labels)
        torch.cuda.synchronize()
        assert torch.equal(loss, want_loss), step
        for n in want:
            assert torch.equal(grads[n], want[n]), (step, n)
        seen.append(grads["0.w1"].clone())
    assert not torch.equal(seen[0], seen[1]) and not torch.equal(seen[1], seen[2])
