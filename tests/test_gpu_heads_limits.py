"""What the training operators take and refuse at their edges: graphs that would
repeat a step."""
import pytest
import torch

from paper_2011_12490_amd import derf, heads
from test_gpu_heads import gen, rand

pytestmark = pytest.mark.gpu


# ---- AdamW in graphs ------------------------------------------------------------------

@pytest.mark.parametrize("bits", [32, 8])
def test_adamw_step_is_not_recorded(bits):
    """A recorded step would repeat its step number and rate at every replay: it raises,
    the recording goes on without it, and steps beside the replays are the eager ones."""
    g = gen(1)
    p, grad = rand(g, 3000), rand(g, 3000)
    q = p.clone()
    opt, ref = heads.AdamW([p], [grad], state_bits=bits), heads.AdamW([q], [grad], state_bits=bits)
    other = torch.zeros(100, device="cuda")
    s = torch.cuda.Stream()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=s):
        other.add_(1)
        with pytest.raises(derf.DerfError, match="captur"):
            opt.step()
        other.add_(1)
    assert opt.steps == 0
    for i in range(3):
        graph.replay()
        torch.cuda.synchronize()
        assert bool((other == 2 * (i + 1)).all()) and torch.equal(p, q)
        opt.step()
        ref.step()
        torch.cuda.synchronize()
        assert torch.equal(p, q) and opt.steps == i + 1
