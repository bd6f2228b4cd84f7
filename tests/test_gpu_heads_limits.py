"""What the training operators take and refuse at their edges: graphs that would
repeat a step, one row of a wide buffer."""
import pytest
import torch

from paper_2011_12490_amd import derf, heads
from test_gpu_heads import BF16, FP32, gen, layer, rand

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


# ---- one row ----------------------------------------------------------------------------

def one_row(x, stride=1 << 22):
    """x [1, D] as a row of a buffer whose rows are `stride` apart."""
    view = torch.empty((1, stride), dtype=x.dtype, device=x.device)[:, :x.shape[1]]
    assert view.stride(0) == stride
    return view.copy_(x)


@pytest.mark.parametrize("dtype", [FP32, BF16])
def test_one_row_of_a_wide_buffer(dtype):
    """A single row has no next one, so its distance means nothing."""
    I, O = 40, 72
    x, w, b, offsets, g = layer([0, 1], 0, I, O, 0, 0, dtype, 1)
    y = heads.linear(x, w, b, offsets, True)
    far_y = heads.linear(one_row(x), w, b, offsets, True, one_row(torch.zeros_like(y)))
    assert torch.equal(far_y, y)
    dy = rand(g, 1, O).to(dtype)
    got = heads.linear_backward(one_row(dy), one_row(x), w, offsets, far_y, out_x=one_row(torch.zeros_like(x)))
    for a, c in zip(got, heads.linear_backward(dy, x, w, offsets, y)):
        assert torch.equal(a, c)
    r = heads.route(torch.zeros((1, 1), dtype=torch.int32, device="cuda"), 2)
    weights = torch.full((1, 1), 0.5, device="cuda")
    assert torch.equal(heads.dispatch(one_row(x), r, one_row(torch.zeros_like(x))), x)
    assert torch.equal(heads.combine(one_row(x), r, weights), heads.combine(x, r, weights))
