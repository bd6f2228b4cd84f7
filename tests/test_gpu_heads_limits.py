"""What the training operators take and refuse at their edges: graphs that would
repeat a step, one row of a wide buffer, sizes beyond the limits, tensors that
autograd follows."""
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


# ---- sizes beyond the limits ----------------------------------------------------------

def test_what_does_not_fit_raises_value_error():
    z = lambda *shape, dtype=FP32: torch.zeros(shape, dtype=dtype, device="cuda")  # noqa: E731
    ints = lambda *shape: z(*shape, dtype=torch.int32)  # noqa: E731
    wide, many, two = 65537, 17, ints(2)
    far = torch.empty((1 << 21) + 64, device="cuda").as_strided((2, 8), (1 << 21, 1))  # rows 2^21 apart
    p = z(10)
    opt = heads.AdamW([p], [z(10)])
    pairs = heads.Routing(ints(3), ints(4), ints(2, 2), 2)
    slots = heads.Routing(ints(3), ints(2 * many), ints(2, many), 2)
    bad = [
        lambda: heads.dispatch(z(2, wide), pairs), lambda: heads.combine(z(4, wide), pairs),
        lambda: heads.combine_backward(z(2, wide), None, pairs),
        lambda: heads.dispatch(z(2, 4), slots), lambda: heads.combine(z(2 * many, 4), slots),
        lambda: heads.combine_backward(z(2, 4), None, slots), lambda: heads.route(ints(2, many), 2),
        lambda: heads.linear(z(2, 8), z(257, 4, 8), None, ints(258)), lambda: heads.linear(z(2, wide), z(1, 1, wide), None, two),
        lambda: heads.linear(z(2, 1), z(1, wide, 1), None, two), lambda: heads.linear(far, z(1, 4, 8), None, two),
        lambda: heads.linear(z(2, 4), z(1, 8, 4), None, two, out=far),
        lambda: heads.linear_backward(z(2, 4), z(2, 8), z(257, 4, 8), ints(258)),
        lambda: heads.linear_backward(far, z(2, 4), z(1, 8, 4), two), lambda: heads.linear_backward(z(2, 4), far, z(1, 4, 8), two),
        lambda: opt.step(step=0),
    ]
    for i, call in enumerate(bad):
        with pytest.raises(ValueError):
            call()
            pytest.fail("case %d was taken" % i)
    for lr, betas, eps, decay in ((-1.0, (0.9, 0.99), 1e-8, 0.0), (1e-3, (1.0, 0.99), 1e-8, 0.0), (1e-3, (0.9, 0.99), float("nan"), 0.0),
                                  (1e-3, (0.9, 0.99), 1e-8, -0.1)):
        opt.lr, opt.betas, opt.eps, opt.weight_decay = lr, betas, eps, decay
        with pytest.raises(ValueError):
            opt.step()
    assert opt.steps == 0 and not bool(p.any())


# ---- autograd ---------------------------------------------------------------------------

def test_tensors_that_autograd_follows():
    """No graph is recorded, so a tensor that requires a gradient is refused where one
    would be expected; without autograd, and in the optimizer, it is as any other."""
    g = gen(2)
    x, w, b, offsets, _ = layer([3, 2], 0, 8, 6, 0, 0, FP32, 3)
    dy, dout, weights = rand(g, 5, 6), rand(g, 5, 8), rand(g, 5, 1)
    r = heads.route(torch.zeros((5, 1), dtype=torch.int32, device="cuda"), 2)
    leaf = lambda t: t.clone().requires_grad_()  # noqa: E731
    calls = [lambda f: heads.linear(f(x), w, b, offsets), lambda f: heads.linear(x, f(w), b, offsets),
             lambda f: heads.linear(x, w, f(b), offsets), lambda f: heads.linear_backward(f(dy), x, w, offsets)[0],
             lambda f: heads.linear_backward(dy, x, f(w), offsets)[0], lambda f: heads.dispatch(f(x), r),
             lambda f: heads.combine(f(x), r, weights), lambda f: heads.combine(x, r, f(weights)),
             lambda f: heads.combine_backward(f(dout), x, r, weights)[0],
             lambda f: heads.combine_backward(dout, f(x), r, weights)[1], lambda f: heads.dispatch_backward(f(x), r)]
    for i, call in enumerate(calls):
        with pytest.raises(ValueError, match="autograd"):
            call(leaf)
            pytest.fail("case %d was taken" % i)
        with torch.no_grad():
            got = call(leaf)
        assert torch.equal(got, call(lambda t: t)), i
        assert torch.equal(call(lambda t: leaf(t).detach()), got), i
    p, q = torch.nn.Parameter(x.clone()), x.clone()
    for v in (p, q):
        heads.AdamW([v], [dout]).step(grad_scale=leaf(torch.ones(1, device="cuda")))
    assert torch.equal(p, q) and p.requires_grad
