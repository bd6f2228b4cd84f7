"""What the gated layers, lookups and orthogonalised updates take at their edges: rows
behind 2^32 bytes, one row of a wide buffer, two calls at once, the same rows twice,
tensors that autograd follows, and a run of them all in one graph."""
import pytest
import torch
from torch.autograd import forward_ad

from paper_2011_12490_amd import heads
from test_gpu_heads import BF16, FP32, far_rows, gen, rand
from test_gpu_heads_gated import gated_layer
from test_gpu_heads_limits import one_row

pytestmark = pytest.mark.gpu


def near(a, c, most):
    """Sums of the same products in another order: 2^-24 for each of up to 4,608 products of
    magnitudes that add up to less than `most`; and a rounding to bf16 to either side."""
    bound = 4608 * 2.0 ** -24 * most + (2.0 ** -7 if a.dtype == BF16 else 2.0 ** -23) * c.double().abs()
    assert bool(((a.double() - c.double()).abs() <= bound).all())


@pytest.mark.parametrize("dtype,stride", [(BF16, 1 << 20), (FP32, (1 << 19) + 1)])
@pytest.mark.parametrize("I,O", [(40, 72), (150, 136)])
def test_rows_beyond_32_bits(dtype, stride, I, O):
    R = 2304
    x, w, b, offsets, g = gated_layer([1000, R - 1000], 0, I, O, 0, 0, dtype, 5)
    y, pre = heads.gated(x, w, b, offsets, "gelu", keep=True)
    dy = rand(g, R, O).to(dtype)
    want = heads.gated_backward(dy, pre, x, w, offsets, "gelu")
    far = lambda n: far_rows(R, n, stride, dtype)  # noqa: E731
    fx = far(I).copy_(x)
    fy, fpre = heads.gated(fx, w, b, offsets, "gelu", out=far(O), out_pre=far(2 * O))
    near(fy, y, 100)
    near(fpre, pre, 20)
    del fx
    fpre.copy_(pre)
    fx = far(I).copy_(x)
    got = heads.gated_backward(dy, fpre, fx, w, offsets, "gelu", out_x=far(I))
    near(got[0], want[0], 100)
    near(got[1], want[1], 1000)
    near(got[2], want[2], 1000)


@pytest.mark.parametrize("dtype", [FP32, BF16])
def test_one_row_of_a_wide_buffer(dtype):
    x, w, b, offsets, g = gated_layer([0, 1], 0, 40, 72, 0, 0, dtype, 1)
    y, pre = heads.gated(x, w, b, offsets, keep=True)
    dy = rand(g, 1, 72).to(dtype)
    for a, c in zip(heads.gated(one_row(x), w, b, offsets, out=one_row(torch.zeros_like(y)), out_pre=one_row(torch.zeros_like(pre))), (y, pre)):
        assert torch.equal(a, c)
    for a, c in zip(heads.gated_backward(one_row(dy), one_row(pre), one_row(x), w, offsets, out_x=one_row(x)),
                    heads.gated_backward(dy, pre, x, w, offsets)):
        assert torch.equal(a, c)
    ids = torch.tensor([0], dtype=torch.int32, device="cuda")
    assert torch.equal(heads.lookup(one_row(x), ids, 2.0), 2 * x)
    assert torch.equal(heads.lookup_backward(one_row(x), ids, 1, 2.0), 2 * x.float())


def test_two_calls_at_once():
    """On two streams, each with its own workspace."""
    x, w, b, offsets, g = gated_layer([3000, 0, 6000], 40, 160, 96, 0, 0, BF16, 4)
    x[-40:] = 0
    dy, table = rand(g, x.shape[0], 96).to(BF16), rand(g, 300, 96)
    ids = torch.randint(0, 300, (x.shape[0],), generator=g, device="cuda", dtype=torch.int32)
    matrices = rand(g, 6, 200, 300)

    def run():
        y, pre = heads.gated(x, w, b, offsets, keep=True)
        return (y, pre) + heads.gated_backward(dy, pre, x, w, offsets) + (
            heads.lookup(table, ids), heads.lookup_backward(dy, ids, 300), heads.orthogonalise(matrices))

    want = run()
    streams = [torch.cuda.Stream() for _ in range(2)]
    got = []
    for s in streams:
        s.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(s):
            got.append([run() for _ in range(3)])
    for s in streams:
        s.synchronize()
    for runs in got:
        for outs in runs:
            assert all(torch.equal(a, c) for a, c in zip(outs, want))


def test_a_run_of_them_in_a_graph():
    """Lookup, gated layers, their gradients and the table's, recorded together; the updates' direction
    too, and the step itself beside the replays."""
    x, w, b, offsets, g = gated_layer([500, 300, 0], 0, 48, 64, 0, 0, BF16, 6)
    table = rand(g, 90, 48).to(BF16)
    ids = torch.randint(-1, 90, (800,), generator=g, device="cuda", dtype=torch.int32)
    dy = rand(g, 800, 64).to(BF16)
    others = [(torch.randint(-1, 90, (800,), generator=g, device="cuda", dtype=torch.int32), rand(g, 800, 64).to(BF16)) for _ in range(3)]

    def run():
        rows = heads.lookup(table, ids, 1.5)
        y, pre = heads.gated(rows, w, b, offsets, keep=True)
        dx, dw, db = heads.gated_backward(dy, pre, rows, w, offsets)
        return y, dw, db, heads.lookup_backward(dx, ids, 90, 1.5), heads.orthogonalise(dw.view(6, 64, 48))

    run()
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        captured = run()
    for new_ids, new_dy in others:
        ids.copy_(new_ids)
        dy.copy_(new_dy)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, c) for a, c in zip(captured, run()))


def test_a_padded_batch():
    """Samples without a row and rows without a head, of any content, change nothing for the others."""
    x, w, b, offsets, g = gated_layer([70, 50], 8, 24, 40, 0, 0, FP32, 7)
    y, pre = heads.gated(x, w, b, offsets, keep=True)
    clean = x.clone()
    clean[-8:] = 0
    assert torch.equal(heads.gated(clean, w, b, offsets)[0], y) and not bool(y[-8:].any())
    dy = rand(g, 128, 40)
    want = heads.gated_backward(dy, pre, clean, w, offsets)
    dy[-8:], pre[-8:] = float("inf"), float("nan")
    for a, c in zip(heads.gated_backward(dy, pre, x, w, offsets), want):
        assert torch.equal(a, c)
    ids = torch.cat([torch.arange(120, device="cuda") % 7, torch.full((8,), -1, device="cuda")]).int()
    assert torch.equal(heads.lookup_backward(dy, ids, 7), heads.lookup_backward(dy[:120], ids[:120], 7))


def test_tensors_that_autograd_follows():
    x, w, b, offsets, g = gated_layer([5, 6], 0, 8, 12, 0, 0, FP32, 1)
    y, pre = heads.gated(x, w, b, offsets, keep=True)
    table, ids = rand(g, 4, 8), torch.zeros(11, dtype=torch.int32, device="cuda")
    leaf = lambda t: t.clone().requires_grad_()  # noqa: E731
    calls = [lambda f: heads.gated(f(x), w, b, offsets), lambda f: heads.gated(x, f(w), b, offsets), lambda f: heads.gated(x, w, f(b), offsets),
             lambda f: heads.gated_backward(f(y), pre, x, w, offsets), lambda f: heads.gated_backward(y, f(pre), x, w, offsets),
             lambda f: heads.lookup(f(table), ids), lambda f: heads.lookup_backward(f(x), ids, 4), lambda f: heads.orthogonalise(f(table))]
    for call in calls:
        with pytest.raises(ValueError, match="requires a gradient"):
            call(leaf)
        with torch.no_grad():
            call(leaf)
    # the optimizer's parameters may be leaves, as AdamW's
    p = leaf(table)
    heads.Muon([p], [rand(g, 4, 8)], lr=0.1).step()
    assert p.requires_grad and not torch.equal(p.detach(), table)


def test_a_backward_pass_in_a_graph_beside_live_autograd():
    """Recorded while autograd holds a graph of the same weights: nothing here is autograd's."""
    x, w, b, offsets, g = gated_layer([50, 30], 0, 16, 24, 0, 0, FP32, 3)
    leaf = w.clone().requires_grad_()
    loss = (leaf * leaf).sum()
    y, pre = heads.gated(x, leaf.detach(), b, offsets, keep=True)
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        grads = heads.gated_backward(y, pre, x, leaf.detach(), offsets)
    graph.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(a, c) for a, c in zip(grads, heads.gated_backward(y, pre, x, leaf.detach(), offsets)))
    loss.backward()
    assert torch.equal(leaf.grad, 2 * w)


def test_tensors_with_forward_mode_tangents():
    """Refused, also where nothing records a graph: the results would silently be without them."""
    x, w, b, offsets, g = gated_layer([5, 6], 0, 8, 12, 0, 0, FP32, 1)
    y, pre = heads.gated(x, w, b, offsets, keep=True)
    table, ids = rand(g, 4, 8), torch.zeros(11, dtype=torch.int32, device="cuda")
    p, m = rand(g, 4, 8), torch.zeros(4, 8, device="cuda")
    optimizers = [heads.Muon([p], [table]), heads.AdamW([p], [table])]
    one = torch.ones(1, device="cuda")
    plain = [lambda f: heads.gated(f(x), w, b, offsets), lambda f: heads.gated(x, f(w), b, offsets), lambda f: heads.gated(x, w, f(b), offsets),
             lambda f: heads.gated_backward(f(y), pre, x, w, offsets), lambda f: heads.gated_backward(y, f(pre), x, w, offsets),
             lambda f: heads.lookup(f(table), ids), lambda f: heads.lookup_backward(f(x), ids, 4), lambda f: heads.orthogonalise(f(table)),
             lambda f: heads.linear(f(x), w[:, 0].contiguous(), b[:, 0].contiguous(), offsets),
             lambda f: heads.Muon([p], [f(table)]), lambda f: heads.Muon([f(p)], [table], m=[m]),
             lambda f: optimizers[0].step(f(one)), lambda f: optimizers[1].step(grad_scale=f(one))]
    with forward_ad.dual_level():
        for call in plain:
            for mode in (torch.enable_grad, torch.no_grad):
                with mode(), pytest.raises(ValueError, match="tangent"):
                    call(lambda t: forward_ad.make_dual(t, torch.ones_like(t)))
            call(lambda t: t)  # without one, within a level
            call(lambda t: forward_ad.unpack_dual(forward_ad.make_dual(t, torch.ones_like(t))).primal)


def test_views_that_torch_has_yet_to_negate():
    """The imaginary part of a conjugate: memory of the other sign.  Refused, and right once resolved."""
    z = torch.complex(torch.zeros(3, 1, device="cuda"), torch.tensor([[1.0], [2.0], [3.0]], device="cuda")).conj()
    table, one = z.imag, z[0, 0:1].imag
    ids = torch.tensor([2, 0], dtype=torch.int32, device="cuda")
    p, m = torch.ones(4, 8, device="cuda"), torch.zeros(4, 8, device="cuda")
    muon = heads.Muon([p], [torch.ones(4, 8, device="cuda")], m=[m])
    for call in (lambda f: heads.lookup(f(table), ids), lambda f: heads.lookup_backward(f(table)[:2], ids, 3),
                 lambda f: heads.lookup(z.real, ids, out=f(table)[:2]), lambda f: heads.orthogonalise(f(one)[None]),
                 lambda f: muon.step(f(one))):
        with pytest.raises(ValueError, match="negated"):
            call(lambda t: t)
        call(lambda t: t.resolve_neg().clone())
    assert heads.lookup(table.resolve_neg(), ids).flatten().tolist() == [-3.0, -1.0]
    assert float(m[0, 0]) == -1.0  # a step whose gradients were scaled by -1


@pytest.mark.parametrize("dtype", [FP32, BF16])
@pytest.mark.parametrize("K,O,I", [(5, 40, 60), (3, 200, 128), (2, 90, 400), (3, 300, 200)])
def test_orthogonalise_in_place(K, O, I, dtype):
    x = rand(gen(2), K, O, I).to(dtype)
    want = heads.orthogonalise(x)
    assert heads.orthogonalise(x, out=x) is x and torch.equal(x, want)


def test_outputs_that_share_memory():
    x, w, b, offsets, g = gated_layer([70, 50], 8, 24, 24, 0, 0, BF16, 7)
    wide = torch.zeros(128, 24 * 4 + 3, dtype=BF16, device="cuda")
    part = lambda at, n: wide[:, at:at + n]  # noqa: E731
    part(0, 24).copy_(x)
    y, pre = heads.gated(x, w, b, offsets, keep=True)
    # columns side by side in one buffer do not overlap
    got = heads.gated(part(0, 24), w, b, offsets, out=part(24, 24), out_pre=part(48, 48))
    assert torch.equal(got[0], y) and torch.equal(got[1], pre) and not bool(wide[:, 96:].any())
    dy, table, ids = rand(g, 128, 24).to(BF16), rand(g, 24, 24), torch.zeros(24, dtype=torch.int32, device="cuda")
    for call in (lambda: heads.gated(x, w, b, offsets, out=x), lambda: heads.gated(part(0, 24), w, b, offsets, out=part(23, 24)),
                 lambda: heads.gated(x, w, b, offsets, out=part(24, 24), out_pre=part(47, 48)),
                 lambda: heads.gated_backward(dy, pre, x, w, offsets, out_x=dy), lambda: heads.gated_backward(dy, pre, x, w, offsets, out_weight=w),
                 lambda: heads.lookup(table, ids, out=table), lambda: heads.lookup_backward(table, ids, 24, out=table),
                 lambda: heads.orthogonalise(table[:12], out=table[6:18])):
        with pytest.raises(ValueError, match="overlaps"):
            call()
