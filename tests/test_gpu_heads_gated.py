"""The heads' gated layers on the GPU against plain float64 implementations.

Tolerances, beside those of test_gpu_heads.  An activation or its slope is within
REL(g) = (g^2 + |g| + 20) 2^-22 of the sum of its terms' magnitudes: the exponent's
rounding costs up to 1.5 |g| 2^-24 (for exp(-g^2 / 2): 1.5 g^2 2^-24, of which a complement of
the error function is a product), the hardware's exp and reciprocal a unit in the last
place (2^-23) each, a fitted polynomial up to 16 of them, the few products and sums half a
unit each.  Gates and ups off by d move y by at most 1.13 |u| d + |act(g)| d (no slope of
an activation is above 1.13).  dg and du are rounded to the rows' type before the
products; the biases' gradients sum them unrounded.
"""
import math

import numpy as np
import pytest
import torch

from paper_2011_12490_amd import heads
from test_gpu_heads import BF16, FP32, HALF_ULP, LINEAR_CASES, gen, rand, strided

pytestmark = pytest.mark.gpu

ACTS = list(heads.ACTIVATIONS)
# large tiles; whole lines; narrow with both halves in 128 columns; many stretches
CASES = LINEAR_CASES + [([16000, 16700], 9, 512, 1024, 0, 0), ([9000, 300], 3, 64, 64, 0, 0), ([70000], 0, 128, 128, 0, 0),
                        ([40000, 10], 6, 30, 24, 1, 1)]

# More kernels' cases: counts by head, rows without a head, fan_in, fan_out.  Shallow layers of
# every depth and both widths (odd ones, which do not go to LDS by themselves), rows' gradients
# of shallow ones, weights' of many heads as wholes, and narrow results of middling rows
MORE = [([20000, 0, 13000], 7, I, O) for I in (20, 63, 90, 127, 155, 191, 255, 319) for O in (24, 130)]
MORE += [([32000, 1000], 5, 190, 60), ([32000, 1000], 5, 192, 16), ([32000, 1000], 0, 192, 60), ([32000, 1000], 0, 190, 30),
         ([32000, 1000], 0, 256, 30), ([32000, 1000], 0, 190, 16), ([20] * 64, 3, 256, 256), ([20] * 200, 0, 40, 140), ([5] * 256, 2, 200, 20), ([9000, 300], 3, 400, 24),
         ([3000, 900], 0, 100, 50), ([3000, 900], 0, 128, 64)]


def near(got, want, size, n, rel):
    """size: the products' magnitudes summed; rel: what their factors are off by, of size."""
    bound = ((2 * n + 8) * 2.0 ** -24 + rel) * size + HALF_ULP[got.dtype] * want.abs() + 2.0 ** -110
    off = (got.double() - want).abs() - bound
    assert bool((off <= 0).all()), "worst excess %g" % off.max()


def act_of(g, act):
    """The activation, its slope and the magnitudes of the slope's terms, in float64."""
    if act == "relu":
        slope = (g > 0).double()
        return g.clamp_min(0), slope, slope
    if act == "gelu":
        part, bell = torch.erfc(-g / math.sqrt(2)) / 2, torch.exp(-g * g / 2) / math.sqrt(2 * math.pi)
        return g * part, part + g * bell, part + g.abs() * bell
    part, rest = torch.sigmoid(g), torch.sigmoid(-g)
    if act == "sigmoid":
        return part, part * rest, part * rest
    return g * part, part * (1 + g * rest), part * (1 + g.abs() * rest)


def rel_of(g):
    return (g * g + g.abs() + 20) * 2.0 ** -22


def gated_layer(counts, tail, I, O, pad, shift, dtype, seed):
    g = gen(seed)
    K, R = len(counts), sum(counts) + tail
    x = strided(rand(g, R, I).to(dtype), pad, shift)
    if tail:
        x[R - tail:] = float("nan")  # rows without a head are not looked at
    w = (rand(g, K, 2, O, I) * (1.5 / math.sqrt(I))).to(dtype)
    b = rand(g, K, 2, O)
    offsets = torch.tensor(np.concatenate([[0], np.cumsum(counts)]), dtype=torch.int32, device="cuda")
    return x, w, b, offsets, g


def check_gated(y, pre, x, w, b, offsets, act, I):
    ends = offsets.tolist()
    for h, (start, end) in enumerate(zip(ends, ends[1:])):
        s, halves = slice(start, end), []
        for part in range(2):
            want = x[s].double() @ w[h, part].double().T
            size = x[s].double().abs() @ w[h, part].double().abs().T
            if b is not None:
                want, size = want + b[h, part].double(), size + b[h, part].double().abs()
            halves += [want, size]
        g, g_size, u, u_size = halves
        if pre is not None:
            near(pre[s], torch.cat([g, u], 1), torch.cat([g_size, u_size], 1), I + 1, 0.0)
        value = act_of(g, act)[0]
        near(y[s], value * u, 1.13 * u.abs() * g_size + value.abs() * u_size, I + 1,
             0.0 if not y.numel() else rel_of(g) * value.abs() * u.abs() / (1.13 * u.abs() * g_size + value.abs() * u_size + 2.0 ** -100))
    assert not bool(y[ends[-1]:].any()) and (pre is None or not bool(pre[ends[-1]:].any()))


@pytest.mark.parametrize("dtype", [FP32, BF16])
@pytest.mark.parametrize("at,case", list(enumerate(CASES + [c + (0, 0) for c in MORE])))
def test_gated(at, case, dtype):
    counts, tail, I, O, pad, shift = case
    x, w, b, offsets, _ = gated_layer(*case, dtype, I + O)
    R = x.shape[0]
    full = lambda n: strided(torch.full((R, n), 7.0, dtype=dtype, device="cuda"), pad, shift)  # noqa: E731
    act, bias = ACTS[at % 4], b if at % 3 else None
    y, pre = heads.gated(x, w, bias, offsets, act, out=full(O), out_pre=full(2 * O))
    check_gated(y, pre, x, w, bias, offsets, act, I)
    for out, n in ((y, O), (pre, 2 * O)):
        if pad and R > 1:
            assert bool(out.as_strided((R - 1, pad), (n + pad, 1), out.storage_offset() + n).isnan().all())
    alone, none = heads.gated(x, w, bias, offsets, act)
    assert none is None and torch.equal(alone, y)


@pytest.mark.parametrize("dtype", [FP32, BF16])
@pytest.mark.parametrize("act", ACTS)
def test_every_activation(act, dtype):
    for case in (([3, 5, 0, 1], 2, 63, 65, 0, 0), ([33000, 1], 5, 40, 48, 0, 0), ([900, 700], 0, 264, 136, 0, 0)):
        x, w, b, offsets, _ = gated_layer(*case, dtype, 3)
        y, pre = heads.gated(3 * x, w, b, offsets, act, keep=True)
        check_gated(y, pre, 3 * x, w, b, offsets, act, case[2])


@pytest.mark.parametrize("dtype", [FP32, BF16])
@pytest.mark.parametrize("at,case", list(enumerate(CASES + [c + (0, 0) for c in MORE])))
def test_gated_gradients(at, case, dtype):
    counts, tail, I, O, pad, shift = case
    x, w, _, offsets, g = gated_layer(*case, dtype, I + 7 * O)
    R, K, act = x.shape[0], len(counts), ACTS[(at + 1) % 4]
    dy = strided(rand(g, R, O).to(dtype), pad, shift)
    pre = strided((2 * rand(g, R, 2 * O)).to(dtype), pad, shift)
    if tail:
        dy[R - tail:] = float("nan")
        pre[R - tail:] = float("inf")
    dx, dw, db = heads.gated_backward(dy, pre, x, w, offsets, act)
    assert dw.dtype == dtype and db.dtype == FP32
    ends = offsets.tolist()
    rounded = HALF_ULP[dtype]
    for h in range(K):
        s, n = slice(ends[h], ends[h + 1]), counts[h]
        gate, up, d = pre[s, :O].double(), pre[s, O:].double(), dy[s].double()
        value, slope, slope_size = act_of(gate, act)
        dz = torch.cat([d * up * slope, d * value], 1)
        size = torch.cat([(d * up).abs() * slope_size, (d * value).abs()], 1)
        off = torch.cat([rel_of(gate), rel_of(gate)], 1) * size
        xh, wh = x[s].double(), w[h].double().reshape(2 * O, I)
        near(db[h].reshape(-1), dz.sum(0), size.sum(0), n, off.sum(0) / size.sum(0).clamp_min(2.0 ** -100))
        off = off + rounded * size
        for got, want, both, extra, depth in (
                (dw[h].reshape(2 * O, I), dz.T @ xh, size.T @ xh.abs(), off.T @ xh.abs(), n),
                (dx[s], dz @ wh, size @ wh.abs(), off @ wh.abs(), 2 * O)):
            near(got, want, both, depth, extra / both.clamp_min(2.0 ** -100))
    if tail:
        assert not bool(dx[R - tail:].any())
    none, dw2, db2 = heads.gated_backward(dy, pre, x, w, offsets, act, need_dx=False)
    assert none is None and torch.equal(dw2, dw) and torch.equal(db2, db)


def test_gradients_against_autograd_and_differences():
    """float32 through the layer and back, against autograd in float64 and against central
    differences of the layer in float64: the gradients are those of the formula."""
    x, w, b, offsets, g = gated_layer([40, 0, 23], 0, 27, 36, 0, 0, FP32, 2)
    dy = rand(g, 63, 36)
    for act in ACTS:
        y, pre = heads.gated(x, w, b, offsets, act, keep=True)
        got = heads.gated_backward(dy, pre, x, w, offsets, act)
        leaves = [t.double().cpu().requires_grad_() for t in (x, w, b)]

        def plain(x, w, b):
            parts = []
            for h, (s, e) in enumerate(((0, 40), (40, 40), (40, 63))):
                u = [x[s:e] @ w[h, i].T + b[h, i] for i in range(2)]
                f = {"silu": torch.nn.functional.silu, "gelu": torch.nn.functional.gelu, "relu": torch.relu,
                     "sigmoid": torch.sigmoid}[act]
                parts.append(f(u[0]) * u[1])
            return torch.cat(parts)

        out = plain(*leaves)
        assert torch.allclose(y.double().cpu(), out, rtol=0, atol=1e-4)  # 27 products of magnitude a few: 2^-24 x 62 x 30
        want = torch.autograd.grad(out, leaves, dy.double().cpu())
        for a, e in zip(got, want):
            # 72 products at most for dx, 40 for dw, of magnitudes up to 30: 152 x 2^-24 x 72 x 30
            assert torch.allclose(a.double().cpu(), e, rtol=0, atol=2e-2 * 2.0 ** -10 * 72 * 30 / 10)
        with torch.no_grad():
            for i, leaf in enumerate(leaves):
                way = torch.randn(leaf.shape, dtype=torch.float64, generator=torch.Generator().manual_seed(i))
                step = 1e-6
                there = plain(*[t + step * way if j == i else t for j, t in enumerate(leaves)])
                back = plain(*[t - step * way if j == i else t for j, t in enumerate(leaves)])
                slope = float(((there - back) / (2 * step) * dy.double().cpu()).sum())
                # the gradients' sums of a few thousand float32 values; a ReLU's corner within a step moves little
                assert abs(float((got[i].double().cpu() * way).sum()) - slope) < 1e-3 * max(1.0, abs(slope))


@pytest.mark.parametrize("dtype", [FP32, BF16])
def test_extreme_gates(dtype):
    """Gates far out: no NaN from an overflowing exponential; NaN and infinities stay in their rows."""
    O = 40
    gate = torch.tensor([-3e38, -200.0, -88.0, -30.0, 0.0, 30.0, 88.0, 200.0, 3e38, -0.0], device="cuda").to(dtype)
    pre = torch.ones(gate.numel() + 2, 2 * O, dtype=dtype, device="cuda")
    pre[:-2, :O] = gate[:, None]
    pre[-2, 3] = float("nan")
    pre[-1, O + 5] = float("inf")
    R = pre.shape[0]
    offsets = torch.tensor([0, R], dtype=torch.int32, device="cuda")
    w, x = torch.ones(1, 2, O, 8, dtype=dtype, device="cuda"), torch.ones(R, 8, dtype=dtype, device="cuda")
    dy = torch.ones(R, O, dtype=dtype, device="cuda") / 1024
    for act in ("silu", "gelu", "sigmoid"):
        dx = heads.gated_backward(dy, pre, x, w, offsets, act)[0]
        assert bool(dx[1:8].isfinite().all()) and bool(dx[9].isfinite().all())
        assert bool(dx[-2].isnan().all()) and not bool(dx[-1].isfinite().any())
    ident = torch.zeros(1, 2, O, 2, dtype=dtype, device="cuda")
    ident[0, 0, :, 0] = 1
    ident[0, 1, :, 1] = 1
    xs = torch.ones(gate.numel(), 2, dtype=dtype, device="cuda")
    xs[:, 0] = gate
    offsets = torch.tensor([0, gate.numel()], dtype=torch.int32, device="cuda")
    for act in ("silu", "gelu", "sigmoid", "relu"):
        y, _ = heads.gated(xs, ident, None, offsets, act)
        assert bool(y[1:].isfinite().all())
        assert bool((y[1:3].abs() < 1e-30).all()) and (act == "sigmoid" or bool((y[7] == gate[7]).all()))


@pytest.mark.parametrize("dtype,I,O,counts", [(BF16, 128, 128, [5000, 0, 9000, 70]), (FP32, 63, 128, [3000, 41]),
                                              (BF16, 319, 256, [2100, 35000])])
def test_same_inputs_same_bits(dtype, I, O, counts):
    x, w, b, offsets, g = gated_layer(counts, 0, I, O, 0, 0, dtype, 3)
    dy = rand(g, x.shape[0], O).to(dtype)

    def run():
        y, pre = heads.gated(x, w, b, offsets, keep=True)
        return (y, pre) + heads.gated_backward(dy, pre, x, w, offsets)

    first = run()
    for _ in range(3):
        assert all(torch.equal(a, c) for a, c in zip(first, run()))


def test_offsets_outside_the_rows_are_clamped():
    x, w, b, offsets, _ = gated_layer([20, 30, 14], 0, 40, 48, 0, 0, BF16, 9)
    odd = torch.tensor([-5, 20, 50, 1 << 30], dtype=torch.int32, device="cuda")
    y, pre = heads.gated(x, w, b, offsets, keep=True)
    for a, c in zip(heads.gated(x, w, b, odd, keep=True), (y, pre)):
        assert torch.equal(a, c)
    for a, c in zip(heads.gated_backward(y, pre, x, w, odd), heads.gated_backward(y, pre, x, w, offsets)):
        assert torch.equal(a, c)


def test_no_rows():
    w = torch.ones(3, 2, 5, 4, device="cuda")
    offsets = torch.zeros(4, dtype=torch.int32, device="cuda")
    x = torch.empty(0, 4, device="cuda")
    y, pre = heads.gated(x, w, None, offsets, keep=True)
    assert y.shape == (0, 5) and pre.shape == (0, 10)
    dx, dw, db = heads.gated_backward(y, pre, x, w, offsets, out_weight=torch.full_like(w, 7.0))
    assert dx.shape == (0, 4) and not bool(dw.any()) and not bool(db.any())


def test_on_a_stream_and_from_a_graph():
    """Captured with workspaces of its own and replayed with other inputs between eager work."""
    x, w, b, offsets, g = gated_layer([700, 0, 900], 10, 64, 96, 0, 0, BF16, 4)
    x[-10:] = 0
    dy = rand(g, x.shape[0], 96).to(BF16)
    inputs = [(rand(g, *x.shape).to(BF16), rand(g, *dy.shape).to(BF16)) for _ in range(3)]

    def run():
        y, pre = heads.gated(x, w, b, offsets, "gelu", keep=True)
        return (y, pre) + heads.gated_backward(dy, pre, x, w, offsets, "gelu")

    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        on_stream = run()
    s.synchronize()
    assert all(torch.equal(a, c) for a, c in zip(on_stream, run()))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        captured = run()
    for new_x, new_dy in inputs:
        x.copy_(new_x)
        dy.copy_(new_dy)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, c) for a, c in zip(captured, run()))


def test_python_refusals():
    x, w, b, offsets, _ = gated_layer([5, 6], 0, 8, 12, 0, 0, FP32, 1)
    y, pre = heads.gated(x, w, b, offsets, keep=True)
    for call in (lambda: heads.gated(x, w, b, offsets, act="tanh"), lambda: heads.gated(x, w[:, 0], b, offsets),
                 lambda: heads.gated(x, w, b[:, 0], offsets), lambda: heads.gated(x[:, :7], w, b, offsets),
                 lambda: heads.gated(x, w.bfloat16(), b, offsets), lambda: heads.gated(x, w, b, offsets[:2]),
                 lambda: heads.gated(x, w, b, offsets, out_pre=y), lambda: heads.gated(x, w.requires_grad_(), b, offsets),
                 lambda: heads.gated_backward(y, pre[:, :12], x, w.detach(), offsets),
                 lambda: heads.gated_backward(y, pre, x[:, :7], w.detach(), offsets),
                 lambda: heads.gated_backward(y, pre, x, w.detach(), offsets, need_dx=False, out_x=x),
                 lambda: heads.gated_backward(y, pre, x, w.detach(), offsets, out_weight=b)):
        with pytest.raises(ValueError):
            call()
