"""The training operators on the GPU against plain float64 implementations.

Tolerances.  A sum of n products taken in float32 in any order is within
(n + 1) 2^-24 S of the exact one, S being the sum of the products' magnitudes;
(2 n + 8) 2^-24 S is allowed (the matrix units' own accumulation included).  A
result is then rounded once: 2^-24 of its magnitude in float32, 2^-8 in bf16
(spacing 2^-7 of the leading bit).  Moved values, indices and zeros are exact.
"""
import math

import numpy as np
import pytest
import torch

from paper_2011_12490_amd import heads

pytestmark = pytest.mark.gpu

FP32, BF16 = torch.float32, torch.bfloat16
HALF_ULP = {FP32: 2.0 ** -24, BF16: 2.0 ** -8}


def gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def rand(g, *shape):
    return torch.randn(*shape, generator=g, device="cuda")


def strided(x, pad, shift=0):
    """x with `pad` elements between its rows, `shift` elements into its memory."""
    if not pad and not shift:
        return x
    buf = torch.full((x.shape[0] * (x.shape[1] + pad) + shift,), float("nan"), dtype=x.dtype, device=x.device)
    view = buf[shift:].view(x.shape[0], x.shape[1] + pad)[:, :x.shape[1]]
    view.copy_(x)
    return view


def assert_near(got, want, size, n):
    """got: rounded to its type; want: float64; size: the products' magnitudes summed."""
    bound = (2 * n + 8) * 2.0 ** -24 * size + HALF_ULP[got.dtype] * want.abs() + 2.0 ** -120
    off = (got.double() - want).abs() - bound
    assert bool((off <= 0).all()), "worst excess %g" % off.max()


def order_of(ids, K):
    """offsets, pair, row of the stable order in numpy."""
    flat = ids.reshape(-1)
    key = np.where((flat >= 0) & (flat < K), flat, K)
    pair = np.argsort(key, kind="stable")
    place = np.empty_like(pair)
    place[pair] = np.arange(len(pair))
    row = np.where(key < K, place, -1 - place).reshape(ids.shape)
    return np.searchsorted(key[pair], np.arange(K + 1)), pair, row


def some_ids(seed, T, k, K, masked):
    rng = np.random.default_rng(seed)
    ids = rng.choice(K, size=(T, k), p=(lambda p: p / p.sum())(rng.gamma(1.0, 1.0, K) + 1e-3))
    if masked == "some":
        ids = np.where(rng.random((T, k)) < 0.3, rng.choice([-1, K, 1 << 30, -(1 << 31)], size=(T, k)), ids)
    elif masked == "all":
        ids = np.full((T, k), -1)
    elif masked == "one head":
        ids = np.full((T, k), K - 1)
    return ids.astype(np.int32)


# ---- route ----------------------------------------------------------------------

@pytest.mark.parametrize("T,k,K,masked", [
    (0, 2, 5, "none"), (1, 1, 1, "none"), (1, 1, 1, "all"), (1, 16, 256, "none"), (7, 3, 5, "some"), (64, 1, 2, "some"),
    (4096, 2, 16, "some"), (4097, 2, 16, "some"), (8191, 1, 256, "some"), (8193, 1, 255, "some"), (2731, 3, 64, "one head"),
    (30000, 1, 3, "all"), (65536, 2, 16, "none"), (50001, 7, 100, "some"), (70000, 16, 256, "some")])
def test_route(T, k, K, masked):
    ids = some_ids(T + k, T, k, K, masked)
    r = heads.route(torch.from_numpy(ids).cuda(), K)
    offsets, pair, row = order_of(ids, K)
    assert np.array_equal(r.offsets.cpu().numpy(), offsets)
    assert np.array_equal(r.pair.cpu().numpy(), pair)
    assert np.array_equal(r.row.cpu().numpy(), row)


# ---- rows to the heads and back -------------------------------------------------

ROW_CASES = [  # T, k, K, dim, masked, pad, shift
    (1, 1, 1, 1, "none", 0, 0), (1, 2, 4, 3, "some", 1, 1), (5, 16, 16, 4, "some", 0, 0), (9, 2, 3, 7, "some", 2, 1),
    (33, 2, 16, 8, "some", 0, 0), (257, 3, 16, 9, "none", 0, 1), (130, 2, 16, 63, "some", 0, 0),
    (77, 2, 5, 64, "all", 0, 0), (100, 8, 64, 100, "some", 4, 3), (19, 4, 8, 511, "some", 1, 0), (40, 2, 8, 2051, "one head", 5, 1),
    (3000, 3, 7, 512, "some", 0, 0)]


@pytest.mark.parametrize("dtype", [FP32, BF16])
@pytest.mark.parametrize("T,k,K,D,masked,pad,shift", ROW_CASES)
def test_dispatch_and_its_gradient(T, k, K, D, masked, pad, shift, dtype):
    ids = some_ids(T + D, T, k, K, masked)
    offsets, pair, row = order_of(ids, K)
    r = heads.route(torch.from_numpy(ids).cuda(), K)
    g = gen(T * D)
    x = strided(rand(g, T, D).to(dtype), pad, shift)
    out = heads.dispatch(x, r, strided(torch.zeros(T * k, D, dtype=dtype, device="cuda"), pad, shift))
    want = x[torch.from_numpy(pair // k).cuda()].clone()
    want[offsets[-1]:] = 0
    assert torch.equal(out, want)
    if pad:  # nothing between the rows was written
        assert bool(out.as_strided((T * k - 1, pad), (D + pad, 1), out.storage_offset() + D).isnan().all())
    dout = strided(rand(g, T * k, D).to(dtype), pad, shift)
    dout[offsets[-1]:] = float("nan")  # rows without a head are not looked at
    dx = heads.dispatch_backward(dout, r)
    place = torch.from_numpy(np.where(row < 0, 0, row)).cuda()
    has = torch.from_numpy(row >= 0).cuda()
    terms = torch.where(has[..., None], dout.double()[place], 0.0)
    assert_near(dx, terms.sum(1), terms.abs().sum(1), k)


@pytest.mark.parametrize("dtype", [FP32, BF16])
@pytest.mark.parametrize("T,k,K,D,masked,pad,shift", ROW_CASES)
def test_combine_and_its_gradients(T, k, K, D, masked, pad, shift, dtype):
    ids = some_ids(T + D, T, k, K, masked)
    offsets, pair, row = order_of(ids, K)
    r = heads.route(torch.from_numpy(ids).cuda(), K)
    g = gen(T + 3 * D)
    rows = strided(rand(g, T * k, D).to(dtype), pad, shift)
    rows[offsets[-1]:] = float("nan")
    has = torch.from_numpy(row >= 0).cuda()
    weights = torch.where(has, rand(g, T, k), float("nan"))  # nor are their weights
    place = torch.from_numpy(np.where(row < 0, 0, row)).cuda()
    back = torch.from_numpy(np.where(row < 0, -1 - row, row)).cuda()
    dout = strided(rand(g, T, D).to(dtype), pad, shift)
    for w in (weights, None):
        factor = torch.where(has, 1.0 if w is None else w.double(), 0.0)
        terms = torch.where(has[..., None], rows.double()[place] * factor[..., None], 0.0)
        assert_near(heads.combine(rows, r, w), terms.sum(1), terms.abs().sum(1), k)
        drows, dw = heads.combine_backward(dout, rows, r, w)
        want = torch.empty(T * k, D, dtype=torch.float64, device="cuda")
        want[back.reshape(-1)] = torch.where(has[..., None], dout.double()[:, None] * factor[..., None], 0.0).reshape(-1, D)
        assert_near(drows, want, want.abs(), 1)
        terms = torch.where(has[..., None], rows.double()[place] * dout.double()[:, None], 0.0)
        assert_near(dw, terms.sum(-1), terms.abs().sum(-1), D)
        again, none = heads.combine_backward(dout, None, r, w)
        assert none is None and torch.equal(again, drows)


# ---- the heads' layers ------------------------------------------------------------

LINEAR_CASES = [  # counts by head, rows without a head, fan_in, fan_out, pad, shift
    ([0], 0, 5, 3, 0, 0), ([1], 0, 1, 1, 0, 0), ([0, 0, 0], 7, 8, 8, 0, 0), ([1, 0, 2], 0, 64, 64, 0, 0),
    ([3, 5, 0, 1], 2, 63, 65, 0, 0), ([17, 16, 15], 1, 32, 4, 0, 0), ([65, 127, 129, 0, 1], 70, 39, 128, 0, 0),
    ([130, 1], 0, 319, 256, 0, 0), ([64, 200], 3, 91, 3, 0, 0), ([300], 0, 256, 1, 0, 0), ([257, 0, 63], 200, 96, 160, 5, 3),
    ([40, 300, 8], 5, 128, 128, 8, 0), ([33] * 9, 0, 72, 264, 0, 1), ([5] * 256, 9, 24, 40, 0, 0), ([2, 1100], 0, 283, 136, 0, 0),
    ([9000, 10], 4, 64, 64, 0, 0), ([31, 600], 50, 512, 520, 0, 0), ([2, 3, 0, 1], 1, 1030, 300, 0, 0), ([700, 900], 0, 520, 1032, 0, 0),
    ([9000, 2100, 1], 130, 264, 520, 0, 0), ([9000, 2100, 1], 130, 263, 519, 2, 1), ([40] * 255 + [300], 9, 136, 144, 0, 0),
    ([40] * 256, 0, 131, 137, 0, 0), ([100] * 30 + [0, 1500], 20, 1024, 1032, 0, 0),
    ([20000, 0, 13000, 5], 70, 319, 256, 0, 0), ([20000, 0, 13000, 5], 300, 63, 64, 1, 1), ([33000], 5, 128, 300, 0, 0),
    ([11000, 11100, 11200], 0, 40, 5, 0, 0), ([300] * 120, 0, 190, 130, 2, 1), ([1] * 200 + [33000], 1, 250, 128, 6, 0),
    # few rows and long depths
    ([3, 0, 60, 1], 2, 40, 1500, 0, 0), ([149], 0, 155, 2816, 3, 1), ([7] * 20, 3, 1601, 70, 0, 0), ([33, 31, 32], 0, 1152, 136, 0, 0),
    # too many rows for those, too few to stream
    ([5000, 0, 1300], 40, 300, 333, 0, 0), ([5000, 1300], 40, 264, 328, 0, 0), ([5000, 1300], 40, 263, 331, 2, 1),
    ([21000, 9000], 20, 400, 40, 0, 0), ([21000, 9000], 20, 40, 400, 0, 0), ([21000, 9000], 20, 39, 401, 2, 1),
    # results in whole lines of longer rows
    ([32000, 1000], 5, 128, 256, 64, 0), ([5000, 7000], 5, 512, 640, 64, 0)]


def layer(counts, tail, I, O, pad, shift, dtype, seed):
    g = gen(seed)
    K, R = len(counts), sum(counts) + tail
    x = strided(rand(g, R, I).to(dtype), pad, shift)
    if tail:
        x[R - tail:] = float("nan")  # rows without a head are not looked at
    w = (rand(g, K, O, I) / math.sqrt(I)).to(dtype)
    b = rand(g, K, O)
    offsets = torch.tensor(np.concatenate([[0], np.cumsum(counts)]), dtype=torch.int32, device="cuda")
    return x, w, b, offsets, g


@pytest.mark.parametrize("dtype", [FP32, BF16])
@pytest.mark.parametrize("relu,with_bias", [(False, False), (True, True)])
@pytest.mark.parametrize("counts,tail,I,O,pad,shift", LINEAR_CASES)
def test_linear(counts, tail, I, O, pad, shift, relu, with_bias, dtype):
    x, w, b, offsets, _ = layer(counts, tail, I, O, pad, shift, dtype, I + O)
    R = x.shape[0]
    y = heads.linear(x, w, b if with_bias else None, offsets, relu,
                     strided(torch.full((R, O), 7.0, dtype=dtype, device="cuda"), pad, shift))
    want, size = torch.zeros(R, O, dtype=torch.float64, device="cuda"), torch.zeros(R, O, dtype=torch.float64, device="cuda")
    ends = offsets.tolist()
    for h in range(len(counts)):
        s = slice(ends[h], ends[h + 1])
        want[s] = x[s].double() @ w[h].double().T
        size[s] = x[s].double().abs() @ w[h].double().abs().T
        if with_bias:
            want[s] += b[h].double()
            size[s] += b[h].double().abs()
    assert_near(y, want.clamp_min(0) if relu else want, size, I + 1)
    if tail:
        assert not bool(y[R - tail:].any())
    if pad and R > 1:
        assert bool(y.as_strided((R - 1, pad), (O + pad, 1), y.storage_offset() + O).isnan().all())


@pytest.mark.parametrize("dtype", [FP32, BF16])
@pytest.mark.parametrize("relu", [False, True])
@pytest.mark.parametrize("counts,tail,I,O,pad,shift", LINEAR_CASES)
def test_linear_gradients(counts, tail, I, O, pad, shift, relu, dtype):
    x, w, _, offsets, g = layer(counts, tail, I, O, pad, shift, dtype, I + 7 * O)
    R, K = x.shape[0], len(counts)
    dy = strided(rand(g, R, O).to(dtype), pad, shift)
    y = strided(rand(g, R, O).clamp_min(0).to(dtype), pad, shift) if relu else None
    if tail:
        dy[R - tail:] = float("nan")
    dx, dw, db = heads.linear_backward(dy, x, w, offsets, y)
    ends = offsets.tolist()
    wx, sx = torch.zeros(R, I, dtype=torch.float64, device="cuda"), torch.zeros(R, I, dtype=torch.float64, device="cuda")
    for h in range(K):
        s = slice(ends[h], ends[h + 1])
        dz = dy[s].double()
        if relu:
            dz = torch.where(y[s] > 0, dz, 0.0)
        xh, wh, n = x[s].double(), w[h].double(), counts[h]
        wx[s], sx[s] = dz @ wh, dz.abs() @ wh.abs()
        assert_near(dw[h], dz.T @ xh, dz.abs().T @ xh.abs(), n)
        assert_near(db[h], dz.sum(0), dz.abs().sum(0), n)
    assert_near(dx, wx, sx, O)
    if tail:
        assert not bool(dx[R - tail:].any())
    none, dw2, db2 = heads.linear_backward(dy, x, w, offsets, y, need_dx=False)
    assert none is None and torch.equal(dw2, dw) and torch.equal(db2, db)


@pytest.mark.parametrize("dtype", [FP32, BF16])
def test_relu_keeps_nan_and_masks_it_out_of_gradients(dtype):
    """A NaN output stays NaN; where the output was zero, a NaN gradient is not passed on."""
    x, w, b, offsets, g = layer([40, 30], 0, 48, 72, 0, 0, dtype, 5)
    x[3, 5] = float("nan")
    x[50, 1] = float("inf")
    y = heads.linear(x, w, b, offsets, relu=True)
    assert bool(y[3].isnan().all()) and not bool(y[:3].isnan().any()) and not bool(y[4:50].isnan().any())
    assert bool((y[50].isinf() | (y[50] == 0)).all())
    x, w, b, offsets, g = layer([40, 30], 0, 48, 72, 0, 0, dtype, 6)
    y = heads.linear(x, w, b, offsets, relu=True)
    dy = torch.where(y > 0, rand(g, 70, 72), float("nan")).to(dtype)
    for out in heads.linear_backward(dy, x, w, offsets, y):
        assert bool(out.isfinite().all())


@pytest.mark.parametrize("dtype", [FP32, BF16])
def test_offsets_outside_the_rows_are_clamped(dtype):
    x, w, b, offsets, _ = layer([20, 30, 14], 0, 40, 48, 0, 0, dtype, 9)
    odd = torch.tensor([-5, 20, 50, 1 << 30], dtype=torch.int32, device="cuda")
    assert torch.equal(heads.linear(x, w, b, odd), heads.linear(x, w, b, offsets))
    for a, c in zip(heads.linear_backward(heads.linear(x, w, b, offsets), x, w, odd),
                    heads.linear_backward(heads.linear(x, w, b, offsets), x, w, offsets)):
        assert torch.equal(a, c)


@pytest.mark.parametrize("dtype,I,O,counts", [(BF16, 128, 128, [5000, 0, 9000, 70]), (FP32, 63, 128, [3000, 41]),
                                              (BF16, 319, 256, [2100, 5000])])
def test_same_inputs_same_bits(dtype, I, O, counts):
    x, w, b, offsets, g = layer(counts, 0, I, O, 0, 0, dtype, 3)
    dy = rand(g, x.shape[0], O).to(dtype)
    first = (heads.linear(x, w, b, offsets, True),) + heads.linear_backward(dy, x, w, offsets)
    for _ in range(3):
        again = (heads.linear(x, w, b, offsets, True),) + heads.linear_backward(dy, x, w, offsets)
        assert all(torch.equal(a, c) for a, c in zip(first, again))


# ---- one step through everything ---------------------------------------------------

def mixture(ids, x, w0, b0, w1, b1, weights, K, relu=True):
    r = heads.route(ids, K)
    x0 = heads.dispatch(x, r)
    y0 = heads.linear(x0, w0, b0, r.offsets, relu)
    y1 = heads.linear(y0, w1, b1, r.offsets)
    return r, x0, y0, y1, heads.combine(y1, r, weights)


def mixture_backward(dout, r, x0, y0, y1, w0, w1, weights, relu=True):
    dy1, dweights = heads.combine_backward(dout, y1, r, weights)
    dy0, dw1, db1 = heads.linear_backward(dy1, y0, w1, r.offsets)
    dx0, dw0, db0 = heads.linear_backward(dy0, x0, w0, r.offsets, y0 if relu else None)
    return heads.dispatch_backward(dx0, r), dw0, db0, dw1, db1, dweights


def mixture_inputs(T, k, K, I, H, O, seed):
    g = gen(seed)
    ids = torch.from_numpy(some_ids(seed, T, k, K, "some")).cuda()
    return (ids, rand(g, T, I), rand(g, K, H, I) / math.sqrt(I), 0.1 * rand(g, K, H), rand(g, K, O, H) / math.sqrt(H),
            0.1 * rand(g, K, O), torch.rand(T, k, generator=g, device="cuda")), g


def test_gradients_of_a_two_layer_mixture_against_autograd():
    """float32 against autograd in float64 on the CPU; a sample is the sum over
    its pairs, so shared heads and repeated inputs are in it."""
    K, T, k = 5, 300, 3
    (ids, *args), g = mixture_inputs(T, k, K, 27, 64, 4, 11)
    r, x0, y0, y1, out = mixture(ids, *args, K)
    dout = rand(g, T, 4)
    got = mixture_backward(dout, r, x0, y0, y1, args[1], args[3], args[5])
    leaves = [a.double().cpu().requires_grad_() for a in args]
    x, w0, b0, w1, b1, weights = leaves
    want = torch.zeros(T, 4, dtype=torch.float64)
    for h in range(K):
        for j in range(k):
            t = torch.nonzero(ids.cpu()[:, j] == h)[:, 0]
            want = want.index_add(0, t, (torch.relu(x[t] @ w0[h].T + b0[h]) @ w1[h].T + b1[h]) * weights[t, j, None])
    assert float((out.cpu() - want.detach()).abs().max()) < 64 * 2.0 ** -24 * 64  # sums of at most 64 + 27 terms of a few units
    want.backward(dout.double().cpu())
    for name, a, leaf in zip("dx dw0 db0 dw1 db1 dweights".split(), got, leaves):
        # sums of up to 300 terms behind sums of 64: n 2^-24 of the largest gradient, with as much again for the size of the terms
        bound = 2 * 400 * 2.0 ** -24 * float(leaf.grad.abs().max())
        assert float((a.cpu() - leaf.grad).abs().max()) <= bound, name


def test_gradients_against_differences():
    """Without the ReLU the mixture is linear in each of its arguments, so a central
    difference of any size is its directional derivative: <gradient, d> =
    (f(a + d) - f(a - d)) / 2, f = <dout, mixture(a)>, up to rounding."""
    K, T, k = 4, 200, 2
    (ids, *args), g = mixture_inputs(T, k, K, 31, 40, 5, 12)
    dout = rand(g, T, 5)
    r, x0, y0, y1, _ = mixture(ids, *args, K, relu=False)
    grads = mixture_backward(dout, r, x0, y0, y1, args[1], args[3], args[5], relu=False)

    def f(a):
        return float((mixture(ids, *a, K, relu=False)[-1].double() * dout.double()).sum())

    for i, grad in enumerate(grads):
        d = rand(g, *args[i].shape) * 0.5
        up, down = ([a + s * d if j == i else a for j, a in enumerate(args)] for s in (1, -1))
        fu, fd = f(up), f(down)
        want = float((grad.double() * d.double()).sum())
        # 1000 outputs of a few units, each from sums of 31, 40 and 2 terms: 2^-24 of each product's size
        bound = 2 * (31 + 40 + 2 + 8) * 2.0 ** -24 * float(dout.abs().sum()) * 8
        assert abs((fu - fd) / 2 - want) <= bound, i


# ---- AdamW -----------------------------------------------------------------------

def adamw_inputs(sizes, dtype, grad_dtype, seed, shift=0):
    g = gen(seed)

    def one(n, t):
        return torch.zeros(n + shift, dtype=t, device="cuda")[shift:].copy_((rand(g, n) * 0.1).to(t))

    return [one(n, dtype) for n in sizes], [one(n, grad_dtype) for n in sizes], g


SIZES = [1, 3, 255, 256, 257, 1000, 1024, 1025, 4099, 70001]


@pytest.mark.parametrize("dtype,grad_dtype,copy,shift", [(FP32, FP32, False, 0), (FP32, BF16, True, 0), (BF16, BF16, False, 0),
                                                         (FP32, FP32, True, 1), (BF16, FP32, False, 3)])
def test_adamw_32(dtype, grad_dtype, copy, shift):
    """Three steps against float64.  Each step adds a few roundings of 2^-24 to the
    moments (3 each) and to the parameter (of its size, 2; and of lr: 8)."""
    p, grads, g = adamw_inputs(SIZES, dtype, grad_dtype, 1, shift)
    copies = [torch.zeros_like(x, dtype=BF16) for x in p] if copy else None
    scale = torch.tensor([0.37], device="cuda")
    lr, b1, b2, eps, wd = 1e-2, 0.9, 0.99, 1e-8, 0.1
    opt = heads.AdamW(p, grads, lr=lr, betas=(b1, b2), eps=eps, weight_decay=wd, copies=copies)
    ref = [[x.double(), torch.zeros_like(x, dtype=torch.float64), torch.zeros_like(x, dtype=torch.float64)] for x in p]
    for t in range(1, 4):
        for x in grads:
            x.copy_((rand(g, *x.shape) * 0.1).to(x.dtype))
        before = [x.clone() for x in p]
        opt.step(grad_scale=scale)
        for i, (rp, rm, rv) in enumerate(ref):
            gd = grads[i].double() * scale.double()
            rm.mul_(b1).add_(gd * (1 - b1))
            rv.mul_(b2).add_(gd * gd * (1 - b2))
            rp.copy_(before[i].double())  # a bf16 parameter is rounded each step: from what it was
            rp.mul_(1 - lr * wd).sub_(lr / (1 - b1 ** t) * rm / (rv.sqrt() / math.sqrt(1 - b2 ** t) + eps))
            tiny = 2.0 ** -24 * 0.1 * t
            assert float((opt.m[i].double() - rm).abs().max()) <= 6 * tiny
            assert float(((opt.v[i].double() - rv).abs() - 8 * t * 2.0 ** -24 * rv).max()) <= 0
            # an update of lr times at most ~3: its relative error grows where m cancels
            bound = 2.0 ** -24 * (4 * rp.abs() + 40 * t * 3 * lr) + 8 * t * 2.0 ** -24 * lr * 0.1 / (rv.sqrt() + 1e-12)
            bound = bound + (HALF_ULP[BF16] * rp.abs() if dtype == BF16 else 0)
            assert float(((p[i].double() - rp).abs() - bound).max()) <= 0, (t, i)
            if copy:
                assert torch.equal(copies[i], p[i].to(BF16))


def to8(x, root):
    """The code of x over its block's scale, with elementary float32 operations."""
    n = x.numel()
    y = torch.zeros(-(-n // 256) * 256, device=x.device)
    y[:n] = x
    y = y.reshape(-1, 256)
    fine = torch.where(y.isfinite(), y, 0.0)
    scale = (fine.abs().amax(1, keepdim=True) * y.new_tensor(1 / 448)).clamp_min(2.0 ** -120)
    q = (fine * scale.reciprocal()).clamp(-448, 448)
    if root:
        q = torch.where(fine > 0, q.clamp_min(2.0 ** -9), q)
    q = torch.where(y.isfinite(), q, float("nan"))
    return q.reshape(-1)[:n].to(torch.float8_e4m3fn), scale.reshape(-1)


@pytest.mark.parametrize("dtype,grad_dtype,shift", [(FP32, FP32, 0), (FP32, BF16, 1), (BF16, BF16, 0)])
def test_adamw_8(dtype, grad_dtype, shift):
    """Each step's codes are exactly those of the moments in float32 (every
    operation rounded alone), and the parameter takes the moments before they are
    rounded to 8 bits."""
    p, grads, g = adamw_inputs(SIZES, dtype, grad_dtype, 2, shift)
    lr, b1, b2, eps, wd = 1e-2, 0.9, 0.99, 1e-8, 0.1
    opt = heads.AdamW(p, grads, lr=lr, betas=(b1, b2), eps=eps, weight_decay=wd, state_bits=8)
    f = lambda x: torch.tensor(x, dtype=FP32, device="cuda")  # noqa: E731
    for t in range(1, 5):
        for i, x in enumerate(grads):  # sizes from block to block over many orders of magnitude
            size = torch.exp(rand(g, -(-x.numel() // 256)) * 6).repeat_interleave(256)[:x.numel()]
            x.copy_((rand(g, *x.shape) * size * (torch.rand(x.shape, generator=g, device="cuda") > 0.2)).to(x.dtype))
            if i % 3 == 2:
                x.zero_()
        before = [x.clone() for x in p]
        old = [opt.moments(i) for i in range(len(p))]
        opt.step()
        for i, (m, root) in enumerate(old):
            gr = grads[i].float()
            m = m * f(b1) + gr * f(1 - b1)
            root = torch.sqrt((root * root) * f(b2) + (gr * gr) * f(1 - b2))
            x = before[i].float() * f(1 - lr * wd) - m / (root * f(1 / math.sqrt(1 - b2 ** t)) + f(eps)) * f(lr / (1 - b1 ** t))
            for new, codes, scale, is_root in ((m, opt.m[i], opt.m_scale[i], False), (root, opt.v[i], opt.v_scale[i], True)):
                want, want_scale = to8(new, is_root)
                assert torch.equal(scale, want_scale)
                assert torch.equal(codes.view(torch.uint8) & (0x7F if is_root else 0xFF), want.view(torch.uint8))
            assert torch.equal(p[i], x.to(dtype))


def test_adamw_not_finite():
    """A gradient that is not finite stays with its own value; in 8 bits its block's
    scale is that of the others."""
    for bits in (32, 8):
        p, grads, _ = adamw_inputs([700], FP32, FP32, 3)
        grads[0][5], grads[0][300] = float("nan"), float("inf")
        clean = [grads[0].clone()]
        clean[0][5] = clean[0][300] = 0.0
        q = [p[0].clone()]
        opt, ref = heads.AdamW(p, grads, state_bits=bits), heads.AdamW(q, clean, state_bits=bits)
        opt.step()
        ref.step()
        bad = torch.zeros(700, dtype=torch.bool, device="cuda")
        bad[5] = bad[300] = True
        assert torch.equal(p[0][~bad], q[0][~bad]) and not bool(p[0][bad].isfinite().any())
        for a, b in zip(opt.moments(0), ref.moments(0)):
            assert torch.equal(a[~bad], b[~bad]) and not bool(a[bad].isfinite().any())


def test_adamw_of_nothing():
    """Zero gradients leave zero moments; without decay the parameter stays."""
    for bits in (32, 8):
        p = [torch.ones(300, device="cuda")]
        opt = heads.AdamW(p, [torch.zeros(300, device="cuda")], weight_decay=0.0, state_bits=bits)
        opt.step()
        opt.step()
        assert bool((p[0] == 1).all()) and not bool(opt.moments(0)[0].any()) and not bool(opt.moments(0)[1].any())


# ---- streams, graphs, refusals -----------------------------------------------------

def test_on_a_stream_of_its_own():
    K, T, k = 4, 5000, 2
    (ids, *args), _ = mixture_inputs(T, k, K, 63, 64, 4, 21)
    want = mixture(ids, *args, K)[-1]
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        got = mixture(ids, *args, K)[-1]
    s.synchronize()
    assert torch.equal(got, want)


def test_replayed_from_a_graph():
    """A training step captured once and replayed on new inputs, every replay
    against the eager one, other work in between."""
    K, T, k = 6, 9000, 2
    (ids, *args), g = mixture_inputs(T, k, K, 39, 64, 4, 22)
    dout = rand(g, T, 4)

    def step(ids, args, dout):
        r, x0, y0, y1, out = mixture(ids, *args, K)
        return (out,) + mixture_backward(dout, r, x0, y0, y1, args[1], args[3], args[5])

    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        step(ids, args, dout)
    s.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=s):
        captured = step(ids, args, dout)
    for i in range(4):
        ids.copy_(torch.from_numpy(some_ids(50 + i, T, k, K, "some")))
        args[0].copy_(rand(g, *args[0].shape))
        dout.copy_(rand(g, T, 4))
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        want = step(ids, args, dout)
        assert all(torch.equal(a, b) for a, b in zip(captured, want)), i


def test_python_refusals():
    (ids, x, w0, b0, *_), _ = mixture_inputs(50, 2, 3, 16, 24, 4, 30)
    r = heads.route(ids, 3)
    rows = heads.dispatch(x, r)
    bad = [
        lambda: heads.route(ids.long(), 3), lambda: heads.route(ids[:, :1], 3), lambda: heads.route(ids, 0), lambda: heads.route(ids, 257),
        lambda: heads.dispatch(x[:-1], r), lambda: heads.dispatch(x.half(), r), lambda: heads.dispatch(x.T, r),
        lambda: heads.dispatch(x, r, torch.empty(99, 16, device="cuda")), lambda: heads.dispatch(x.cpu(), r),
        lambda: heads.dispatch(x[:1].expand(50, 16), r),
        lambda: heads.combine(rows, r, torch.ones(50, 3, device="cuda")), lambda: heads.combine(rows[:-1], r),
        lambda: heads.combine_backward(x, rows.to(BF16), r), lambda: heads.combine_backward(x, None, r, out_weights=torch.ones(50, 2, device="cuda")),
        lambda: heads.linear(rows, w0.to(BF16), b0, r.offsets), lambda: heads.linear(rows, w0, b0.to(BF16), r.offsets),
        lambda: heads.linear(rows, w0, b0, r.offsets[:-1]), lambda: heads.linear(rows, w0, b0, r.offsets.long()),
        lambda: heads.linear(rows[:, :15], w0, b0, r.offsets), lambda: heads.linear(rows, w0[:, ::2], b0, r.offsets),
        lambda: heads.linear_backward(rows, rows, w0, r.offsets),
        lambda: heads.AdamW([x], [x[:-1]]), lambda: heads.AdamW([x], []), lambda: heads.AdamW([x], [x], state_bits=16),
        lambda: heads.AdamW([x.half()], [x]), lambda: heads.AdamW([x], [x], m=[x.to(BF16)], v=[x]),
        lambda: heads.AdamW([x], [x], m_scale=[x]), lambda: heads.AdamW([x], [x], copies=[x]),
    ]
    for i, call in enumerate(bad):
        with pytest.raises(ValueError):
            call()
            print("case", i)


# ---- beyond 32 bits ------------------------------------------------------------------

def far_rows(rows, dim, stride, dtype):
    """Rows so far apart that the last ones start behind 2^32 bytes."""
    buf = torch.empty((rows * stride,), dtype=dtype, device="cuda")
    view = buf.view(rows, stride)[:, :dim]
    assert (rows - 1) * stride * dtype.itemsize > 1 << 32
    return view


@pytest.mark.parametrize("dtype,stride", [(BF16, 1 << 20), (FP32, (1 << 19) + 1)])
def test_rows_beyond_32_bits(dtype, stride):
    """Dispatch, combine and a layer with its gradients on rows behind 2^32 bytes give
    what they give on rows side by side."""
    R, I, O = 2304, 40, 72
    g = gen(40)
    x = far_rows(R, I, stride, dtype)
    x.copy_(rand(g, R, I).to(dtype))
    near = x.contiguous()
    w, b = (rand(g, 2, O, I) / 6).to(dtype), rand(g, 2, O)
    offsets = torch.tensor([0, 1000, R], dtype=torch.int32, device="cuda")
    y = heads.linear(near, w, b, offsets, True)
    far_y = heads.linear(x, w, b, offsets, True, far_rows(R, O, stride, dtype))
    dy = rand(g, R, O).to(dtype)
    want = heads.linear_backward(dy, near, w, offsets, y)
    got = heads.linear_backward(dy, x, w, offsets, far_y, out_x=far_rows(R, I, stride, dtype))
    # the order of sums goes by the form that a stride's alignment allows
    assert_near(far_y, y.double(), y.double().abs() + 10, I)
    assert_near(got[0], want[0].double(), want[0].double().abs() + 10, O)
    for a, c in zip(got[1:], want[1:]):
        assert_near(a, c.double(), c.double().abs() + 100, R)
    ids = torch.from_numpy(some_ids(1, R // 2, 2, 3, "some")).cuda()
    r = heads.route(ids, 3)
    half = x[:R // 2]
    assert torch.equal(heads.dispatch(half, r, far_rows(R, I, stride, dtype)), heads.dispatch(near[:R // 2], r))
    weights = torch.rand(R // 2, 2, generator=g, device="cuda")
    assert torch.equal(heads.combine(x, r, weights), heads.combine(near, r, weights))
    for a, c in zip(heads.combine_backward(half, x, r, weights), heads.combine_backward(near[:R // 2], near, r, weights)):
        assert torch.equal(a, c)


def test_adamw_of_more_than_2_31_values():
    """The last values of a tensor of 2^31 + 1000 in 8 bits are updated as a tensor of
    their own is."""
    n, tail = (1 << 31) + 1000, (1 << 31) - 512
    p, grad = torch.zeros(n, dtype=BF16, device="cuda"), torch.zeros(n, dtype=BF16, device="cuda")
    g = gen(41)
    p[tail:] = (rand(g, n - tail) * 0.1).to(BF16)
    grad[tail:] = (rand(g, n - tail) * 0.1).to(BF16)
    q = p[tail:].clone()
    opt, ref = heads.AdamW([p], [grad], state_bits=8), heads.AdamW([q], [grad[tail:].clone()], state_bits=8)
    for _ in range(2):
        opt.step()
        ref.step()
    assert torch.equal(p[tail:], q) and not bool(p[:256].any()) and not bool(p[tail - 512:tail].any())
    assert torch.equal(opt.m[0][tail:].view(torch.uint8), ref.m[0].view(torch.uint8))
    assert torch.equal(opt.v_scale[0][tail // 256:], ref.v_scale[0])
