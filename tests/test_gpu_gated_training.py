"""Codes, gated heads and orthogonalised updates together, as a training step uses them:
gradients of the whole against autograd and against differences, and steps that run."""
import numpy as np
import pytest
import torch

from paper_2011_12490_amd import heads, scenes, training
from test_gpu_heads import FP32
from test_gpu_muon import check, formula

pytestmark = pytest.mark.gpu


def trainer_and_batch(precision, act="silu", T=400, images=7):
    rng = np.random.default_rng(3)
    t = training.GatedTrainer(rng.uniform(-1, 1, (4, 3)), images, code_dim=5, width=24, depth=2, pos_freqs=3, dir_freqs=1,
                              act=act, precision=precision, seed=1)
    for b in t.bias + [t.out_bias]:
        b.copy_(torch.from_numpy(rng.uniform(-0.2, 0.2, b.shape)).float())
    g = torch.Generator(device="cuda").manual_seed(7)
    x, d = torch.rand(T, 3, generator=g, device="cuda") * 2 - 1, torch.randn(T, 3, generator=g, device="cuda")
    image = torch.randint(-1, images, (T,), generator=g, device="cuda", dtype=torch.int32)  # -1: a sample of no image
    return t, x, d, image, torch.randn(T, 4, generator=g, device="cuda")


def plain(t, x, d, image, leaves):
    """The same in float64 on the CPU, sample by sample's heads."""
    codes, weights, biases, out_w, out_b = leaves
    ids, mix = training.nearest_sites(x, t.sites, t.top_k, t.beta)
    f = {"silu": torch.nn.functional.silu, "gelu": torch.nn.functional.gelu, "sigmoid": torch.sigmoid}[t.act]
    gx = training.encode(x, t.pos_freqs).double().cpu()
    gd = training.encode(d / d.norm(dim=1, keepdim=True), t.dir_freqs).double().cpu()
    code = torch.where((image >= 0).cpu()[:, None], codes[image.long().clamp_min(0).cpu()] * t.code_scale, 0.0)
    want = 0
    for j in range(t.top_k):
        k = ids[:, j].long().cpu()
        h = torch.cat([gx, gd, code], 1)
        for w, b in zip(weights, biases):
            gate, up = ((w[k, i] * h[:, None]).sum(-1) + b[k, i] for i in range(2))
            h = f(gate) * up
        row = (out_w[k] * h[:, None]).sum(-1) + out_b[k]
        want = want + mix[:, j, None].double().cpu() * torch.cat([row[:, :1].clamp_min(0), torch.sigmoid(row[:, 1:])], 1)
    return want


@pytest.mark.parametrize("act", ["silu", "gelu", "sigmoid"])
def test_gradients_of_the_whole(act):
    """float32, against autograd in float64: norms over a parameter's values, since the density's
    ReLU may differ in sign where its sum is within rounding of zero; then one direction
    against differences of the float64 formula."""
    t, x, d, image, dout = trainer_and_batch("fp32", act)
    out = t.forward(x, d, image)
    t.backward(dout)
    params = [t.codes] + t.weight + t.bias + [t.out_weight, t.out_bias]
    got = [t.codes_grad] + t.weight_grad + t.bias_grad + [t.out_weight_grad, t.out_bias_grad]
    leaves = [p.double().cpu().requires_grad_() for p in params]
    n = len(t.weight)
    shaped = lambda v: (v[0], v[1:1 + n], v[1 + n:1 + 2 * n], v[-2], v[-1])  # noqa: E731
    want = plain(t, x, d, image, shaped(leaves))
    assert float((out.cpu() - want.detach()).abs().max()) <= 1e-4
    grads = torch.autograd.grad(want, leaves, dout.double().cpu())
    for a, e in zip(got, grads):
        assert float((a.cpu() - e).norm()) <= 1e-3 * float(e.norm()) + 1e-6
    with torch.no_grad():
        way = [torch.randn(p.shape, dtype=torch.float64, generator=torch.Generator().manual_seed(i)) for i, p in enumerate(leaves)]
        step = 1e-6
        there, back = (plain(t, x, d, image, shaped([p + s * step * v for p, v in zip(leaves, way)])) for s in (1, -1))
        slope = float(((there - back) / (2 * step) * dout.double().cpu()).sum())
        along = sum(float((a.double().cpu() * v).sum()) for a, v in zip(got, way))
        size = sum(float(e.norm() * v.norm()) for e, v in zip(grads, way))
        assert abs(along - slope) <= 1e-3 * size


@pytest.mark.parametrize("precision", ["fp32", "bf16"])
def test_steps_run_and_repeat(precision):
    """A few steps: finite, the copies are the rounded parameters, and the same again bit for bit."""
    def run():
        t, x, d, image, target = trainer_and_batch(precision)
        errors = torch.stack([t.step(x, d, image, target) for _ in range(4)])
        return t, errors

    t, errors = run()
    assert bool(errors.isfinite().all())
    if precision == "bf16":
        for w, c in zip(t.weight + [t.codes, t.out_weight], t.rows_weight + [t.rows_codes, t.rows_out]):
            assert torch.equal(c, w.to(torch.bfloat16))
    twin, again = run()
    assert torch.equal(errors, again) and torch.equal(t.codes, twin.codes)
    assert all(torch.equal(a, b) for a, b in zip(t.weight, twin.weight))


def test_a_step_of_bf16_is_near_float32s():
    """Gradients in bf16 rows: a few roundings of 2^-8 through two layers and back, as norms."""
    got = {}
    for precision in ("fp32", "bf16"):
        t, x, d, image, dout = trainer_and_batch(precision)
        t.forward(x, d, image)
        t.backward(dout)
        got[precision] = [g.float() for g in [t.codes_grad] + t.weight_grad + t.bias_grad + [t.out_weight_grad]]
    for a, e in zip(got["bf16"], got["fp32"]):
        # inputs, weights, codes, two layers' results and gradients: ten roundings of up to 2^-8
        assert float((a - e).norm()) <= 10 * 2.0 ** -8 * float(e.norm())


@pytest.mark.parametrize("precision", ["fp32", "bf16"])
def test_hidden_layers_along_orthogonal_directions(precision):
    """HeadTrainer with Muon: a step moves the hidden weights along orthogonalised momentum and the
    others by AdamW, and the result renders."""
    rng = np.random.default_rng(5)
    arch = scenes.ARCH_TINY
    t = training.HeadTrainer(rng.uniform(-1, 1, (3, 3)), arch, training.start_weights(3, arch, 2), precision, optimizer="muon")
    assert len(t.muon.params) == sum("hidden" in n for n in t.names)
    assert len(t.optimizer.params) == len(t.weight) + len(t.bias) - len(t.muon.params)
    g = torch.Generator(device="cuda").manual_seed(1)
    x, d = torch.rand(900, 3, generator=g, device="cuda") * 2 - 1, torch.randn(900, 3, generator=g, device="cuda")
    before = [w.clone() for w in t.weight]
    t.step(x, d, training.analytic_field(x, d))
    for name, w, was, grad in zip(t.names, t.weight, before, t.weight_grad):
        assert not torch.equal(w, was)
        if "hidden" in name:
            # the first step's update is (1 + momentum) times the gradient
            size = 0.02 * max(1.0, w.shape[1] / w.shape[2]) ** 0.5
            way = heads.orthogonalise(grad * 1.95)
            # p - size X in float32: three roundings.  g + 0.95 g is not 1.95 g to the last bit: two
            # roundings of 2^-24 apart, a matrix of norm 2^-23 beside one of norm 1, of which five
            # steps make 3.4445^5 times as much where the singular values are small
            off = ((was - w) - size * way).square().sum((1, 2)).sqrt()
            assert float(off.max()) <= size * 3.4445 ** 5 * 2.0 ** -23 + 2.0 ** -22 * float(was.square().sum((1, 2)).sqrt().max())
    if precision == "bf16":
        assert all(torch.equal(c, w.to(torch.bfloat16)) for w, c in zip(t.weight, t.rows_weight))
    t.renderer()


def test_fits_run():
    for precision in ("fp32", "bf16"):
        _, errors = training.fit_images(steps=3, samples=512, num_heads=3, images=4, precision=precision)
        assert np.isfinite(errors).all()
    _, errors = training.fit(steps=3, samples=512, num_heads=3, optimizer="muon")
    assert np.isfinite(errors).all()


def adamw_formula(p, g, m, v, step, lr):
    """AdamW's parameters after a step in float64, without decay, and how far float32 may be: three
    roundings of the first moment's terms, 16 of the update (the second moment's sums, a root, a
    quotient), two of the parameter."""
    p, g, m, v = (t.double() for t in (p, g, m.reshape(p.shape), v.reshape(p.shape)))
    size, m = 0.9 * m.abs() + 0.1 * g.abs(), 0.9 * m + 0.1 * g
    root = ((0.999 * v + 0.001 * g * g) / (1 - 0.999 ** step)).sqrt() + 1e-8
    rate = lr / (1 - 0.9 ** step) / root
    return p - rate * m, 2.0 ** -24 * (rate * (3 * size + 16 * m.abs()) + 2 * p.abs()) + lr * 2.0 ** -30


def check_steps(t, run, adamw, muon, lr, muon_lr):
    """adamw, muon: pairs of a parameter and the gradient that belongs to it, in the optimizers' order.
    Three steps of run(), each against the formulas on the state before it."""
    assert len(t.optimizer.params) == len(adamw) and len(t.muon.params) == len(muon)
    for step in range(1, 4):
        was = [(p.clone(), t.optimizer.m[i].clone(), t.optimizer.v[i].clone()) for i, (p, _) in enumerate(adamw)]
        before = [(p.clone(), t.muon.m[i].clone()) for i, (p, _) in enumerate(muon)]
        run()
        for (p, grad), (old, m, v) in zip(adamw, was):
            assert bool(grad.any())
            want, far = adamw_formula(old, grad, m, v, step, lr)
            assert bool(((p.double() - want).abs() <= far).all())
        for (p, grad), (old, m) in zip(muon, before):
            assert bool(grad.any())
            shape = m.shape
            _, want, far = formula(old.view(shape), grad.view(shape), m, 1.0, muon_lr, 0.95, True, 0.0, FP32)
            check(p.view(shape), want, far, 3 * 2.0 ** -24 * want.square().sum((-2, -1)).sqrt())


@pytest.mark.parametrize("precision", ["fp32", "bf16"])
def test_gated_steps_follow_their_own_gradients(precision):
    """Every parameter moves by its optimizer's formula along the gradient that the backward pass left."""
    t, x, d, image, target = trainer_and_batch(precision)
    adamw = [(t.codes, t.codes_grad), (t.out_weight, t.out_weight_grad), (t.out_bias, t.out_bias_grad)] + list(zip(t.bias, t.bias_grad))
    check_steps(t, lambda: t.step(x, d, image, target), adamw, list(zip(t.weight, t.weight_grad)), 2e-3, 0.02)


@pytest.mark.parametrize("precision", ["fp32", "bf16"])
def test_steps_with_muon_follow_their_own_gradients(precision):
    rng = np.random.default_rng(5)
    arch = scenes.ARCH_TINY
    t = training.HeadTrainer(rng.uniform(-1, 1, (3, 3)), arch, training.start_weights(3, arch, 2), precision, optimizer="muon")
    g = torch.Generator(device="cuda").manual_seed(1)
    x, d = torch.rand(900, 3, generator=g, device="cuda") * 2 - 1, torch.randn(900, 3, generator=g, device="cuda")
    pairs = list(zip(t.weight, t.weight_grad))
    hidden = ["hidden" in n for n in t.names]
    adamw = [p for p, h in zip(pairs, hidden) if not h] + list(zip(t.bias, t.bias_grad))
    check_steps(t, lambda: t.step(x, d, training.analytic_field(x, d)), adamw, [p for p, h in zip(pairs, hidden) if h], 5e-4, 0.02)
