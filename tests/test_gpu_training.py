"""Heads trained with the operators: the same field as the renderer's, gradients of
a whole head network against autograd, and an error that falls."""
import numpy as np
import pytest
import torch

from paper_2011_12490_amd import derf, scenes, training

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("precision,tol", [("fp32", 1e-4), ("bf16", 2e-2)])
@pytest.mark.parametrize("arch", [scenes.ARCH_TINY, scenes.ARCH_SMALL, scenes.ARCH_128])
def test_one_head_a_sample_is_the_renderers_field(arch, precision, tol):
    """top_k = 1: density and colour at a renderer's samples are the renderer's,
    within the pixel tolerances of the renders' parity tests."""
    cfg = scenes.with_changes(scenes.CONFIGS["tiny"], arch=arch)
    sc = scenes.make_scene(cfg)
    t = training.HeadTrainer(sc.sites, arch, sc.weights, precision, top_k=1)
    o, d = torch.from_numpy(sc.rays_o).cuda()[:200].contiguous(), torch.from_numpy(sc.rays_d).cuda()[:200].contiguous()
    _, _, _, dbg = t.renderer().render(o, d, cfg.near, cfg.far, 32, debug=True)
    x = (o[:, None] + dbg["t"][..., None] * d[:, None]).reshape(-1, 3).contiguous()
    dirs = d[:, None].expand(-1, 32, -1).reshape(-1, 3).contiguous()
    got = t.forward(x, dirs).reshape(200, 32, 4)
    ids, _ = training.nearest_sites(x, t.sites, 1, t.beta)
    same = (ids.reshape(200, 32) == dbg["cell"])
    assert float(same.float().mean()) > 0.999  # but for samples between two sites
    want = torch.cat([dbg["sigma"][..., None], dbg["rgb"]], dim=-1)
    off = (got - want).abs()[same]
    assert float(off.max()) <= tol * max(1.0, float(want.abs().max()))


@pytest.mark.parametrize("arch", [scenes.HeadArch(6, 4, 3, 32, 1, 16), scenes.HeadArch(2, 1, 2, 24, -1, 0)])
def test_gradients_of_a_head_network(arch):
    """float32, two heads a sample, against autograd in float64 through the same
    formula.  A unit's sign may differ where its sum is within rounding of zero, so
    a gradient is compared over all of a parameter's values at once."""
    K, T = 4, 500
    rng = np.random.default_rng(3)
    t = training.HeadTrainer(rng.uniform(-1, 1, (K, 3)), arch, training.start_weights(K, arch, 5), "fp32", top_k=2)
    for b in t.bias:
        b.copy_(torch.from_numpy(rng.uniform(-0.2, 0.2, b.shape)).float())
    g = torch.Generator(device="cuda").manual_seed(7)
    x, d = torch.rand(T, 3, generator=g, device="cuda") * 2 - 1, torch.randn(T, 3, generator=g, device="cuda")
    dout = torch.randn(T, 4, generator=g, device="cuda")
    out = t.forward(x, d)
    t.backward(dout)
    ids, mix = training.nearest_sites(x, t.sites, 2, t.beta)
    W = {n: w.double().cpu().requires_grad_() for n, w in zip(t.names, t.weight)}
    B = {n: b.double().cpu().requires_grad_() for n, b in zip(t.names, t.bias)}
    gx = training.encode(x, arch.pos_freqs).double().cpu()
    gd = training.encode(d / d.norm(dim=1, keepdim=True), arch.dir_freqs).double().cpu()
    want = 0
    for j in range(2):
        k = ids[:, j].long().cpu()
        lin = lambda n, h: torch.einsum("toi,ti->to", W[n][k], h) + B[n][k]  # noqa: E731
        h = gx
        for l in range(arch.depth):
            h = torch.relu(lin("hidden%d" % l, torch.cat([gx, h], 1) if l == arch.skip_layer else h))
        view = torch.cat([h, gd], 1)
        colour = torch.relu(lin("rgb_hidden", view)) if arch.rgb_hidden else view
        row = torch.cat([torch.relu(lin("sigma", h)), torch.sigmoid(lin("rgb_out", colour))], 1)
        want = want + mix[:, j, None].double().cpu() * row
    assert float((out.cpu() - want.detach()).abs().max()) <= 1e-4
    want.backward(dout.double().cpu())
    for n, dw, db in zip(t.names, t.weight_grad, t.bias_grad):
        for got, leaf in ((dw, W[n]), (db, B[n])):
            assert float((got.cpu() - leaf.grad).norm()) <= 1e-3 * float(leaf.grad.norm()) + 1e-6, n


@pytest.mark.parametrize("precision,state_bits", [("fp32", 32), ("bf16", 32), ("bf16", 8)])
def test_the_error_falls(precision, state_bits):
    trainer, errors = training.fit(steps=200, samples=4096, precision=precision, state_bits=state_bits)
    assert np.isfinite(errors).all()
    assert errors[-10:].mean() < 0.1 * errors[:3].mean()
    if precision == "bf16":
        for w, c in zip(trainer.weight, trainer.rows_weight):
            assert torch.equal(c, w.to(torch.bfloat16))
    r = trainer.renderer()
    assert r.precision == precision and isinstance(r, derf.Renderer)
