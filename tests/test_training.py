"""The trainer's own pieces that need no GPU: the encoding, the sites' weights, the
start weights' layout, and what it refuses."""
import numpy as np
import pytest
import torch

import oracle
from paper_2011_12490_amd import scenes, training


@pytest.mark.parametrize("freqs", [0, 1, 6, 10])
def test_encoding_is_the_heads_encoding(freqs):
    """float32 sines of arguments up to pi 2^9: off by 2^-24 of the argument."""
    p = np.random.default_rng(1).uniform(-1, 1, (50, 3)).astype(np.float32)
    got = training.encode(torch.from_numpy(p), freqs).numpy()
    want = np.stack([oracle.posenc(freqs, q) for q in p])
    assert got.shape == want.shape == (50, 3 + 6 * freqs)
    assert np.abs(got - want).max() <= 2 * np.pi * 2.0 ** max(freqs - 1, 0) * 2.0 ** -23 + 1e-6


def test_nearest_sites():
    sites = torch.tensor([[0.0, 0, 0], [1, 0, 0], [0, 3, 0]])
    ids, w = training.nearest_sites(torch.tensor([[0.9, 0, 0], [0.0, 2.0, 0]]), sites, 2, 10.0)
    assert ids.tolist() == [[1, 0], [2, 0]] and ids.dtype == torch.int32
    assert torch.allclose(w.sum(1), torch.ones(2))
    assert float(w[0, 1] / w[0, 0]) == pytest.approx(np.exp(-10 * 0.8), rel=1e-4)


def test_start_weights_have_the_packed_size():
    for arch in (scenes.ARCH_TINY, scenes.ARCH_128):
        w = training.start_weights(3, arch, 0)
        assert w.shape == (3, arch.weights_count()) and w.dtype == np.float32


def test_trainer_refusals():
    w = training.start_weights(3, scenes.ARCH_TINY, 0)
    for kw in (dict(precision="fp16"), dict(top_k=0), dict(top_k=4)):
        with pytest.raises(ValueError):
            training.HeadTrainer(np.zeros((3, 3)), scenes.ARCH_TINY, w, device="cpu", **kw)


def test_renderer_is_made_on_the_trainers_device(monkeypatch):
    """derf.Renderer binds to the current device, which need not be the trainer's."""
    current, seen = ["another"], []

    class Device:
        def __init__(self, device):
            self.device = device

        def __enter__(self):
            self.before, current[0] = current[0], self.device

        def __exit__(self, *_):
            current[0] = self.before

    monkeypatch.setattr(torch.cuda, "device", Device)
    monkeypatch.setattr(training.derf, "Renderer", lambda *args: seen.append((current[0],) + args[3:]))
    t = object.__new__(training.HeadTrainer)
    t.device, t.host_sites, t.arch, t.precision = torch.device("cuda:1"), None, None, "fp32"
    t.packed = lambda: None
    t.renderer()
    assert seen == [(torch.device("cuda:1"), "fp32")] and current == ["another"]
