"""What the trainers refuse before any GPU work."""
import numpy as np
import pytest

from paper_2011_12490_amd import scenes, training


def test_refusals():
    for kw in (dict(precision="fp16"), dict(top_k=0), dict(top_k=4), dict(images=0), dict(width=0), dict(depth=0), dict(code_dim=0)):
        with pytest.raises(ValueError):
            training.GatedTrainer(np.zeros((3, 3)), **{"images": 2, "device": "cpu", **kw})
    with pytest.raises(ValueError):
        training.HeadTrainer(np.zeros((3, 3)), scenes.ARCH_TINY, training.start_weights(3, scenes.ARCH_TINY, 0), optimizer="sgd",
                             device="cpu")
