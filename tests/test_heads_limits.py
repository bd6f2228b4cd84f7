"""Refusals of the training operators' Python side that need no GPU."""
import pytest
import torch

from paper_2011_12490_amd import heads


@pytest.mark.parametrize("params,grads", [([1.0], [1.0]), (["t"], [None]), ([None], ["t"]), (["t", 3], ["t", "t"]),
                                          (["t"], [2])])
def test_adamw_of_what_is_no_tensor(params, grads):
    x = torch.zeros(4)
    with pytest.raises(ValueError):
        heads.AdamW([x if p == "t" else p for p in params], [x if g == "t" else g for g in grads])
