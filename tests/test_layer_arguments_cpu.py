"""Arguments of the layer operators that are no tensors are refused by name."""
import numpy as np
import pytest
import torch

import paper_2606_06510_amd as oz


@pytest.mark.parametrize("wrong", [None, 3, [[1.0]], np.zeros((6, 8), np.float32)],
                         ids=["None", "number", "list", "array"])
def test_no_tensor(wrong, monkeypatch):
    from paper_2606_06510_amd import layers
    monkeypatch.setattr(layers, "_device", lambda name, t: t.device)
    x, w, dy = torch.zeros(4, 8), torch.zeros(6, 8), torch.zeros(4, 6)
    w3, off = torch.zeros(3, 6, 8), torch.zeros(4, dtype=torch.int32)
    rows, slots = torch.zeros(8, dtype=torch.int32), torch.zeros((4, 2), dtype=torch.int32)
    order, weights = oz.ExpertOrder(off, rows, slots), torch.zeros(4, 2)
    calls = {"x": [lambda: oz.linear(wrong, w), lambda: oz.grouped_linear(wrong, w3, off),
                   lambda: oz.linear_backward(dy, wrong, w), lambda: oz.expert_gather(wrong, order),
                   lambda: oz.grouped_linear_backward(dy, wrong, w3, off)],
             "w": [lambda: oz.linear(x, wrong), lambda: oz.linear_backward(dy, x, wrong),
                   lambda: oz.grouped_linear(x, wrong, off),
                   lambda: oz.grouped_linear_backward(dy, x, wrong, off)],
             "dy": [lambda: oz.linear_backward(wrong, x, w),
                    lambda: oz.expert_combine_backward(wrong, x, order, weights)],
             "ys": [lambda: oz.expert_combine(wrong, order),
                    lambda: oz.expert_combine_backward(x, wrong, order, weights)],
             "order.slots": [lambda: oz.expert_gather(x, order._replace(slots=wrong))],
             "order.offsets": [lambda: oz.expert_gather(x, order._replace(offsets=wrong))],
             "experts": [lambda: oz.expert_sort(wrong, 4)]}
    for name, some in calls.items():
        for call in some:
            with pytest.raises(TypeError, match=f"{name}: expected a torch tensor"):
                call()
