"""Checks of the base losses' binding that need no GPU."""
import pytest
import torch

import paper_2602_05774_amd as vsd
from paper_2602_05774_amd import _lib, losses


def test_a_weight_gradient_without_a_place_is_refused():
    """A gradient that was asked for is written or refused, never left out."""
    h, w = torch.zeros(3, 64, dtype=torch.bfloat16), torch.zeros(5, 64, dtype=torch.bfloat16)
    head, rows = vsd.LmHead(h, w), _lib.VsdRows(3, 0, 5, _lib.VSD_BF16, 64)
    buf = vsd.LmHeadGrad(torch.empty_like(h), None, None)
    for kind in (True, torch.float32, torch.bfloat16):
        with pytest.raises(ValueError, match="weight_grad"):
            losses._gradient(head, rows, h.device, buf, kind)
    assert losses._gradient(head, rows, h.device, buf, False)[0] is buf
    full = vsd.LmHeadGrad(torch.empty_like(h), None, torch.empty_like(w))
    assert losses._gradient(head, rows, h.device, full, True)[0] is full
    made = losses._gradient(head, rows, h.device, True, torch.bfloat16)[0]
    assert made.grad_weight.dtype == torch.bfloat16 and made.grad_weight.shape == w.shape
