"""Clipping where nothing is left to divide by."""
import pytest
import torch

import paper_2506_22033_amd as sip

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_gradients_of_zero_stay_zero(dtype):
    """max_norm / (norm + eps) is 0 / 0: there is nothing to scale."""
    for max_norm in (0.0, 1.0, float("inf")):
        for eps in (0.0, 1e-6):
            g, o = torch.zeros(70001, dtype=dtype, device=DEV), torch.full((70001,), 7.0, dtype=dtype, device=DEV)
            norm = sip.sip_grad_clip(sip.GradTable([g], [o]), max_norm, eps=eps)
            assert float(norm) == 0.0 and not o.any(), (max_norm, eps)
            sip.sip_grad_clip([g], max_norm, eps=eps)
            assert not g.any()


def test_a_bound_of_zero_leaves_zeros():
    for dtype in (torch.float32, torch.bfloat16):
        for x in (1.0, 1e-38):
            g = torch.full((5000,), x, dtype=dtype, device=DEV)
            sip.sip_grad_clip([g], 0.0, eps=0.0)
            assert not g.any()
