"""Adapters whose weights, scales or products are not finite: which logits that spoils, and that it spoils no others."""
import math

import pytest
import torch

import paper_2506_22033_amd as sip
from tests.test_gpu_adapt import BF16, DEV, F32, _inputs

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("what", [math.inf, -math.inf, math.nan])
@pytest.mark.parametrize("xt,zt", [(BF16, F32), (F32, BF16)])
@pytest.mark.parametrize("B,A,r,V,D", [(9, 3, 16, 700, 64), (80, 5, 40, 1003, 72), (64, 64, 40, 70001, 64)])
def test_entries_of_up_spoil_their_own_logits(B, A, r, V, D, xt, zt, what):
    logits, hidden, down, up, which, scales = _inputs(B, A, r, V, D, xt, zt)
    clean = sip.sip_head_adapt(logits.clone(), hidden, down, up, which, scales)
    up[1, 5, 3] = up[1, V - 1, r - 1] = what
    got = sip.sip_head_adapt(logits.clone(), hidden, down, up, which, scales)
    bad = torch.zeros_like(got, dtype=torch.bool)
    bad[(which == 1)[:, None] & torch.isin(torch.arange(V, device=DEV), torch.tensor([5, V - 1], device=DEV))[None]] = True
    assert torch.equal(got[~bad], clean[~bad]) and not torch.isfinite(got[bad]).any()


@pytest.mark.parametrize("xt", [BF16, F32])
@pytest.mark.parametrize("B", [9, 80])
def test_entries_of_down_and_scales_spoil_their_adapter_s_rows(B, xt):
    logits, hidden, down, up, which, scales = _inputs(B, 4, 16, 700, 64, xt, F32)
    hidden[:], down[2, 0] = hidden.abs() + 1.0, 2.0        # (t[:, 0] of adapter 2 is 2 * 64 at least, times its scale beyond fp32)
    clean = sip.sip_head_adapt(logits.clone(), hidden, down, up, which, scales)
    down[1, 3, 7], scales[2] = math.inf, 3e38
    got = sip.sip_head_adapt(logits.clone(), hidden, down, up, which, scales)
    bad = (which == 1) | (which == 2)
    assert torch.equal(got[~bad], clean[~bad]) and got[which == 1].isnan().all() and got[which == 2].isnan().all()
