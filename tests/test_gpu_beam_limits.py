"""What the beams' selection asks of a call, and says of totals that fp32 does not hold."""
import pytest
import torch

import paper_2506_22033_amd as sip

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
INF = float("inf")


def test_finished_beams_need_an_end_token():
    logits, scores = torch.zeros(4, 64, device=DEV), torch.zeros(4, device=DEV)
    done = torch.tensor([0, 1, 1, 0], dtype=torch.bool, device=DEV)
    with pytest.raises(TypeError, match="end_token"):
        sip.sip_beam_select(logits, scores, 2, finished=done)
    tokens, parents, _ = sip.sip_beam_select(logits, scores, 2, finished=done, end_token=0)
    assert tokens.tolist() == [[0, 0], [0, 0]] and parents.tolist() == [[1, 0], [0, 1]]
    assert sip.sip_beam_select(logits, scores, 2)[0].tolist() == [[0, 1], [0, 1]]          # (nothing finished: none is needed)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("scale", [1e-30, 1e30])
def test_the_ends_of_logit_scale(scale, dtype):
    # At 1e30 each logit but the largest has no probability, at 1e-30 all have the same.  Rounding of the total, and lse's 3e-6.
    V, scale32 = 500, float(torch.tensor(scale))
    logits = torch.empty(1, 504, dtype=dtype, device=DEV)[:, :V]
    logits.copy_(torch.randperm(V, generator=torch.Generator().manual_seed(1)).float()[None] / 4 - 30.0)      # (exact in 16 bits)
    tokens, parents, out = sip.sip_beam_select(logits, torch.tensor([-1.5], device=DEV), 1, 4, logit_scale=scale)
    z = logits[0].double().cpu()
    order = torch.sort(z, descending=True, stable=True).indices[:4]
    total = -1.5 + torch.log_softmax(z * scale32, 0)[order]
    assert tokens[0].cpu().tolist() == order.tolist() and (parents == 0).all()
    assert ((out[0].cpu().double() - total).abs() <= 3e-6 + 2.0 ** -24 * total.abs()).all()


def test_totals_below_the_range_of_fp32():
    # Masks of the lowest value, and a temperature below 1: continuations still, of a score that fp32 has no number for.
    logits = torch.full((1, 8), torch.finfo(torch.float32).min, device=DEV)
    logits[0, 5] = 0.0
    tokens, parents, out = sip.sip_beam_select(logits, torch.zeros(1, device=DEV), 1, 4, logit_scale=2.0)
    assert tokens.tolist() == [[5, 0, 1, 2]] and parents.tolist() == [[0] * 4] and out.tolist() == [[0.0, -INF, -INF, -INF]]
