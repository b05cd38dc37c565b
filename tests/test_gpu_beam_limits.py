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
