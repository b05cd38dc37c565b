"""Rows of codes that lie beyond 2^32 bytes."""
import pytest
import torch

import paper_2506_22033_amd as sip

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def test_codes_whose_last_rows_begin_beyond_two_to_the_32_bytes():
    """Rows 2^15 bytes apart, 2^17 + 9 of them: the last nine begin at 2^32 and behind.  What an offset of 32 bits would read
    instead, the first rows, holds other codes."""
    V, D, stride = (1 << 17) + 9, 256, 1 << 15
    room = torch.zeros(V, stride, dtype=torch.uint8, device=DEV)
    codes = room[:, :D // 2]
    codes[-9:] = 0x99
    scales = torch.ones(V, D // 128, device=DEV)
    for B in (2, 40, 130):
        x = torch.ones(B, D, dtype=torch.bfloat16, device=DEV)
        got = sip.sip_head_logits(x, codes, scales)
        assert (got[:, -9:] == D).all() and (got[:, :-9] == -8.0 * D).all()
    # and the quantiser's writes there
    w = torch.ones(V, D, dtype=torch.bfloat16, device=DEV)
    w[-9:] = -1.0
    room.fill_(0x11)
    sip.sip_head_quantize(w, 128, codes=codes, scales=scales)
    assert (codes[:-9] == 0xFF).all() and (codes[-9:] == 0x11).all() and (room[:, D // 2:] == 0x11).all()
