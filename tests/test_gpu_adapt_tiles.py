"""sip_head_adapt() where a workgroup of the second product takes several tiles of the vocabulary: as many as leave the chip full, so that a call
has to be a batch of many rows under a large vocabulary.  Against the formula in 64 bits, with the tolerance of test_gpu_adapt.py."""
import math

import pytest
import torch

import paper_2506_22033_amd as sip
from tests.test_gpu_adapt import BF16, DEV, F32, _check, _inputs

pytestmark = pytest.mark.gpu


def _tiles(B, A, r, V):
    """Tiles of 128 logits that a workgroup takes: 16 up to rank 32, else 8, halved while there are fewer than 2048 workgroups."""
    batches, each = min(B, A + B // 16), 16 if r <= 32 else 8
    while each > 1 and -(-V // (128 * each)) * batches < 2048:
        each //= 2
    return each


# (tiles, B, A, r, V, D): up to 64 rows a wave finds its batch by itself; V is no whole number of tiles, nor of the eight logits of a lane
SIZES = [
    (16, 64, 64, 16, 70001, 64), (16, 200, 100, 8, 40009, 72), (16, 130, 60, 32, 70013, 64), (16, 40, 40, 24, 105003, 40),
    (8, 64, 64, 40, 70001, 64), (8, 256, 32, 64, 50257, 128), (8, 96, 33, 128, 60005, 64), (8, 48, 41, 96, 50259, 64), (8, 100, 60, 72, 40003, 136),
    (8, 64, 64, 8, 33003, 64), (4, 64, 64, 128, 16389, 64), (4, 64, 64, 32, 16389, 64), (4, 300, 20, 56, 30011, 64), (2, 64, 64, 80, 9001, 64),
    (2, 200, 50, 16, 9011, 200)]


@pytest.mark.parametrize("xt,zt", [(BF16, F32), (F32, BF16), (BF16, BF16)])
@pytest.mark.parametrize("tiles,B,A,r,V,D", SIZES)
def test_several_tiles(tiles, B, A, r, V, D, xt, zt):
    assert _tiles(B, A, r, V) == tiles
    logits, hidden, down, up, which, scales = _inputs(B, A, r, V, D, xt, zt)
    which[B // 3:B // 2] = A // 2                          # batches of more than one row, and more than one batch of an adapter
    got = logits.clone()
    sip.sip_head_adapt(got, hidden, down, up, which, scales)
    _check(got, logits, hidden, down, up, which, scales)


@pytest.mark.parametrize("zt", [F32, BF16])
@pytest.mark.parametrize("tiles,B,A,r,V,D", [(16, 64, 64, 16, 70001, 64), (8, 200, 60, 104, 40003, 64)])
def test_several_tiles_write_nothing_beside(tiles, B, A, r, V, D, zt):
    assert _tiles(B, A, r, V) == tiles
    logits, hidden, down, up, which, scales = _inputs(B, A, r, V, D, BF16, zt, pad=16)
    room = torch.full((B, V + 10), 5.0, dtype=zt, device=DEV)
    got = room[:, 5:5 + V]                                 # aligned to an element only
    got.copy_(logits)
    logits[:, ::3] = -math.inf
    got[:, ::3] = -math.inf
    sip.sip_head_adapt(got, hidden, down, up, which, scales)
    assert (got[:, ::3] == -math.inf).all() and (room[:, :5] == 5.0).all() and (room[:, 5 + V:] == 5.0).all()
    keep = torch.arange(V, device=DEV) % 3 != 0
    _check(got[:, keep], logits[:, keep], hidden, down, up[:, keep], which, scales)


def test_several_tiles_give_the_same_bits_in_a_graph():
    B, A, r, V, D = 100, 60, 72, 40003, 136
    logits, hidden, down, up, which, scales = _inputs(B, A, r, V, D, BF16, F32)
    want = sip.sip_head_adapt(logits.clone(), hidden, down, up, which, scales)
    got = logits.clone()
    ws = torch.empty(sip.sip_head_adapt_workspace_bytes(B, A, r, D), dtype=torch.uint8, device=DEV)
    side, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    sip.sip_init()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph, stream=side):
        sip.sip_head_adapt(got, hidden, down, up, which, scales, workspace=ws)
    for turn in range(3):
        got.copy_(logits)
        ws.fill_(turn * 91)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(got, want)
