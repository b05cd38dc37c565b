"""The ends of what beams, reordering and adapters are documented to take: many equal logits, more rows than one grid dimension has lanes
for, states that are not finite."""
import pytest
import torch

import paper_2506_22033_amd as sip
from tests.test_gpu_beam import _check, _rows

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
F32, BF16 = torch.float32, torch.bfloat16


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("low", [1.0, -1e9, torch.finfo(BF16).min, 0.0])
@pytest.mark.parametrize("share", [1.0, 0.12, 0.07])
@pytest.mark.parametrize("n", [1, 5, 128])
def test_equal_logits_by_the_lower_token(dtype, low, share, n):
    # Of every row a share is `low` (zeros of both signs), three lie above and the rest is no continuation.
    g = torch.Generator().manual_seed(7)
    V = 50003
    z = torch.full((2, V), -float("inf"))
    z[torch.rand(2, V, generator=g) < share] = low
    if low == 0.0:
        z[(torch.rand(2, V, generator=g) < 0.5) & (z == 0)] = -0.0
    top = torch.randperm(V, generator=g)[:3]
    z[:, top] = torch.tensor([3.0, 4.0, 4.0])
    logits = torch.empty(2, V + 5, dtype=dtype, device=DEV)[:, :V]       # (rows start at multiples of 16 bytes)
    logits.copy_(z)
    tokens, parents, _ = sip.sip_beam_select(logits, torch.tensor([0.0, -1.0]).to(DEV), 1, n)
    assert parents.cpu().tolist() == [[0] * n] * 2
    want = torch.sort(z.to(dtype).float() + 0.0, dim=1, descending=True, stable=True).indices[:, :n]
    assert torch.equal(tokens.cpu().long(), want)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("groups,width,V,n", [(2, 64, 1481, 128), (1, 64, 70000, 128), (3, 20, 1116, 40), (2, 54, 1575, 54), (1, 9, 700, 60),
                                              (2, 2, 115984, 2), (1, 30, 9000, 31), (1, 16, 1023, 64), (1, 64, 33, 128), (2, 31, 2100, 100)])
def test_wide_groups_of_few_lists_and_short_chunks(groups, width, V, n, dtype):
    logits, g = _rows(groups * width, V, dtype, V * n)
    scores = -torch.rand(groups * width, generator=g, device=DEV) * 0.5
    _check(logits, scores, width, n, sip.sip_beam_select(logits, scores, width, n))


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("finished", [False, True])
@pytest.mark.parametrize("live", [1, 3, 60])
@pytest.mark.parametrize("width,V,n", [(60, 88820, 120), (64, 150000, 128), (30, 3000, 1), (64, 524288, 2), (30, 170000, 33), (60, 20000, 7)])
def test_many_lists_of_which_few_hold_anything(width, V, n, live, finished, dtype):
    # As before the first step of a search, or near its end.
    logits, g = _rows(width, V, dtype, V + n)
    scores = -torch.rand(width, generator=g, device=DEV) * 9.0
    done = None
    if finished:
        done = torch.ones(width, dtype=torch.uint8, device=DEV)
        done[:live] = 0
    else:
        scores[live:] = -float("inf")
    _check(logits, scores, width, n, sip.sip_beam_select(logits, scores, width, n, finished=done, end_token=2), done, end_token=2)


@pytest.mark.parametrize("width,V,n", [(64, 9000, 128), (64, 40000, 100), (8, 3000, 16), (64, 100, 3), (1, 50000, 128)])
def test_equal_rows_of_equal_logits_by_beam_and_token(width, V, n):
    # Every continuation of every beam has the same total: the first beam's lowest tokens, then the next one's.
    logits = torch.zeros(width, (V + 7) // 8 * 8, device=DEV)[:, :V]
    tokens, parents, _ = sip.sip_beam_select(logits, torch.zeros(width, device=DEV), width, n)
    want = torch.arange(n)
    assert torch.equal(parents[0].cpu().long(), want // V) and torch.equal(tokens[0].cpu().long(), want % V)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("scale,at", [(1e-3, 1.0), (1e-3, -1.0), (0.05, -300.0), (1.0, 0.0)])
def test_many_logits_near_one_another(dtype, scale, at):
    # More than a chunk's list holds reach the bound: few distinct values, above and below 0.
    logits, g = _rows(12, 20000, F32, 5)
    logits = torch.round(logits.clamp(-2, 2) * 2) / 2 * scale + at
    room = torch.empty(12, 20000, dtype=dtype, device=DEV)
    room.copy_(logits)
    scores = -torch.arange(12, device=DEV).float() * 0.25
    _check(room, scores, 4, 100, sip.sip_beam_select(room, scores, 4, 100))


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("low", [-1e30, -1e10, 1e10, 1e35, 3e6, -2e5, 777.0])
def test_rows_of_large_values(low, dtype):
    # Equal logits: the total is -ln V beside the score, whatever they are.  Three of a row are lower by a quarter of it.
    V = 20000
    logits = torch.full((2, V), low, device=DEV).to(dtype)
    logits[1, 5:8] = torch.tensor(low - abs(low) / 4, device=DEV).to(dtype)
    scores = torch.tensor([-0.5, 0.0], device=DEV)
    _check(logits, scores, 2, 9, sip.sip_beam_select(logits, scores, 2, 9))


def test_reorder_of_more_work_than_lanes_along_a_grid():
    # Most rows have no slot; the histories are so long that each of 127000 rows has 136 workgroups of 256 lanes: over 2^32 in all.
    slots, L_max, rows = 4, 1 << 17, 127000
    state = torch.zeros(sip.sip_state_bytes(slots, L_max), dtype=torch.uint8, device=DEV)
    sip.sip_state_init(state, slots, L_max)
    history = torch.arange(100, dtype=torch.int32, device=DEV)
    sip.sip_state_assign(state, slots, L_max, torch.tensor([0], dtype=torch.int32, device=DEV),
                         torch.tensor([0, 100], device=DEV), history)
    slot_of_row = torch.full((rows,), -1, dtype=torch.int32, device=DEV)
    slot_of_row[-2:] = torch.tensor([0, 3], dtype=torch.int32, device=DEV)
    parents = torch.ones(rows, dtype=torch.int32, device=DEV)
    parents[0::2] = 0
    parents[-1] = 0
    tokens = torch.full((rows,), 7, dtype=torch.int32, device=DEV)
    sip.sip_state_reorder(state, slots, L_max, slot_of_row, parents, 2, tokens)
    _, overflow, length, kept = sip.state_views(state, slots, L_max)
    assert int(overflow) == 0 and length.tolist() == [101, 0, 0, 101]
    for slot in (0, 3):
        assert kept[slot, :101].tolist() == list(range(100)) + [7]


@pytest.mark.parametrize("xt", [F32, BF16])
@pytest.mark.parametrize("rows", [3, 80])
def test_adapters_of_states_that_are_not_finite(xt, rows):
    g = torch.Generator(device=DEV).manual_seed(2)
    D, V, rank = 256, 700, 16
    hidden = torch.randn(rows, D, generator=g, device=DEV).to(xt)
    down = torch.randn(2, rank, D, generator=g, device=DEV).to(BF16)
    up = torch.randn(2, V, rank, generator=g, device=DEV).to(BF16)
    which = torch.zeros(rows, dtype=torch.int32, device=DEV)
    which[2] = 5
    logits = torch.randn(rows, V, generator=g, device=DEV)
    want = sip.sip_head_adapt(logits.clone(), hidden, down, up, which)
    hidden[0, 3], hidden[1, 200], hidden[2] = float("inf"), float("nan"), float("nan")
    got = sip.sip_head_adapt(logits.clone(), hidden, down, up, which)
    assert got[:2].isnan().all()
    assert torch.equal(got[2:], want[2:]) and torch.equal(got[2], logits[2])
    masked = logits.clone()
    masked[:, ::3] = -float("inf")
    got = sip.sip_head_adapt(masked.clone(), hidden, down, up, which)
    assert (got[2:, ::3] == -float("inf")).all() and torch.equal(got[2:, 1::3], want[2:, 1::3])
