"""The tables of multiplicities behind sip_state_reorder(): in each of its three forms (a workgroup a group; several, for up to eight beams; for
more) a slot's table counts exactly what its history holds, unless its parent's was given up or its own new token is one too many."""
import numpy as np
import pytest
import torch

import paper_2506_22033_amd as sip
from tests.test_gpu_reorder import _expected, _read, _state

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
MOST = 3072                                               # distinct tokens of a table
# (groups, width, L_max): width * (L_max + 8192) up to 49152 is one workgroup's work, more several's
FORMS = [(5, 4, 300), (3, 5, 1500), (3, 8, 300), (2, 6, 4100), (7, 8, 1027), (2, 9, 300), (2, 16, 2050), (1, 64, 700), (3, 33, 61)]


def _on(x):
    return None if x is None else torch.tensor(np.asarray(x), dtype=torch.int32, device=DEV)


def _counts(history):
    want = {}
    for t in history:
        if t >= 0:
            want[t] = want.get(t, 0) + 1
    return want


def _check_tables(got, histories, given_up=()):
    """Every slot's length, tokens and table; -1 distinct tokens in `given_up` and nowhere else."""
    _, _, length, tokens, distinct, keys, counts = got
    for s, history in enumerate(histories):
        assert length[s] == len(history) and tokens[s, :len(history)].tolist() == list(history), s
        if s in given_up:
            assert distinct[s] == -1, s
            continue
        want, live = _counts(history), keys[s] >= 0
        assert distinct[s] == len(want), s
        assert dict(zip(keys[s][live].tolist(), counts[s][live].tolist())) == want, s


def _step(state, slots, L_max, histories, given_up, slot_of_row, parents, width, new):
    """One call, and what holds behind it: (histories, slots whose table is given up)."""
    moved, over = _expected(histories, slot_of_row, parents, width, new, L_max)
    before = _read(state, slots, L_max)
    sip.sip_state_reorder(state, slots, L_max, _on(slot_of_row), _on(parents), width, _on(new))
    got = _read(state, slots, L_max)
    after = [moved.get(s, histories[s]) for s in range(slots)]
    gone = set()
    for s in range(slots):
        if s not in moved:
            of = s
        else:
            r = slot_of_row.index(s)
            of = slot_of_row[r // width * width + parents[r]]
        if of in given_up or len(_counts(after[s])) > MOST:
            gone.add(s)
    _check_tables(got, after, gone)
    assert got[0] == before[0] and got[1] == before[1] + over
    return after, gone


@pytest.mark.parametrize("groups,width,L_max", FORMS)
@pytest.mark.parametrize("seed", range(2))
def test_steps_of_a_search(groups, width, L_max, seed):
    rng = np.random.default_rng(seed + width)
    slots = groups * width + 3
    histories = [rng.integers(0, 400, n).tolist() for n in rng.integers(0, L_max + 1, slots)]
    histories[0], histories[-1] = [], rng.integers(0, 1 << 19, L_max).tolist()
    state, gone = _state(slots, L_max, histories), set()
    gone = {s for s, h in enumerate(histories) if len(_counts(h)) > MOST}
    _check_tables(_read(state, slots, L_max), histories, gone)
    for step in range(3):
        slot_of_row = rng.permutation(slots)[:groups * width].tolist()
        parents = rng.integers(0, width, groups * width).tolist()
        new = rng.integers(-40, 400, groups * width).tolist() if step != 1 else None
        if step == 2:                                     # some rows stay, some slots are none
            parents[0], parents[-1] = -1, width
            slot_of_row[groups * width // 2] = slots
        histories, gone = _step(state, slots, L_max, histories, gone, slot_of_row, parents, width, new)


@pytest.mark.parametrize("width,L_max", [(3, 4096), (6, 4096), (12, 4096), (40, 3500)])
def test_given_up_tables(width, L_max):
    # Before the call, by the new token, and one that is full but holds the new token.
    rng = np.random.default_rng(width)
    slots = width + 1
    histories = [rng.integers(0, 9, 30).tolist() for _ in range(slots)]
    histories[0], histories[1] = list(range(MOST)), list(range(MOST + 200))
    state = _state(slots, L_max, histories)
    gone = {1}
    _check_tables(_read(state, slots, L_max), histories, gone)
    slot_of_row = list(range(width))
    parents = [0, 2, 1] + [0] * (width - 3)
    new = [7, 5, 3] + [100000 + k for k in range(width - 3)]
    histories, gone = _step(state, slots, L_max, histories, gone, slot_of_row, parents, width, new)
    assert gone == {2} | set(range(3, width))
    parents = [1] * width                                 # all from a short one: every table is there again
    histories, gone = _step(state, slots, L_max, histories, gone, slot_of_row, parents, width, [11] * width)
    assert not gone


@pytest.mark.parametrize("groups,width", [(2, 4), (2, 8), (1, 20)])
def test_penalties_see_the_reordered_tables(groups, width):
    V, L = 20000, 300
    rng = np.random.default_rng(3)
    slots = groups * width
    histories = [rng.integers(0, 300, 200).tolist() for _ in range(slots)]
    state = _state(slots, L, histories)
    histories, gone = _step(state, slots, L, histories, set(), rng.permutation(slots).tolist(),
                            rng.integers(0, width, slots).tolist(), width, rng.integers(0, 300, slots).tolist())
    assert not gone
    fresh = _state(slots, L, histories)
    g = torch.Generator(device=DEV).manual_seed(1)
    logits = torch.randn(slots, V, generator=g, device=DEV)
    logits[:, :300] += 3.0
    params = {"repetition_penalty": torch.full((slots,), 1.3, device=DEV), "frequency_penalty": torch.full((slots,), 0.4, device=DEV)}
    rows = torch.arange(slots, dtype=torch.int32, device=DEV)
    for step in range(3):
        a = sip.sip_sample_state(logits, params, state, slots, L, rows, 7, step, 3)
        b = sip.sip_sample_state(logits, params, fresh, slots, L, rows, 7, step, 3)
        assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])
        assert (a[2] - b[2]).abs().max() < 1e-5
    _check_tables(_read(state, slots, L), [_read(state, slots, L)[3][s, :_read(state, slots, L)[2][s]].tolist() for s in range(slots)])
