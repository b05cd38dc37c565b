"""sip_state_reorder(): every row's slot holds its parent's history and the new token behind it, as a state that was assigned those
histories would."""
import numpy as np
import pytest
import torch

import paper_2506_22033_amd as sip

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def _state(slots, L_max, histories):
    """A state whose slot i holds histories[i] (a list of ints)."""
    state = torch.zeros(sip.sip_state_bytes(slots, L_max), dtype=torch.uint8, device=DEV)
    sip.sip_state_init(state, slots, L_max)
    indptr = torch.tensor(np.cumsum([0] + [len(h) for h in histories]), dtype=torch.int64, device=DEV)
    flat = [t for h in histories for t in h] or [0]
    sip.sip_state_assign(state, slots, L_max, torch.arange(len(histories), dtype=torch.int32, device=DEV), indptr,
                         torch.tensor(flat, dtype=torch.int32, device=DEV))
    return state


def _read(state, slots, L_max):
    tick, overflow, length, tokens = (x.cpu() for x in sip.state_views(state, slots, L_max))
    distinct, keys, counts = (x.cpu() for x in sip.state_table_views(state, slots, L_max))
    return int(tick), int(overflow), length, tokens, distinct, keys, counts


def _check_slot(got, slot, history):
    _, _, length, tokens, distinct, keys, counts = got
    assert length[slot] == len(history)
    assert tokens[slot, :len(history)].tolist() == list(history)
    want = {}
    for t in history:
        if t >= 0:
            want[t] = want.get(t, 0) + 1
    if len(want) > 3072:
        assert distinct[slot] == -1
        return
    if distinct[slot] == -1:
        return
    live = keys[slot] >= 0
    assert distinct[slot] == len(want)
    assert dict(zip(keys[slot][live].tolist(), counts[slot][live].tolist())) == want


def _expected(histories, slot_of_row, parents, width, new, L_max):
    out = {}
    over = 0
    slots = len(histories)
    for r, to in enumerate(slot_of_row):
        first = r // width * width
        if not 0 <= parents[r] < width or not 0 <= to < slots or to in slot_of_row[first:r]:
            continue
        of = slot_of_row[first + parents[r]]
        h = list(histories[of]) if 0 <= of < slots else []
        if new is not None and new[r] >= 0:
            if len(h) < L_max:
                h.append(new[r])
            else:
                over += 1
        out[to] = h
    return out, over


def _run(width, groups, L_max, seed, slots=None, lengths=None, new=True, vocabulary=500, parents=None, slot_of_row=None):
    rng = np.random.default_rng(seed)
    slots = slots or groups * width + 2
    lengths = rng.integers(0, L_max + 1, slots) if lengths is None else lengths
    histories = [rng.integers(0, vocabulary, n).tolist() for n in lengths]
    state = _state(slots, L_max, histories)
    before = _read(state, slots, L_max)
    rows = groups * width
    slot_of_row = rng.permutation(slots)[:rows].tolist() if slot_of_row is None else slot_of_row
    parents = rng.integers(0, width, rows).tolist() if parents is None else parents
    tokens = rng.integers(0, vocabulary, rows).tolist() if new is True else new
    on = lambda x: None if x is None else torch.tensor(x, dtype=torch.int32, device=DEV)        # noqa: E731
    sip.sip_state_reorder(state, slots, L_max, on(slot_of_row), on(parents), width, on(tokens))
    after = _read(state, slots, L_max)
    want, over = _expected(histories, slot_of_row, parents, width, tokens, L_max)
    for s in range(slots):
        _check_slot(after, s, want.get(s, histories[s]))
        n = len(want.get(s, histories[s]))
        assert torch.equal(after[3][s, n:], before[3][s, n:]), "behind the history"
    assert after[0] == before[0] and after[1] == before[1] + over
    return state, histories, after


@pytest.mark.parametrize("width,groups,L_max", [
    (1, 1, 1), (1, 5, 8), (2, 1, 3), (4, 1, 512), (3, 7, 61), (8, 4, 1024), (8, 3, 1026), (9, 2, 4099), (32, 2, 130), (33, 1, 257),
    (64, 2, 1023), (5, 60, 33)])
def test_reorder(width, groups, L_max):
    for seed in range(3):
        _run(width, groups, L_max, seed)


def test_without_tokens_and_with_negative_ones():
    _run(4, 3, 100, 1, new=None)
    _run(4, 1, 100, 2, new=[-1, 5, -7, 6])


def test_full_slots_overflow():
    _run(4, 2, 20, 3, lengths=np.full(10, 20))
    _run(4, 2, 20, 4, lengths=np.full(10, 19))


def test_swaps_and_cycles():
    _run(4, 1, 700, 5, parents=[1, 0, 3, 2])
    _run(4, 1, 700, 6, parents=[1, 2, 3, 0])
    _run(4, 1, 700, 7, parents=[0, 1, 2, 3])
    _run(4, 1, 700, 8, parents=[2, 2, 2, 2])


def test_rows_that_stay():
    """Parents outside the group, slots outside the state, a slot named twice."""
    _run(4, 2, 50, 9, parents=[-1, 0, 4, 1, 2, 2, -2147483648, 2147483647])
    _run(4, 2, 50, 10, slots=9, slot_of_row=[0, -1, 9, 3, 4, 5, 2147483647, 6], parents=[1, 0, 0, 2, 2, 0, 1, 3])
    _run(4, 1, 50, 11, slots=6, slot_of_row=[2, 5, 2, 5], parents=[1, 0, 3, 3])


def test_given_up_tables():
    """A history of more distinct tokens than its table holds, before and by the new token."""
    rng = np.random.default_rng(12)
    histories = [list(range(3072)), list(range(4000)), [1, 2, 2], rng.integers(0, 9, 30).tolist()]
    state = _state(4, 4096, histories)
    on = lambda x: torch.tensor(x, dtype=torch.int32, device=DEV)        # noqa: E731
    sip.sip_state_reorder(state, 4, 4096, on([0, 1, 2, 3]), on([0, 3, 1, 0]), 4, on([5000, 2, 9, 7]))
    got = _read(state, 4, 4096)
    for s, h in enumerate((histories[0] + [5000], histories[3] + [2], histories[1] + [9], histories[0] + [7])):
        _check_slot(got, s, h)
    assert got[4].tolist()[0] == -1 and got[4].tolist()[2] == -1 and got[4].tolist()[3] == 3072


def test_sampling_goes_on_as_from_an_assigned_state():
    """Penalties see the reordered histories."""
    V, L = 20000, 300
    state, histories, after = _run(4, 3, L, 13, lengths=np.full(14, 200), vocabulary=300)
    length, tokens = after[2], after[3]
    fresh = _state(14, L, [tokens[s, :length[s]].tolist() for s in range(14)])
    g = torch.Generator(device=DEV).manual_seed(1)
    logits = torch.randn(14, V, generator=g, device=DEV)
    logits[:, :300] += 3.0
    params = {"repetition_penalty": torch.full((14,), 1.3, device=DEV), "frequency_penalty": torch.full((14,), 0.4, device=DEV)}
    rows = torch.arange(14, dtype=torch.int32, device=DEV)
    for step in range(3):
        a = sip.sip_sample_state(logits, params, state, 14, L, rows, 7, step, 3)
        b = sip.sip_sample_state(logits, params, fresh, 14, L, rows, 7, step, 3)
        assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])
        assert (a[2] - b[2]).abs().max() < 1e-5


def test_in_a_graph_and_on_another_stream():
    width, groups, L = 8, 3, 400
    rng = np.random.default_rng(14)
    slots = width * groups
    histories = [rng.integers(0, 99, rng.integers(0, 300)).tolist() for _ in range(slots)]
    on = lambda x: torch.tensor(np.asarray(x), dtype=torch.int32, device=DEV)        # noqa: E731
    rows, parents = on(rng.permutation(slots)), on(rng.integers(0, width, slots))
    new = on(rng.integers(0, 99, slots))
    one, two = _state(slots, L, histories), _state(slots, L, histories)
    side, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    sip.sip_init()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph, stream=side):
        sip.sip_state_reorder(two, slots, L, rows, parents, width, new)
    for _ in range(5):
        sip.sip_state_reorder(one, slots, L, rows, parents, width, new)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(one, two)
    with torch.cuda.stream(side):
        sip.sip_state_reorder(two, slots, L, rows, parents, width, new)
    sip.sip_state_reorder(one, slots, L, rows, parents, width, new, stream=side)
    side.synchronize()
    assert torch.equal(one, two)


def test_refusals():
    state = torch.zeros(sip.sip_state_bytes(8, 16), dtype=torch.uint8, device=DEV)
    r = torch.zeros(8, dtype=torch.int32, device=DEV)
    for bad in (lambda: sip.sip_state_reorder(state, 8, 16, r, r, 3), lambda: sip.sip_state_reorder(state, 8, 16, r, r[:4], 4),
                lambda: sip.sip_state_reorder(state, 8, 16, r.long(), r, 4), lambda: sip.sip_state_reorder(state, 8, 16, r, r, 4, r[:2]),
                lambda: sip.sip_state_reorder(state.cpu(), 8, 16, r, r, 4)):
        with pytest.raises(TypeError):
            bad()
    for bad in (lambda: sip.sip_state_reorder(state, 9, 16, r, r, 4), lambda: sip.sip_state_reorder(state, 0, 16, r, r, 4),
                lambda: sip.sip_state_reorder(state[1:], 8, 16, r, r, 4)):
        with pytest.raises(sip.SipError):
            bad()
