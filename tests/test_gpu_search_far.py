"""Reordering, lookup, gradient and adapters at the largest sizes that the headers name, where offsets pass 32 bits."""
import numpy as np
import pytest
import torch

import paper_2506_22033_amd as sip
from tests.test_gpu_adapt import _check as _check_adapted
from tests.test_gpu_adapt import _inputs
from tests.test_gpu_embed import BF16, DEV, F32, _check_gradient, _gen
from tests.test_gpu_reorder import _check_slot

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("width", [3, 8, 20])
def test_histories_beyond_32_bits(width):
    # Slots whose token rows begin past 2^31 words, and their tables with them; others of the same groups at the beginning.
    slots, L = 16500, 1 << 17
    assert (slots - 100) * L > 1 << 31
    state = torch.empty(sip.sip_state_bytes(slots, L), dtype=torch.uint8, device=DEV)
    sip.sip_state_init(state, slots, L)
    rng = np.random.default_rng(width)
    used = np.concatenate([rng.permutation(50)[:width], slots - 1 - rng.permutation(50)[:width]])
    histories = {int(s): rng.integers(0, 900, rng.integers(1, 3000)).tolist() for s in used}
    histories[int(used[-1])] = rng.integers(0, 900, L - 1).tolist()      # a long one, to its last token but one
    on = lambda x: torch.tensor(np.asarray(x), dtype=torch.int32, device=DEV)        # noqa: E731
    indptr = torch.tensor(np.cumsum([0] + [len(histories[int(s)]) for s in used]), dtype=torch.int64, device=DEV)
    sip.sip_state_assign(state, slots, L, on(used), indptr, on([t for s in used for t in histories[int(s)]]))
    rows = rng.permutation(used)                          # (two groups, of slots from both ends)
    parents = rng.integers(0, width, 2 * width)
    k = list(rows).index(used[-1])
    parents[k], parents[k // width * width + (k + 1) % width] = k % width, k % width
    new = rng.integers(0, 900, 2 * width)
    sip.sip_state_reorder(state, slots, L, on(rows), on(parents), width, on(new))
    tick, overflow, length, tokens = sip.state_views(state, slots, L)
    distinct, keys, counts = sip.state_table_views(state, slots, L)
    assert int(overflow) == 0 and int((length > 0).sum()) == 2 * width
    for r, s in enumerate(rows):
        want = histories[int(rows[r // width * width + parents[r]])] + [int(new[r])]
        assert distinct[s] == len(set(want))
        _check_slot((0, 0, {0: length[s].cpu()}, tokens[s:s + 1].cpu(), {0: distinct[s].cpu()}, {0: keys[s].cpu()}, {0: counts[s].cpu()}), 0, want)


def test_the_largest_lookup():
    N, D, V = 1 << 20, 16384, 9                           # 2^31 units of eight entries
    w = torch.randn(V, D, generator=_gen(1), device=DEV).to(BF16)
    ids = (torch.arange(N, device=DEV) % (V + 1)).to(torch.int32)        # (every tenth is none)
    out = torch.full((N, D), 7.0, dtype=BF16, device=DEV)
    sip.sip_embed(w, ids, out=out)
    rows = torch.cat((w, torch.zeros(1, D, dtype=BF16, device=DEV)))
    for i in range(0, N, 1 << 16):
        assert torch.equal(out[i:i + (1 << 16)], rows[ids[i:i + (1 << 16)].long()])


def test_the_largest_matrix_of_a_gradient():
    V, D = sip.SIP_MAX_V, sip.SIP_MAX_D                   # 2^31 units of 16 bytes
    g = _gen(2)
    gw = torch.full((V, D), 7.0, device=DEV)
    ids = torch.cat((torch.randint(0, V, (90,), generator=g, device=DEV), torch.tensor([V - 1, V - 1, 0, V, -1], device=DEV))).to(torch.int32)
    grad = torch.randn(ids.numel(), D, generator=g, device=DEV)
    sip.sip_embed_backward(grad, ids, V, grad_weight=gw)
    rows, at = torch.unique(ids[(ids >= 0) & (ids < V)].long(), return_inverse=True)
    _check_gradient(gw[rows], grad[(ids >= 0) & (ids < V)], at.to(torch.int32), rows.numel(), 1.0)
    gw[rows] = 0.0
    assert not any(gw[i:i + (1 << 14)].any() for i in range(0, V, 1 << 14))
    sip.sip_embed_backward(grad, ids, V, grad_weight=gw, accumulate=True)
    _check_gradient(gw[rows], grad[(ids >= 0) & (ids < V)], at.to(torch.int32), rows.numel(), 1.0)


@pytest.mark.parametrize("accumulate", [False, True])
def test_gradient_rows_beyond_32_bits(accumulate):
    # A stride that puts row 40000 past 2^32 elements; the most tokens and the widest rows in one call.
    N, D, V, stride = sip.SIP_MAX_TOKENS, sip.SIP_MAX_D, 40, 110000
    g = _gen(3)
    grad = torch.empty(N * stride, dtype=BF16, device=DEV).as_strided((N, D), (stride, 1))
    for i in range(0, N, 1 << 12):
        grad[i:i + (1 << 12)] = torch.randn(min(1 << 12, N - i), D, generator=g, device=DEV).to(BF16)
    ids = torch.randint(-3, V + 2, (N,), generator=g, device=DEV, dtype=torch.int32)
    start = torch.randn(V, D, generator=g, device=DEV)
    gw = start.clone()
    sip.sip_embed_backward(grad, ids, V, grad_weight=gw, accumulate=accumulate)
    for c in range(0, D, 2048):                           # (64 bits of all columns are large)
        _check_gradient(gw[:, c:c + 2048].contiguous(), grad[:, c:c + 2048], ids, V, 1.0,
                        start[:, c:c + 2048].contiguous() if accumulate else None)


@pytest.mark.parametrize("B,A,r,V,D", [(65536, 4096, 8, 40, 16), (64, 4096, 8, 40, 16), (65, 4096, 16, 1000, 16), (2000, 1, 16, 5000, 64)])
def test_the_most_rows_and_adapters(B, A, r, V, D):
    logits, hidden, down, up, which, scales = _inputs(B, A, r, V, D, BF16, F32)
    got = logits.clone()
    sip.sip_head_adapt(got, hidden, down, up, which, scales)
    some = torch.arange(0, B, max(1, B // 300), device=DEV)
    _check_adapted(got[some], logits[some], hidden[some], down, up, which[some], scales)
    ok = which >= 0
    a = which.long().clamp(min=0)
    for i in range(0, B, 4096):                           # (a row or adapter that is another's is off by 1)
        at = slice(i, i + 4096)
        t = torch.bmm(down[a[at]].double(), hidden[at].double()[:, :, None].contiguous())
        add = torch.bmm(up[a[at]].double(), t)[:, :, 0] * scales.double()[a[at]][:, None]
        want = torch.where(ok[at, None], logits[at].double() + add, logits[at].double())
        assert (got[at].double() - want).abs().max() <= 1e-4


def test_logits_beyond_32_bits():
    # Rows of logits whose offset passes 2^32 elements.
    B, V, stride = 70, 1003, 1 << 26
    logits, hidden, down, up, which, scales = _inputs(B, 5, 16, V, 64, BF16, BF16)
    got = torch.empty(B * stride, dtype=BF16, device=DEV).as_strided((B, V), (stride, 1))
    got.copy_(logits)
    sip.sip_head_adapt(got, hidden, down, up, which, scales)
    _check_adapted(got.contiguous(), logits, hidden, down, up, which, scales)
