"""Cross entropy where its terms leave the ordinary: scales, logits and losses at the ends of their range."""
import math

import pytest
import torch

import paper_2506_22033_amd as sip

from .test_gpu_xent import make, reference

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


@pytest.mark.parametrize("N,V,D", [(1, 1, 8), (1, 1000, 64), (33, 300, 40), (65, 4097, 72), (300, 5000, 1032), (700, 70001, 64),
                                   (2, 40000, 128), (129, 513, 264)])
def test_an_infinite_temperature(N, V, D):
    """logit_scale 0: every logit is 0, loss and lse are ln V (the sum of V ones in fp32, its logarithm: 2^-20 is ample), and
    nothing depends on hidden states or weights."""
    hidden, weight, targets = make(N, V, D, seed=N, masked=0.2)
    live = (targets >= 0) & (targets < V)
    for zero in (0.0, -0.0):
        loss, lse = sip.sip_xent_forward(hidden, weight, targets, zero)
        want = torch.where(live, math.log(V), 0.0)
        assert ((loss - want).abs() <= 2.0 ** -20 * want).all() and ((lse - want).abs() <= 2.0 ** -20 * want).all()
        for g in sip.sip_xent_backward(hidden, weight, targets, loss, lse, logit_scale=zero):
            assert not g.any()


def test_lse_of_a_token_that_is_nearly_impossible():
    """lse does not depend on the target, whose own logit may lie far below: logits of -1 to 1, exact in fp32, and one of -L.
    exp and the sums are off by some 2^-22 each, and so is the result by its rounding: 2^-21 of 1 + |lse|."""
    V, D = 3001, 8
    for L in (10.0, 1000.0, 1e5, 1e30, math.inf):
        weight = torch.zeros(V, D, dtype=torch.bfloat16)
        weight[:, 0] = torch.linspace(-1.0, 1.0, V).bfloat16()
        weight[77, 0] = -L
        hidden = torch.zeros(1, D, dtype=torch.bfloat16)
        hidden[0, 0] = 1.0
        t = torch.tensor([77], dtype=torch.int32, device=DEV)
        loss, lse = sip.sip_xent_forward(hidden.to(DEV), weight.to(DEV), t)
        z = weight[:, 0].double()
        want = torch.logsumexp(z, 0)
        assert abs(float(lse) - float(want)) <= 2.0 ** -21 * (1.0 + abs(float(want))), (L, float(lse), float(want))
        gap = float(want - z[77])
        assert float(loss) == gap or abs(float(loss) - gap) <= 2.0 ** -21 * (1.0 + gap)


@pytest.mark.parametrize("N,live,V,D", [(65, 1, 3001, 136), (100, 2, 20000, 256), (100, 64, 3001, 136), (128, 40, 4097, 520), (2000, 3, 20000, 256),
                                        (5000, 64, 3000, 64), (3000, 17, 70000, 1032), (65536, 9, 5000, 16)])
def test_few_tokens_among_masked_ones(N, live, V, D):
    """What counts for dz's two parts is the tokens that take part: the bound is that of a call of nothing else (2^-8 of 2^-8 of a
    term lost in dz; the result's rounding, 2^-8; the probabilities' error; sums in fp32, a random walk)."""
    hidden, weight, targets = make(N, V, D, seed=N + live)
    g = torch.Generator().manual_seed(live)
    off = torch.randperm(N, generator=g)[live:].to(DEV)
    targets[off] = -100
    hidden[off] = math.nan
    loss, lse = sip.sip_xent_forward(hidden, weight, targets, 0.8)
    gh, gw = sip.sip_xent_backward(hidden, weight, targets, loss, lse, None, 0.5, 0.8)
    ref = reference(hidden, weight, targets, 0.8, None, 0.5)
    p_err = 8 * 2.0 ** -24 * math.sqrt(D) * float(ref[4].max()) + 2.0 ** -20
    for got, want, terms, count in ((gh, ref[2], ref[5], V), (gw, ref[3], ref[6], live)):
        bound = 2.0 ** -8 * want.abs() + (2.0 ** -16 + p_err + 4 * 2.0 ** -24 * math.sqrt(count)) * 1.01 * terms + 1e-30
        assert ((got.double() - want).abs() <= bound).all()
    assert not gh[off].any()
    # each gradient alone, the same bits
    a, _ = sip.sip_xent_backward(hidden, weight, targets, loss, lse, None, 0.5, 0.8, want_weight=False)
    _, b = sip.sip_xent_backward(hidden, weight, targets, loss, lse, None, 0.5, 0.8, want_hidden=False)
    assert torch.equal(a, gh) and torch.equal(b, gw)


def test_one_workspace_for_batches_of_any_size():
    """A workspace that is enough for the largest batch serves the smaller ones, both ways, and gives their bits."""
    V, D, most = 3001, 264, 700
    ws = torch.empty(sip.sip_xent_workspace_bytes(most, V, D, True), dtype=torch.uint8, device=DEV)
    small = torch.empty(sip.sip_xent_workspace_bytes(most, V, D, False), dtype=torch.uint8, device=DEV)
    for N in (700, 699, 513, 384, 257, 130, 128, 100, 65, 64, 63, 33, 20, 3, 1):
        hidden, weight, targets = make(N, V, D, seed=N, masked=0.1)
        want = sip.sip_xent_forward(hidden, weight, targets)
        for w in (ws, small):
            assert all(torch.equal(a, b) for a, b in zip(sip.sip_xent_forward(hidden, weight, targets, workspace=w), want))
        for a, b in zip(sip.sip_xent_backward(hidden, weight, targets, *want, workspace=ws),
                        sip.sip_xent_backward(hidden, weight, targets, *want)):
            assert torch.equal(a, b)
