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
