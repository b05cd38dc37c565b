"""The 4-bit head on hidden states whose mean is not zero, where the zero points' share is as large as the sums it is taken off."""
import math

import pytest
import torch

import paper_2506_22033_amd as sip

from .test_gpu_head import BF16, DEV, F32, make, weights

pytestmark = pytest.mark.gpu
SPAN = 256                                 # entries after which the zero points' share has been taken off, at the latest


@pytest.mark.parametrize("B", [9, 33, 64, 130, 256])
@pytest.mark.parametrize("D,group", [(4096, 128), (4096, 64), (4096, 32), (8192, 128), (16384, 128), (16384, 32), (2080, 32)])
@pytest.mark.parametrize("mean", [1.0, 10.0])
def test_states_with_a_mean(B, D, group, mean):
    """A span's sums run over (16 + q) x in place of (q - zero) x, of 24 |x| s on average; what is rounded at that size is its
    scaled sums, one for each group, and the zero points' share, up to eight additions a span.  Roundings of 2^-24 that are
    independent of each other: sqrt(D / group + D / 32) of them in a row's rms, and those of the result's size, its last one
    among them."""
    for hidden in (BF16, F32):
        for zeros in (False, True):
            x, codes, s, z = make(B, 300, D, group, zeros, hidden, F32, seed=B + D)
            x = (x.float() + mean).to(hidden)
            got = sip.sip_head_logits(x, codes, s, z).double()
            want = x.double() @ weights(codes, s, z).t()
            # the largest span's sum of magnitudes
            spans = []
            for d in range(0, D, SPAN):
                e = min(D, d + SPAN)
                spans.append(x[:, d:e].double().abs() @ (24.0 * s.double().repeat_interleave(group, 1)[:, d:e]).t())
            top = torch.stack(spans).amax(0)
            rms = lambda t: t.square().mean(1).sqrt()                                        # noqa: E731
            allow = 2.0 ** -24 * math.sqrt(D / group + D / 32) * (rms(top) + rms(want))
            assert (rms(got - want) <= allow).all(), float((rms(got - want) / allow).max())
