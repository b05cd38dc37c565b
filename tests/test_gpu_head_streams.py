"""Calls with `stream=`: what they allocate themselves is that stream's, so that nobody else is handed it while they run."""
import pytest
import torch

import paper_2506_22033_amd as sip

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
BF16 = torch.bfloat16


def _inputs(seed):
    g = torch.Generator(device=DEV).manual_seed(seed)
    h = torch.randn(200, 256, generator=g, device=DEV).to(BF16)
    w = (torch.randn(3000, 256, generator=g, device=DEV) * 0.1).to(BF16)
    t = torch.randint(0, 3000, (200,), generator=g, device=DEV, dtype=torch.int32)
    return h, w, t


def _calls(seed):
    """(name, call with a stream or None) of every entry point that allocates outputs or scratch memory."""
    h, w, t = _inputs(seed)
    loss, lse = sip.sip_xent_forward(h, w, t)
    codes, scales, zeros = sip.sip_head_quantize(w, 64)
    grads = [w.clone(), h.clone()]
    outs = [torch.empty_like(x) for x in grads]
    table = sip.GradTable(grads, outs)

    def clip(s):
        return [sip.sip_grad_clip(table, 0.5, stream=s)] + outs

    return [("xent_forward", lambda s: sip.sip_xent_forward(h, w, t, stream=s)),
            ("xent_backward", lambda s: sip.sip_xent_backward(h, w, t, loss, lse, stream=s)),
            ("grad_clip", clip),
            ("head_quantize", lambda s: sip.sip_head_quantize(w, 64, stream=s)),
            ("head_logits", lambda s: [sip.sip_head_logits(h, codes, scales, zeros, stream=s)])]


@pytest.mark.parametrize("which", range(5))
def test_everything_is_allocated_on_the_stream(which, monkeypatch):
    name, call = _calls(1)[which]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    plain, seen = torch.empty, []

    def recorded(*a, **k):
        seen.append(torch.cuda.current_stream())
        return plain(*a, **k)

    monkeypatch.setattr(torch, "empty", recorded)
    got = call(side)
    monkeypatch.undo()
    assert torch.cuda.current_stream() != side
    assert seen and all(s == side for s in seen), name
    side.synchronize()
    for a, b in zip(got, call(None)):
        assert torch.equal(a, b), name


def test_two_streams_and_other_allocations_beside_them():
    sides = [torch.cuda.Stream() for _ in range(2)]
    calls = [_calls(seed) for seed in (3, 4)]
    want = [[[x.clone() for x in call(None)] for _, call in c] for c in calls]
    torch.cuda.synchronize()
    for _ in range(3):
        got = []
        for i in range(5):
            for c, s in zip(calls, sides):
                got.append(c[i][1](s))
                junk = [torch.full((1 << n,), 0x7f, dtype=torch.uint8, device=DEV) for n in range(12, 24)]   # noqa: F841
        torch.cuda.synchronize()
        for i in range(5):
            for j in range(2):
                for a, b in zip(got[2 * i + j], want[j][i]):
                    assert torch.equal(a, b), calls[j][i][0]


def test_the_gradient_of_no_tokens_is_cleared_on_the_stream():
    """Behind what the stream does already, not ahead of it."""
    h, w, t = torch.empty(0, 64, dtype=BF16, device=DEV), torch.zeros(50, 64, dtype=BF16, device=DEV), torch.empty(
        0, dtype=torch.int32, device=DEV)
    none = torch.empty(0, device=DEV)
    gw = torch.empty(50, 64, dtype=BF16, device=DEV)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        for _ in range(50):
            big = torch.randn(4096, 4096, device=DEV).sort(dim=1)[0]                 # (some work ahead)
        gw.copy_(big[:50, :64].to(BF16).abs() + 1.0)
    sip.sip_xent_backward(h, w, t, none, none, grad_weight=gw, stream=side)
    side.synchronize()
    torch.cuda.synchronize()
    assert not gw.any()
