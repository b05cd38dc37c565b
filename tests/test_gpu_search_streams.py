"""Calls of beams, adapters and embedding with `stream=`: what they allocate themselves is that stream's, and two of them at once do
not meet."""
import pytest
import torch

import paper_2506_22033_amd as sip

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
BF16 = torch.bfloat16


def _calls(seed):
    """(name, call with a stream or None) of every entry point; each gives new tensors."""
    g = torch.Generator(device=DEV).manual_seed(seed)
    w = (torch.randn(3000, 256, generator=g, device=DEV) * 0.1).to(BF16)
    ids = torch.randint(-5, 3000, (700,), generator=g, device=DEV, dtype=torch.int32)
    grad = torch.randn(700, 256, generator=g, device=DEV).to(BF16)
    many = torch.randint(-5, 3000, (9000,), generator=g, device=DEV, dtype=torch.int32)
    grads = torch.randn(9000, 256, generator=g, device=DEV).to(BF16)
    codes, scales, zeros = sip.sip_head_quantize(w, 64)
    logits = torch.randn(24, 30000, generator=g, device=DEV)
    scores = -torch.rand(24, generator=g, device=DEV)
    hidden = torch.randn(24, 256, generator=g, device=DEV).to(BF16)
    down = (torch.randn(3, 16, 256, generator=g, device=DEV) * 0.1).to(BF16)
    up = (torch.randn(3, 30000, 16, generator=g, device=DEV) * 0.1).to(BF16)
    which = torch.randint(-1, 3, (24,), generator=g, device=DEV, dtype=torch.int32)
    adapted = logits.clone()

    def adapt(s):
        with torch.cuda.stream(s or torch.cuda.current_stream()):
            adapted.copy_(logits)
        return [sip.sip_head_adapt(adapted, hidden, down, up, which, stream=s).clone() if s is None else
                sip.sip_head_adapt(adapted, hidden, down, up, which, stream=s)]

    return [("beam_select", lambda s: sip.sip_beam_select(logits, scores, 8, 16, stream=s)),
            ("embed", lambda s: [sip.sip_embed(w, ids, 2.0, stream=s)]),
            ("embed_codes", lambda s: [sip.sip_embed_codes(codes, scales, zeros, ids, stream=s)]),
            ("embed_backward small", lambda s: [sip.sip_embed_backward(grad, ids, 3000, stream=s)]),
            ("embed_backward", lambda s: [sip.sip_embed_backward(grads, many, 3000, stream=s)]),
            ("head_adapt", adapt)]


@pytest.mark.parametrize("which", range(6))
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
    got = [x.clone() for x in got]
    for a, b in zip(got, call(None)):
        assert torch.equal(a, b), name


def test_two_streams_and_other_allocations_beside_them():
    sides = [torch.cuda.Stream() for _ in range(2)]
    calls = [_calls(seed) for seed in (3, 4)]
    want = [[[x.clone() for x in call(None)] for _, call in c] for c in calls]
    torch.cuda.synchronize()
    for _ in range(3):
        got = []
        for i in range(6):
            for c, s in zip(calls, sides):
                got.append(c[i][1](s))
                junk = [torch.full((1 << n,), 0x7f, dtype=torch.uint8, device=DEV) for n in range(12, 24)]   # noqa: F841
        torch.cuda.synchronize()
        for i in range(6):
            for j in range(2):
                for a, b in zip(got[2 * i + j], want[j][i]):
                    assert torch.equal(a, b), calls[j][i][0]
