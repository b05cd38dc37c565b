"""The sampling calls with `stream=`: outputs and workspaces that they allocate are that stream's."""
import pytest
import torch

import paper_2506_22033_amd as sip
from paper_2506_22033_amd.binding import sip_sample_call

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
B, V, SLOTS, L = 20, 5000, 32, 64


def _calls():
    g = torch.Generator(device=DEV).manual_seed(2)
    logits = torch.randn(B, V, generator=g, device=DEV)
    params = {"temperature": torch.full((B,), 0.9, device=DEV), "top_p": torch.full((B,), 0.8, device=DEV)}
    half = [logits[:, :2496].contiguous(), logits[:, 2496:4992].contiguous()]
    state = torch.zeros(sip.sip_state_bytes(SLOTS, L), dtype=torch.uint8, device=DEV)
    rows = torch.arange(B, dtype=torch.int32, device=DEV)

    def on_state(s):
        sip.sip_state_init(state, SLOTS, L, stream=s)
        return sip.sip_sample_state(logits, params, state, SLOTS, L, rows, 5, 0, 3, stream=s)

    return [lambda s: sip.sip_sample(logits, params, None, None, 5, 0, 3, stream=s), on_state,
            lambda s: sip.sip_sample_sharded(half, params, None, None, 5, 0, 3, stream=s),
            lambda s: sip_sample_call(logits=logits, params=params, seed=5, step=0, k_logprobs=3, stream=s)]


@pytest.mark.parametrize("which", range(4))
def test_everything_is_allocated_on_the_stream(which, monkeypatch):
    call = _calls()[which]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    plain, seen = torch.empty, []

    def recorded(*a, **k):
        seen.append(torch.cuda.current_stream())
        return plain(*a, **k)

    monkeypatch.setattr(torch, "empty", recorded)
    got = call(side)
    monkeypatch.undo()
    assert len(seen) == 4 and all(s == side for s in seen)
    side.synchronize()
    for a, b in zip(got, call(None)):
        assert torch.equal(a, b)
