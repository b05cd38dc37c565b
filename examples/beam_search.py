"""Beam search for many requests on one GPU, every request with an adapter of its own, over one 4-bit matrix that is embedding and head.

A toy recurrent model: state' = tanh(state A + embedding[token]), logits = W state' + the request's low-rank addition.  A step is sip_embed_codes,
the model, sip_head_logits, sip_head_adapt, sip_beam_select and sip_state_reorder; histories stay in a sampler state, and the loop never
waits for the device.  The recurrent states follow their beams by torch's indexing.

    python examples/beam_search.py [--requests 16] [--beams 4] [--steps 20] [--vocab 32000] [--width 512]
"""
from __future__ import annotations

import argparse
import os
import sys

import torch

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
if ROOT not in sys.path:
    sys.path.insert(0, ROOT)

import paper_2506_22033_amd as sip  # noqa: E402

DEV = "cuda:0"


class Model:
    def __init__(self, vocab, width, adapters, rank, seed, group=64):
        g = torch.Generator(device=DEV).manual_seed(seed)
        normal = lambda *size: torch.randn(*size, generator=g, device=DEV)          # noqa: E731
        self.vocab, self.width = vocab, width
        self.codes, self.scales, self.zeros = sip.sip_head_quantize((normal(vocab, width) * 3.0 / width ** 0.5).bfloat16(), group)
        self.step_matrix = normal(width, width) / width ** 0.5
        self.down = (normal(adapters, rank, width) / width ** 0.5).bfloat16()
        self.up = (normal(adapters, vocab, rank) / rank ** 0.5).bfloat16()
        self.adapter_scales = torch.ones(adapters, device=DEV)

    def step(self, state, tokens, adapter_of_row):
        """(the next state, logits in the form that sip_beam_select takes)."""
        vectors = sip.sip_embed_codes(self.codes, self.scales, self.zeros, tokens, 1.5, dtype=torch.float32)
        state = torch.tanh(state @ self.step_matrix + vectors)
        logits = sip.sip_head_logits(state, self.codes, self.scales, self.zeros)
        return state, sip.sip_head_adapt(logits, state, self.down, self.up, adapter_of_row, self.adapter_scales)


def search(model, starts, adapters, beams, steps, end_token):
    """(tokens [requests, beams, steps], scores [requests, beams]) of the best continuations of each start token."""
    requests = starts.numel()
    rows = requests * beams
    slot_of_row = torch.arange(rows, dtype=torch.int32, device=DEV)
    histories = torch.zeros(sip.sip_state_bytes(rows, steps), dtype=torch.uint8, device=DEV)
    sip.sip_state_init(histories, rows, steps)
    adapter_of_row = adapters.repeat_interleave(beams)
    state = torch.zeros(rows, model.width, device=DEV)
    tokens = starts.repeat_interleave(beams)
    scores = torch.full((requests, beams), -torch.inf, device=DEV)
    scores[:, 0] = 0.0                                     # there is one beam before the first step
    finished = torch.zeros(rows, dtype=torch.bool, device=DEV)
    first_row = torch.arange(rows, device=DEV) // beams * beams
    for _ in range(steps):
        state, logits = model.step(state, tokens, adapter_of_row)
        tokens, parents, scores = sip.sip_beam_select(logits, scores.view(-1), beams, finished=finished, end_token=end_token)
        tokens, parents = tokens.view(-1), parents.view(-1)
        sip.sip_state_reorder(histories, rows, steps, slot_of_row, parents, beams, tokens)
        state = state[first_row + parents.long().clamp(min=0)]
        finished = tokens == end_token
    return sip.state_views(histories, rows, steps)[3].view(requests, beams, steps).clone(), scores


def run(requests=16, beams=4, steps=20, vocab=32000, width=512, rank=16, seed=0):
    model = Model(vocab, width, max(1, requests // 2), rank, seed)
    g = torch.Generator(device=DEV).manual_seed(seed + 1)
    starts = torch.randint(0, vocab, (requests,), generator=g, device=DEV, dtype=torch.int32)
    adapters = torch.arange(requests, device=DEV, dtype=torch.int32) // 2 - 1            # (the first two have none)
    tokens, scores = search(model, starts, adapters, beams, steps, end_token=vocab - 1)
    return model, starts, adapters, tokens, scores


def main():
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    for name, value in (("requests", 16), ("beams", 4), ("steps", 20), ("vocab", 32000), ("width", 512)):
        ap.add_argument("--" + name, type=int, default=value)
    a = ap.parse_args()
    _, _, _, tokens, scores = run(a.requests, a.beams, a.steps, a.vocab, a.width)
    alone = run(a.requests, 1, a.steps, a.vocab, a.width)[4]
    print(f"log-probability of the best beam: {float(scores[:, 0].mean()):.3f} on average over {a.requests} requests; of greedy "
          f"decoding {float(alone[:, 0].mean()):.3f}; the first one's tokens {tokens[0, 0].tolist()}")


if __name__ == "__main__":
    main()
