"""The operators together: the search of examples/beam_search.py, the same steps in a graph, and a training step of a matrix that is
embedding and head."""
import importlib.util
import os

import pytest
import torch

import paper_2506_22033_amd as sip

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
BF16 = torch.bfloat16
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def _example():
    spec = importlib.util.spec_from_file_location("beam_search", os.path.join(ROOT, "examples", "beam_search.py"))
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    return m


def _score(model, start, adapter, tokens, end_token):
    """Log-probability of one sequence under the model, in 64 bits."""
    group = model.width // model.scales.shape[1]
    q = torch.stack((model.codes & 15, model.codes >> 4), dim=2).flatten(1).double().unflatten(1, (-1, group))
    w = ((q - model.zeros.double()[:, :, None]) * model.scales.double()[:, :, None]).flatten(1)
    state, total, token = torch.zeros(model.width, dtype=torch.float64, device=DEV), 0.0, start
    for t in tokens:
        state = torch.tanh(state @ model.step_matrix.double() + 1.5 * w[token])
        z = w @ state
        if adapter >= 0:
            z = z + model.up[adapter].double() @ (model.down[adapter].double() @ state)
        total += float(torch.log_softmax(z, dim=0)[t])
        token = t
        if t == end_token:
            break
    return total


def test_the_example_s_scores_are_those_of_its_sequences():
    m = _example()
    model, starts, adapters, tokens, scores = m.run(requests=6, beams=3, steps=7, vocab=2000, width=128)
    assert (scores[:, :-1] >= scores[:, 1:]).all()
    for r in range(6):
        assert len({tuple(tokens[r, k].tolist()) for k in range(3)}) == 3
        for k in range(3):
            want = _score(model, int(starts[r]), int(adapters[r]), tokens[r, k].tolist(), 1999)
            # states and logits in fp32: sums of 128 terms, seven steps
            assert abs(want - float(scores[r, k])) <= 1e-3, (r, k)
    greedy = m.run(requests=6, beams=1, steps=7, vocab=2000, width=128)
    assert (scores[:, 0] >= greedy[4][:, 0] - 1e-3).all()


def test_steps_in_a_graph():
    """A step recorded once and replayed is the step itself: its own outputs are its next inputs."""
    m = _example()
    requests, beams, steps, vocab, width = 4, 4, 6, 3000, 128
    model = m.Model(vocab, width, 2, 16, 0)
    rows = requests * beams
    starts = torch.arange(10, 10 + requests, dtype=torch.int32, device=DEV)
    adapters = torch.tensor([0, 1, -1, 1], dtype=torch.int32, device=DEV)
    want_tokens, want_scores = m.search(model, starts, adapters, beams, steps, vocab - 1)
    sip.sip_init()
    histories = torch.zeros(sip.sip_state_bytes(rows, steps), dtype=torch.uint8, device=DEV)
    slot_of_row, adapter_of_row = torch.arange(rows, dtype=torch.int32, device=DEV), adapters.repeat_interleave(beams)
    first_row = torch.arange(rows, device=DEV) // beams * beams
    state, tokens = torch.zeros(rows, width, device=DEV), starts.repeat_interleave(beams)
    scores, finished = torch.empty(rows, device=DEV), torch.zeros(rows, dtype=torch.bool, device=DEV)
    parents = torch.empty(rows, dtype=torch.int32, device=DEV)

    def start():
        sip.sip_state_init(histories, rows, steps)
        state.zero_()
        tokens.copy_(starts.repeat_interleave(beams))
        scores.fill_(-torch.inf)
        scores[::beams] = 0.0
        finished.zero_()

    def step():
        new, logits = model.step(state, tokens, adapter_of_row)
        sip.sip_beam_select(logits, scores, beams, finished=finished, end_token=vocab - 1, tokens=tokens, parents=parents, out_scores=scores)
        sip.sip_state_reorder(histories, rows, steps, slot_of_row, parents, beams, tokens)
        state.copy_(new[first_row + parents.long().clamp(min=0)])
        finished.copy_(tokens == vocab - 1)

    side, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    start()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph, stream=side):
        step()
    for _ in range(3):
        start()
        for _ in range(steps):
            graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(sip.state_views(histories, rows, steps)[3].view(requests, beams, steps), want_tokens)
        assert torch.equal(scores.view(requests, beams), want_scores)


def test_a_training_step_of_a_shared_matrix():
    """loss(W) = sum of the cross entropy of next tokens, hidden states being W's own rows: both gradients, added and clipped."""
    N, V, D, scale = 600, 900, 64, 2.0
    g = torch.Generator(device=DEV).manual_seed(0)
    w = (torch.randn(V, D, generator=g, device=DEV) * 0.3).to(BF16)
    ids = torch.randint(0, V, (N,), generator=g, device=DEV, dtype=torch.int32)
    targets = torch.randint(0, V, (N,), generator=g, device=DEV, dtype=torch.int32)
    ids[::50] = -1
    targets[::7] = -100
    hidden = sip.sip_embed(w, ids, scale)
    loss, lse = sip.sip_xent_forward(hidden, w, targets)
    gh, gw = sip.sip_xent_backward(hidden, w, targets, loss, lse, scale=1.0 / N)
    head = gw.clone()
    sip.sip_embed_backward(gh, ids, V, scale, grad_weight=gw, accumulate=True)
    w64 = w.double().requires_grad_()
    ok = (ids >= 0)[:, None]
    h64 = torch.where(ok, w64[ids.long().clamp(min=0)] * scale, 0.0)
    h64 = h64 + (hidden.double() - h64).detach()          # the states as they were rounded
    keep = targets >= 0
    total = torch.nn.functional.cross_entropy(h64[keep] @ w64.t(), targets[keep].long(), reduction="sum") / N
    total.backward()
    off = (gw.double() - w64.grad).norm() / w64.grad.norm()
    # three roundings to bf16 (hidden's gradient, the head's, the sum; dz before them): each half a step, 2^-8
    assert off <= 4 * 2.0 ** -8
    assert not torch.equal(gw, head)
    norm = sip.sip_grad_clip([gw], 0.1)
    assert abs(float(norm) - float(w64.grad.norm())) <= 4 * 2.0 ** -8 * float(norm)
