"""sip_beam_select() against its formula in 64 bits.

Tolerance of a total: lse comes from fp32 terms.  A term 2^x of relative weight p has the error of its exponent's two roundings
(2^-24 |x| each, times ln 2) and of the exponential (2^-23); over the row these weigh at most 2^-23 + 2 * 2^-24 * ln 2 * E|x|, and
E|x| is at most log2(V) + 2 <= 21; sixteen terms are added one after the other in fp32 (16 * 2^-24).  Together below 3e-6.
Of two continuations whose totals differ by less, either may come first; everything else has to be equal."""
import math

import pytest
import torch

import paper_2506_22033_amd as sip

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
TOL = 3e-6
INF = math.inf


def _rows(R, V, dtype, seed, scale=2.5):
    g = torch.Generator(device=DEV).manual_seed(seed)
    stride = (V + 7) // 8 * 8
    return (torch.randn(R, stride, generator=g, device=DEV) * scale).to(dtype)[:, :V], g


def _totals(logits, scores, finished=None, end_token=0, logit_scale=1.0):
    """[R, V] in 64 bits, -inf where there is no continuation."""
    z = logits.double() * logit_scale
    total = scores.double()[:, None] + torch.log_softmax(z, dim=1)
    bad = ~torch.isfinite(scores) | z.isnan().any(1) | (z == INF).any(1) | ~(z > -INF).any(1)
    total[bad] = -INF
    total = torch.where(z > -INF, total, -INF)
    if finished is not None:
        done = finished != 0
        total[done] = -INF
        total[done, end_token] = torch.where(torch.isfinite(scores[done]), scores[done], -INF).double()
    return total


def _check(logits, scores, width, n, got, finished=None, rank_scale=None, end_token=0, logit_scale=1.0):
    tokens, parents, out = (x.cpu() for x in got)
    R, V = logits.shape
    G = R // width
    total = _totals(logits, scores, finished, end_token, logit_scale).cpu()
    scale = torch.ones(R, dtype=torch.float64) if rank_scale is None else rank_scale.double().cpu()
    rank = torch.where(total > -INF, total * scale[:, None], -INF)
    for g in range(G):
        rows = slice(g * width, (g + 1) * width)
        have = int((rank[rows] > -INF).sum())
        m = min(n, have)
        want = rank[rows].flatten().topk(m).values
        t, p, s = tokens[g, :m].long(), parents[g, :m].long(), out[g, :m].double()
        assert (t >= 0).all() and (t < V).all() and (p >= 0).all() and (p < width).all()
        assert len(set(zip(t.tolist(), p.tolist()))) == m, "a continuation twice"
        assert ((rank[rows][p, t] - want).abs() <= TOL * scale[rows].max()).all()
        exact = total[rows][p, t]
        assert ((s - exact).abs() <= TOL + 2.0 ** -24 * exact.abs()).all()
        assert (tokens[g, m:] == -1).all() and (parents[g, m:] == -1).all() and (out[g, m:] == -INF).all()


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("groups,width,V,n", [
    (1, 1, 1, 1), (1, 1, 7, 4), (2, 3, 40, 9), (1, 4, 1000, 4), (3, 2, 8191, 5), (2, 2, 8192, 4), (2, 2, 8193, 4), (5, 4, 32000, 8),
    (1, 64, 5000, 128), (2, 32, 20000, 64), (1, 1, 262144, 128), (1, 3, 524288, 6), (70, 1, 3000, 2), (1, 5, 100, 128)])
def test_selection(groups, width, V, n, dtype):
    logits, g = _rows(groups * width, V, dtype, V + n)
    scores = -torch.rand(groups * width, generator=g, device=DEV) * 20.0
    _check(logits, scores, width, n, sip.sip_beam_select(logits, scores, width, n))


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_finished_beams_scaled_ranks_and_a_temperature(dtype):
    logits, g = _rows(6 * 5, 33333, dtype, 1)
    scores = -torch.rand(30, generator=g, device=DEV) * 8.0
    finished = torch.rand(30, generator=g, device=DEV) < 0.4
    rank_scale = 1.0 / torch.randint(3, 60, (30,), generator=g, device=DEV).float()
    for done in (finished, finished.to(torch.uint8) * 7):
        got = sip.sip_beam_select(logits, scores, 5, 10, finished=done, rank_scale=rank_scale, end_token=33332, logit_scale=0.7)
        _check(logits, scores, 5, 10, got, finished, rank_scale, 33332, float(torch.tensor(0.7)))


def test_scores_of_finished_beams_are_unchanged():
    logits, g = _rows(4, 500, torch.float32, 2)
    scores = torch.tensor([-1.2345678, -0.1, -3.3, -7.7], device=DEV)
    done = torch.tensor([1, 0, 1, 1], dtype=torch.uint8, device=DEV)
    tokens, parents, out = sip.sip_beam_select(logits, scores, 4, 128, finished=done, end_token=9)
    for k in (0, 2, 3):
        at = ((parents == k).nonzero()[:, 1])
        assert at.numel() == 1 and tokens[0, at] == 9 and out[0, at] == scores[k]


def test_beams_that_do_not_exist_are_not_read():
    """What their logits hold, NaN included, goes nowhere; nor does what finished beams' hold."""
    logits, g = _rows(12, 9000, torch.float32, 3)
    scores = -torch.rand(12, generator=g, device=DEV)
    scores[1::2] = -INF
    scores[3], scores[5] = INF, math.nan
    done = torch.zeros(12, dtype=torch.uint8, device=DEV)
    done[6] = 1
    want = sip.sip_beam_select(logits, scores, 4, 8, finished=done, end_token=5)
    _check(logits, torch.where(torch.isfinite(scores), scores, -INF), 4, 8, want, done, None, 5)
    spoilt = logits.clone()
    spoilt[1::2] = math.nan
    spoilt[6] = INF
    stride = (9000 + 7) // 8 * 8
    room = torch.empty(12, stride, device=DEV)[:, :9000]
    room.copy_(spoilt)
    for a, b in zip(want, sip.sip_beam_select(room, scores, 4, 8, finished=done, end_token=5)):
        assert torch.equal(a, b)


@pytest.mark.parametrize("what", [math.nan, INF])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_rows_with_nan_or_infinity_have_no_continuation(what, dtype):
    logits, g = _rows(6, 20000, dtype, 4)
    scores = -torch.rand(6, generator=g, device=DEV)
    logits[1, 19999] = what
    logits[3, 0] = what
    logits[4] = what
    _check(logits, scores, 3, 6, sip.sip_beam_select(logits, scores, 3, 6))


def test_masked_logits():
    """-inf and the type's lowest value: rows with few tokens left, one, none."""
    logits, g = _rows(8, 30000, torch.float32, 5)
    scores = -torch.rand(8, generator=g, device=DEV)
    logits[0] = -INF
    logits[1, 1:] = -INF
    logits[2, :29999] = -INF
    logits[3, 7:] = -INF
    logits[4, torch.rand(30000, generator=g, device=DEV) < 0.9995] = -INF
    logits[5, 3:] = torch.finfo(torch.float32).min
    for n in (1, 4, 16, 128):
        _check(logits, scores, 2, n, sip.sip_beam_select(logits, scores, 2, n))


@pytest.mark.parametrize("n", [1, 5, 128])
@pytest.mark.parametrize("V", [100, 8192, 50001])
def test_equal_logits_go_by_beam_and_token(V, n):
    """All continuations of a group tie: the lowest beam's lowest tokens."""
    logits = torch.zeros(6, (V + 7) // 8 * 8, device=DEV)[:, :V]
    logits[:, ::2] = -0.0                                  # the same number
    scores = torch.full((6,), -2.0, device=DEV)
    tokens, parents, out = (x.cpu() for x in sip.sip_beam_select(logits, scores, 3, n))
    for g in range(2):
        assert tokens[g].tolist() == [i % V for i in range(n)] and parents[g].tolist() == [i // V for i in range(n)]
    assert (out.double() + 2.0 + math.log(V)).abs().max() <= TOL + 2.0 ** -23 * (2 + math.log(V))


def test_ties_within_a_row_and_between_equal_rows():
    logits, g = _rows(1, 40000, torch.bfloat16, 6)
    stride = 40000
    room = torch.empty(4, stride, dtype=torch.bfloat16, device=DEV)
    room.copy_(logits.expand(4, -1))
    scores = torch.full((4,), -1.0, device=DEV)
    tokens, parents, _ = (x.cpu() for x in sip.sip_beam_select(room, scores, 4, 128))
    z = logits[0].double().cpu()
    order = sorted(range(40000), key=lambda v: (-float(z[v]), v))[:200]
    want, i = [], 0
    while len(want) < 128:                                 # equal totals: beam by beam, within it by token
        j = i
        while j < len(order) and z[order[j]] == z[order[i]]:
            j += 1
        want += [(k, v) for k in range(4) for v in order[i:j]]
        i = j
    assert list(zip(parents[0].tolist(), tokens[0].tolist())) == want[:128]


def test_nearly_equal_logits():
    """Thousands of values closer to one another than the first bits tell."""
    V = 24576
    z = 1.0 + torch.randperm(V, generator=torch.Generator().manual_seed(7)).float() * 2.0 ** -23
    logits = torch.stack((z, -z)).to(DEV)
    scores = torch.tensor([-1.0, -1.0], device=DEV)
    tokens, parents, _ = (x.cpu() for x in sip.sip_beam_select(logits, scores, 1, 100))
    for g, x in enumerate((z, -z)):
        assert tokens[g].tolist() == x.double().sort(descending=True, stable=True).indices[:100].tolist()


def test_strides_outputs_workspace_and_no_writes_beside():
    room = torch.full((6, 4096), 7.0, device=DEV)
    logits = room[:, :3001]
    g = torch.Generator(device=DEV).manual_seed(8)
    logits.copy_(torch.randn(6, 3001, generator=g, device=DEV))
    before = room.clone()
    scores = -torch.rand(6, generator=g, device=DEV)
    want = sip.sip_beam_select(logits.clone().new_empty(6, 3008)[:, :3001].copy_(logits), scores, 3)
    need = sip.sip_beam_workspace_bytes(2, 3, 3001, 3)
    ws = torch.full((need + 256,), 0xA5, dtype=torch.uint8, device=DEV)
    got = sip.sip_beam_select(logits, scores, 3, workspace=ws[:need])
    for a, b in zip(want, got):
        assert torch.equal(a, b)
    assert torch.equal(room, before) and (ws[need:] == 0xA5).all()
    # the scores in place
    kept = scores.clone()
    sip.sip_beam_select(logits, kept, 3, out_scores=kept, workspace=ws)
    assert torch.equal(kept.view(2, 3), want[2])


def test_a_workspace_serves_smaller_calls():
    need = sip.sip_beam_workspace_bytes(8, 4, 50000, 8)
    for smaller in ((7, 4, 50000, 8), (8, 3, 50000, 8), (8, 4, 1000, 8), (8, 4, 50000, 1), (1, 1, 1, 1)):
        assert sip.sip_beam_workspace_bytes(*smaller) <= need


def test_the_same_bits_every_time_and_in_a_graph():
    logits, g = _rows(24, 50000, torch.bfloat16, 9)
    scores = -torch.rand(24, generator=g, device=DEV) * 3
    want = [x.clone() for x in sip.sip_beam_select(logits, scores, 8, 16)]
    ws = torch.empty(sip.sip_beam_workspace_bytes(3, 8, 50000, 16), dtype=torch.uint8, device=DEV)
    out = [torch.empty_like(x) for x in want]
    sip.sip_init()
    side = torch.cuda.Stream()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        sip.sip_beam_select(logits, scores, 8, 16, tokens=out[0], parents=out[1], out_scores=out[2], workspace=ws)
    for turn in range(4):
        ws.fill_(0x5A + turn)
        for x in out:
            x.zero_()
        graph.replay()
        torch.cuda.synchronize()
        for a, b, c in zip(want, out, sip.sip_beam_select(logits, scores, 8, 16)):
            assert torch.equal(a, b) and torch.equal(a, c)


def test_rows_beyond_32_bits():
    """A row that starts past 2^31 elements."""
    V, far = 1000, (1 << 31) + 4096
    room = torch.empty(far + 2048, dtype=torch.bfloat16, device=DEV)
    logits = room.as_strided((2, V), (far, 1))
    g = torch.Generator(device=DEV).manual_seed(10)
    z = torch.randn(2, V, generator=g, device=DEV).bfloat16()
    logits.copy_(z)
    scores = torch.tensor([-1.0, -1.5], device=DEV)
    _check(z, scores, 2, 6, sip.sip_beam_select(logits, scores, 2, 6))


def test_refusals():
    logits, g = _rows(6, 100, torch.float32, 11)
    scores = torch.zeros(6, device=DEV)
    for kw in (dict(width=4), dict(width=0), dict(width=3, finished=torch.zeros(6, device=DEV)), dict(width=3, rank_scale=scores[:5]),
               dict(width=3, tokens=torch.empty(2, 4, dtype=torch.int32, device=DEV))):
        with pytest.raises(TypeError):
            sip.sip_beam_select(logits, scores, **kw)
    with pytest.raises(TypeError):
        sip.sip_beam_select(logits, scores[:5], 3)
    with pytest.raises(TypeError):
        sip.sip_beam_select(logits.half(), scores, 3)
    for kw in (dict(n=129), dict(logit_scale=0.0), dict(logit_scale=INF), dict(finished=torch.zeros(6, dtype=torch.bool, device=DEV), end_token=100),
               dict(workspace=torch.empty(16, dtype=torch.uint8, device=DEV)), dict(n=0)):
        with pytest.raises(sip.SipError):
            sip.sip_beam_select(logits, scores, 3, **kw)
    with pytest.raises(sip.SipError):                      # rows that do not start at 16 bytes
        sip.sip_beam_select(torch.zeros(6, 101, device=DEV), scores, 3)
