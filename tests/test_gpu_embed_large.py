"""The forms of the embedding's lookup and gradient that large calls take: four rows' pieces a lane from 2^21 units of eight entries on; sorted
tokens in pieces of 16, 32 and 64 entries, from 2^22 units of the gradient on.  Tolerances as in test_gpu_embed.py."""
import pytest
import torch

import paper_2506_22033_amd as sip
from tests.test_gpu_embed import BF16, DEV, F32, TINY, U, _check_gradient, _gen, _half, _ids, _strided

pytestmark = pytest.mark.gpu


# ---------------------------------------------------------------- lookup

def _check_lookup(out, room, rows, ids, V, D, factors):
    ok = (ids >= 0) & (ids < V)
    for i in range(0, ids.numel(), 1000):                 # (in parts: 64 bits of all rows are large)
        at = slice(i, i + 1000)
        want = torch.where(ok[at, None], rows(ids[at].long().clamp(0, V - 1)), 0.0)
        assert ((out[at].double() - want).abs() <= want.abs() * (factors * U + _half(out.dtype)) * 1.01 + TINY).all()
    assert not out[~ok].any() and (room[:, D:] == 77.0).all()


# (units just above 2^21, no multiple of the 1024 of a workgroup)
@pytest.mark.parametrize("pad", [0, 40])
@pytest.mark.parametrize("wt,ot", [(F32, F32), (F32, BF16), (BF16, F32), (BF16, BF16)])
@pytest.mark.parametrize("N,V,D", [(4099, 3001, 4104), (131073, 700, 128)])
def test_lookup(N, V, D, wt, ot, pad):
    assert N * (D // 8) >= 1 << 21 and N * (D // 8) % 1024
    g = _gen(N)
    w, _ = _strided(V, D, wt, pad)
    w.copy_(torch.randn(V, D, generator=g, device=DEV))
    ids = _ids(N, V, g)
    ids[N // 2:N // 2 + 500] = -1
    ids[-1] = V - 1
    out, room = _strided(N, D, ot, pad)
    sip.sip_embed(w, ids, 1.7, out=out)
    _check_lookup(out, room, lambda at: w[at].double() * float(torch.tensor(1.7)), ids, V, D, 1)


@pytest.mark.parametrize("ot", [F32, BF16])
@pytest.mark.parametrize("zeros", [False, True])
@pytest.mark.parametrize("N,V,D,group", [(4099, 900, 4128, 32), (1047, 300, 16128, 128)])
def test_lookup_from_codes(N, V, D, group, zeros, ot):
    assert N * (D // 8) >= 1 << 21 and N * (D // 8) % 1024
    g = _gen(V)
    w = (torch.randn(V, D, generator=g, device=DEV) * 0.1).to(BF16)
    codes, scales, zero = sip.sip_head_quantize(w, group, use_zeros=zeros, scales_dtype=BF16 if zeros else F32)
    ids = _ids(N, V, g)
    ids[-3:] = torch.tensor([-1, 0, V - 1], dtype=torch.int32, device=DEV)
    q = torch.stack((codes & 15, codes >> 4), dim=2).flatten(1).double().unflatten(1, (-1, group))
    z = 8.0 if zero is None else zero.double()[:, :, None]
    rows = ((q - z) * scales.double()[:, :, None]).flatten(1) * float(torch.tensor(0.3))
    out, room = _strided(N, D, ot, 24)
    sip.sip_embed_codes(codes, scales, zero, ids, 0.3, out=out)
    _check_lookup(out, room, lambda at: rows[at], ids, V, D, 2)


# ---------------------------------------------------------------- gradient

LARGE = [(16, 9001, 4096), (32, 20011, 4096), (64, 65536, 2048), (16, 65531, 520), (32, 65000, 1040)]


def _piece(N, D):
    piece = 8
    while piece < 64 and N * (D // 8) >= 2 * piece << 18:
        piece *= 2
    return piece


def _runs(N, V, piece, g):
    """Tokens that appear as often as the rule for cuts has borders: up to two pieces' entries are not cut, more are; in any order."""
    often = [1, 2, 1, piece - 1, piece, piece + 1, 2 * piece - 1, 2 * piece, 2 * piece + 1, 3 * piece, 5 * piece + 3, 70 * piece + 1, 2 * piece, 1, 2 * piece + 1]
    tokens, left, v = [], N, 0
    while left:
        n = min(often[v % len(often)], left)
        tokens += [v % V] * n
        left -= n
        v += 1
    return torch.tensor(tokens, dtype=torch.int32)[torch.randperm(N, generator=torch.Generator().manual_seed(g))].to(DEV)


@pytest.mark.parametrize("gt,wt,accumulate", [(F32, F32, False), (BF16, F32, True), (BF16, BF16, True), (BF16, BF16, False)])
@pytest.mark.parametrize("kind", ["uniform", "frequent", "runs", "one"])
@pytest.mark.parametrize("piece,N,D", LARGE)
def test_gradient_in_longer_pieces(piece, N, D, kind, gt, wt, accumulate):
    assert _piece(N, D) == piece
    V, g = 3001, _gen(N + D)
    grad = torch.randn(N, D, generator=g, device=DEV).to(gt)
    if kind == "uniform":
        ids = _ids(N, V, g)
    elif kind == "frequent":
        ids = (torch.rand(N, generator=g, device=DEV).pow(12) * V).to(torch.int32)
        ids[N // 3:N // 3 + 300] = -1
    elif kind == "runs":
        ids = _runs(N, V, piece, N)
    else:
        ids = torch.full((N,), 17, dtype=torch.int32, device=DEV)
    start = torch.randn(V, D, generator=g, device=DEV).to(wt)
    gw = start.clone()
    sip.sip_embed_backward(grad, ids, V, 2.5, grad_weight=gw, accumulate=accumulate)
    _check_gradient(gw, grad, ids, V, 2.5, start if accumulate else None)
    again = start.clone()
    sip.sip_embed_backward(grad, ids, V, 2.5, grad_weight=again, accumulate=accumulate)
    assert torch.equal(gw, again)


@pytest.mark.parametrize("accumulate", [False, True])
def test_longer_pieces_of_strided_rows_and_a_workspace_that_is_just_enough(accumulate):
    N, V, D = 20011, 900, 4096
    g = _gen(9)
    grad, _ = _strided(N, D, BF16, 24)
    grad.copy_(torch.randn(N, D, generator=g, device=DEV))
    ids = _runs(N, V, 32, 4)
    gw, room = _strided(V, D, F32, 12)
    old = gw.clone()
    need = sip.sip_embed_workspace_bytes(N, V, D)
    ws = torch.full((need + 512,), 0x77, dtype=torch.uint8, device=DEV)
    sip.sip_embed_backward(grad, ids, V, 1.5, grad_weight=gw, accumulate=accumulate, workspace=ws[:need])
    _check_gradient(gw.contiguous(), grad, ids, V, 1.5, old if accumulate else None)
    assert (room[:, D:] == 77.0).all() and (ws[need:] == 0x77).all()


def test_longer_pieces_in_a_graph():
    N, V, D = 9001, 1500, 4096
    g = _gen(5)
    ids = (torch.rand(N, generator=g, device=DEV).pow(4) * V).to(torch.int32)
    grad = torch.randn(N, D, generator=g, device=DEV).to(BF16)
    start = torch.randn(V, D, generator=g, device=DEV)
    want = sip.sip_embed_backward(grad, ids, V, 1.0, grad_weight=start.clone(), accumulate=True)
    gw = start.clone()
    ws = torch.empty(sip.sip_embed_workspace_bytes(N, V, D), dtype=torch.uint8, device=DEV)
    side, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    sip.sip_init()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph, stream=side):
        sip.sip_embed_backward(grad, ids, V, 1.0, grad_weight=gw, accumulate=True, workspace=ws)
    for turn in range(3):
        gw.copy_(start)
        ws.fill_(turn * 57)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(gw, want)
