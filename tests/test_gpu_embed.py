"""sip_embed(), sip_embed_codes() and sip_embed_backward() against their formulas in 64 bits.

Tolerances, relative to the value: a product in fp32 2^-24, the output's rounding half a step (eps / 2).  A sum of k terms in fp32, in
whatever order: (k - 1) 2^-24 of the sum of their magnitudes."""
import math

import pytest
import torch

import paper_2506_22033_amd as sip

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
F32, BF16 = torch.float32, torch.bfloat16
U = 2.0 ** -24
TINY = 1e-37                                              # (below it fp32's and bf16's steps stop shrinking)


def _gen(seed):
    return torch.Generator(device=DEV).manual_seed(seed)


def _half(dtype):
    return torch.finfo(dtype).eps / 2


def _ids(N, V, g, bad=True):
    ids = torch.randint(0, V, (N,), generator=g, device=DEV, dtype=torch.int32)
    if bad and N > 6:
        ids[1], ids[2], ids[3], ids[4], ids[5] = -1, V, -2 ** 31, 2 ** 31 - 1, V - 1
    return ids


def _strided(n, m, dtype, pad):
    """[n, m] inside rows of m + pad, and the whole."""
    room = torch.full((n, m + pad), 77.0, dtype=dtype, device=DEV)
    return room[:, :m], room


@pytest.mark.parametrize("pad", [0, 24])
@pytest.mark.parametrize("wt", [F32, BF16])
@pytest.mark.parametrize("ot", [F32, BF16])
@pytest.mark.parametrize("N,V,D", [(1, 1, 8), (7, 3, 64), (33, 1000, 520), (2, 500, 16384), (5000, 700, 72), (300, 32000, 2048)])
def test_lookup(N, V, D, ot, wt, pad):
    g = _gen(N + D)
    w, _ = _strided(V, D, wt, pad)
    w.copy_(torch.randn(V, D, generator=g, device=DEV))
    ids = _ids(N, V, g)
    out, room = _strided(N, D, ot, pad)
    assert sip.sip_embed(w, ids, 1.7, out=out) is out
    ok = (ids >= 0) & (ids < V)
    want = torch.where(ok[:, None], w.double()[ids.long().clamp(0, V - 1)] * float(torch.tensor(1.7)), 0.0)
    assert ((out.double() - want).abs() <= want.abs() * (U + _half(ot)) * 1.01 + TINY).all()
    assert not out[~ok].any() and (room[:, D:] == 77.0).all()


def test_masked_rows_read_nothing():
    w = torch.full((10, 64), math.nan, device=DEV)
    out = sip.sip_embed(w, torch.full((9,), -1, dtype=torch.int32, device=DEV))
    assert not out.any()
    assert sip.sip_embed(w, torch.empty(0, dtype=torch.int32, device=DEV)).shape == (0, 64)


def test_rows_beyond_32_bits():
    V, D = (1 << 31) // 8192 + 5, 8192
    w = torch.empty(V, D, dtype=BF16, device=DEV)
    w[-1] = torch.arange(D, device=DEV).to(BF16)
    out = sip.sip_embed(w, torch.tensor([V - 1], dtype=torch.int32, device=DEV), dtype=F32)
    assert torch.equal(out[0], w[-1].float())


@pytest.mark.parametrize("ot", [F32, BF16])
@pytest.mark.parametrize("st", [F32, BF16])
@pytest.mark.parametrize("zeros", [False, True])
@pytest.mark.parametrize("N,V,D,group", [(1, 1, 32, 32), (40, 900, 4096, 128), (257, 5000, 192, 64), (1000, 100, 96, 32)])
def test_lookup_from_codes(N, V, D, group, zeros, st, ot):
    g = _gen(V)
    w = (torch.randn(V, D, generator=g, device=DEV) * 0.1).to(BF16)
    codes, scales, zero = sip.sip_head_quantize(w, group, use_zeros=zeros, scales_dtype=st)
    ids = _ids(N, V, g)
    out = sip.sip_embed_codes(codes, scales, zero, ids, 0.3, dtype=ot)
    q = torch.stack((codes & 15, codes >> 4), dim=2).flatten(1).double().unflatten(1, (-1, group))
    z = 8.0 if zero is None else zero.double()[:, :, None]
    rows = ((q - z) * scales.double()[:, :, None]).flatten(1) * float(torch.tensor(0.3))
    ok = (ids >= 0) & (ids < V)
    want = torch.where(ok[:, None], rows[ids.long().clamp(0, V - 1)], 0.0)
    assert ((out.double() - want).abs() <= want.abs() * (2 * U + _half(ot)) * 1.01 + TINY).all()
    assert not out[~ok].any()
    # the same weights as the head multiplies with: logits of a unit vector are a column
    if N > 30 and D >= 128:
        h = torch.zeros(1, D, dtype=BF16, device=DEV)
        h[0, 5] = 1.0
        column = sip.sip_head_logits(h, codes, scales, zero)[0]
        every = sip.sip_embed_codes(codes, scales, zero, torch.arange(V, dtype=torch.int32, device=DEV), dtype=F32)[:, 5]
        assert (column - every).abs().max() <= 2.0 ** -15 * column.abs().max()


# ---------------------------------------------------------------- gradient

def _gradient(grad, ids, V, scale, old=None):
    """The formula in 64 bits, the sum of magnitudes and the number of terms."""
    ok = (ids >= 0) & (ids < V)
    at, x = ids[ok].long(), grad[ok].double() * scale
    total = torch.zeros(V, grad.shape[1], dtype=torch.float64, device=DEV).index_add_(0, at, x)
    size = torch.zeros_like(total).index_add_(0, at, x.abs())
    terms = torch.bincount(at, minlength=V)[:, None]
    if old is not None:
        total, size = total + old.double(), size + old.double().abs()
    return total, size, terms


def _check_gradient(got, grad, ids, V, scale, old=None):
    scale = float(torch.tensor(scale))
    total, size, terms = _gradient(grad, ids, V, scale, old)
    # the sum, the scale, the addition of what was there; then the rounding
    tol = (terms + 2) * U * size * 1.01 + total.abs() * _half(got.dtype) * 1.01 + TINY
    off = (got.double() - total).abs()
    assert (off <= tol).all(), float((off / tol).max())
    if old is None:
        assert not got[(terms == 0)[:, 0]].any()
    else:
        same = (terms == 0)[:, 0]
        assert torch.equal(got[same].view(torch.uint8), old[same].view(torch.uint8))


SIZES = [(1, 1, 8), (1, 50, 64), (2, 5, 2048), (31, 7, 72), (64, 1000, 520), (513, 40, 128), (1000, 1, 16), (4096, 33, 136),
         (1023, 3000, 256), (3000, 2000, 1024), (5, 300, 16384), (20000, 5000, 64), (65536, 700, 8)]


@pytest.mark.parametrize("accumulate", [False, True])
@pytest.mark.parametrize("gt,wt", [(F32, F32), (BF16, BF16), (BF16, F32), (F32, BF16)])
@pytest.mark.parametrize("N,V,D", SIZES)
def test_gradient(N, V, D, gt, wt, accumulate):
    g = _gen(N + V)
    grad = torch.randn(N, D, generator=g, device=DEV).to(gt)
    ids = _ids(N, V, g)
    gw = torch.randn(V, D, generator=g, device=DEV).to(wt)
    old = gw.clone() if accumulate else None
    assert sip.sip_embed_backward(grad, ids, V, 2.5, grad_weight=gw, accumulate=accumulate) is gw
    _check_gradient(gw, grad, ids, V, 2.5, old)


@pytest.mark.parametrize("N,D,V", [(65536, 16, 50000), (40000, 264, 524288 // 8), (9001, 512, 1000)])
def test_frequent_tokens(N, D, V):
    """A few tokens that are everywhere, runs of one token, the same token alone."""
    g = _gen(N)
    grad = torch.randn(N, D, generator=g, device=DEV)
    ids = (torch.rand(N, generator=g, device=DEV).pow(12) * V).to(torch.int32)
    ids[N // 3:N // 2] = 17
    _check_gradient(sip.sip_embed_backward(grad, ids, V, 1.0, dtype=F32), grad, ids, V, 1.0)
    ids[:] = V - 1
    _check_gradient(sip.sip_embed_backward(grad, ids, V, 1.0, dtype=F32), grad, ids, V, 1.0)


@pytest.mark.parametrize("accumulate", [False, True])
@pytest.mark.parametrize("gt", [F32, BF16])
@pytest.mark.parametrize("N,D,V", [(8192, 64, 300), (1000, 512, 4096), (700, 600, 33), (60, 8192, 20), (333, 1544, 129), (17, 4096, 2000)])
def test_frequent_tokens_of_small_calls(N, D, V, gt, accumulate):
    """Runs of one token that cross the workgroup's shares, in one launch."""
    g = _gen(N + D)
    grad = torch.randn(N, D, generator=g, device=DEV).to(gt)
    start = torch.randn(V, D, generator=g, device=DEV)
    for kind in range(3):
        ids = (torch.rand(N, generator=g, device=DEV).pow(6) * V).to(torch.int32)
        if kind == 1:
            ids[:] = V // 2
        if kind == 2:
            ids = torch.arange(N, dtype=torch.int32, device=DEV) % 2 + V - 2
            ids[::7] = -1
        gw = start.clone()
        sip.sip_embed_backward(grad, ids, V, 1.0, grad_weight=gw, accumulate=accumulate)
        _check_gradient(gw, grad, ids, V, 1.0, start if accumulate else None)
        again = start.clone()
        sip.sip_embed_backward(grad, ids, V, 1.0, grad_weight=again, accumulate=accumulate)
        assert torch.equal(gw, again)


def test_the_largest_vocabulary():
    V, D, N = sip.SIP_MAX_V, 8, 3000
    g = _gen(1)
    ids = torch.randint(0, V, (N,), generator=g, device=DEV, dtype=torch.int32)
    ids[0], ids[1], ids[2] = V - 1, 0, V
    grad = torch.randn(N, D, generator=g, device=DEV)
    _check_gradient(sip.sip_embed_backward(grad, ids, V, dtype=F32), grad, ids, V, 1.0)


def test_masked_tokens_take_no_part():
    g = _gen(2)
    N, V, D = 700, 90, 64
    ids = _ids(N, V, g)
    grad = torch.randn(N, D, generator=g, device=DEV)
    ids[100:600] = -100
    want = sip.sip_embed_backward(grad, ids, V, dtype=F32)
    spoilt = grad.clone()
    spoilt[(ids < 0) | (ids >= V)] = math.nan
    assert torch.equal(sip.sip_embed_backward(spoilt, ids, V, dtype=F32), want)
    ids[:] = -1
    gw = torch.full((V, D), math.nan, device=DEV)
    sip.sip_embed_backward(spoilt, ids, V, grad_weight=gw, accumulate=True)
    assert gw.isnan().all()
    sip.sip_embed_backward(spoilt, ids, V, grad_weight=gw)
    assert not gw.any()


def test_no_tokens():
    gw = torch.full((50, 64), 3.0, device=DEV)
    none = torch.empty(0, 64, device=DEV), torch.empty(0, dtype=torch.int32, device=DEV)
    sip.sip_embed_backward(*none, 50, grad_weight=gw, accumulate=True)
    assert (gw == 3.0).all()
    sip.sip_embed_backward(*none, 50, grad_weight=gw)
    assert not gw.any()


@pytest.mark.parametrize("accumulate", [False, True])
def test_strides_and_no_writes_beside(accumulate):
    g = _gen(3)
    N, V, D = 500, 300, 96
    grad, _ = _strided(N, D, BF16, 40)
    grad.copy_(torch.randn(N, D, generator=g, device=DEV))
    ids = _ids(N, V, g)
    gw, room = _strided(V, D, F32, 12)
    old = gw.clone()
    need = sip.sip_embed_workspace_bytes(N, V, D)
    ws = torch.full((need + 512,), 0x77, dtype=torch.uint8, device=DEV)
    sip.sip_embed_backward(grad, ids, V, 1.5, grad_weight=gw, accumulate=accumulate, workspace=ws[:need])
    _check_gradient(gw.contiguous(), grad, ids, V, 1.5, old if accumulate else None)
    assert (room[:, D:] == 77.0).all() and (ws[need:] == 0x77).all()


def test_a_workspace_serves_fewer_tokens():
    for D in (8, 64, 520, 4096, 16384):
        most = 0
        for N in list(range(0, 300)) + list(range(300, 65537, 977)) + [65536]:
            need = sip.sip_embed_workspace_bytes(N, 1000, D)
            assert need >= most, (N, D)
            most = need


def test_the_gradient_is_the_lookup_s():
    """<embed(W'), G> = <W', embed_backward(G)> for any W': the derivative of a linear map, and differences of it."""
    g = _gen(4)
    N, V, D = 900, 150, 64
    ids = _ids(N, V, g)
    w, dw = torch.randn(V, D, generator=g, device=DEV), torch.randn(V, D, generator=g, device=DEV)
    G = torch.randn(N, D, generator=g, device=DEV)
    gw = sip.sip_embed_backward(G, ids, V, 0.5, dtype=F32)
    right = float((dw.double() * gw.double()).sum())
    # each side is a sum of N D products with errors of a few U each, at random; a bound by their magnitudes
    size = float((sip.sip_embed(dw.abs(), ids, 0.5).double() * G.double().abs()).sum())
    assert abs(float((sip.sip_embed(dw, ids, 0.5).double() * G.double()).sum()) - right) <= 40 * U * size
    h = 2.0 ** -3
    up, down = (float((sip.sip_embed(w + s * h * dw, ids, 0.5).double() * G.double()).sum()) for s in (1, -1))
    size = float((sip.sip_embed(w.abs() + dw.abs(), ids, 0.5).double() * G.double().abs()).sum())
    assert abs((up - down) / (2 * h) - right) <= 40 * U * size / h


def test_the_same_bits_every_time_and_in_a_graph():
    g = _gen(5)
    N, V, D = 6000, 1500, 256
    ids = (torch.rand(N, generator=g, device=DEV).pow(4) * V).to(torch.int32)
    grad = torch.randn(N, D, generator=g, device=DEV).to(BF16)
    start = torch.randn(V, D, generator=g, device=DEV)
    want = sip.sip_embed_backward(grad, ids, V, 1.0, grad_weight=start.clone(), accumulate=True)
    w = torch.randn(V, D, generator=g, device=DEV)
    rows = sip.sip_embed(w, ids, 3.0)
    gw, out = start.clone(), torch.empty_like(rows)
    ws = torch.empty(sip.sip_embed_workspace_bytes(N, V, D), dtype=torch.uint8, device=DEV)
    side, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    sip.sip_init()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph, stream=side):
        sip.sip_embed(w, ids, 3.0, out=out)
        sip.sip_embed_backward(grad, ids, V, 1.0, grad_weight=gw, accumulate=True, workspace=ws)
    for turn in range(4):
        gw.copy_(start)
        out.zero_()
        ws.fill_(turn)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(gw, want) and torch.equal(out, rows)
        assert torch.equal(sip.sip_embed_backward(grad, ids, V, 1.0, grad_weight=start.clone(), accumulate=True), want)


def test_refusals():
    w, ids = torch.zeros(10, 64, device=DEV), torch.zeros(5, dtype=torch.int32, device=DEV)
    for bad in (lambda: sip.sip_embed(w.half(), ids), lambda: sip.sip_embed(w, ids.long()), lambda: sip.sip_embed(w.cpu(), ids),
                lambda: sip.sip_embed(w, ids, out=torch.zeros(4, 64, device=DEV)),
                lambda: sip.sip_embed_backward(torch.zeros(4, 64, device=DEV), ids, 10),
                lambda: sip.sip_embed_backward(torch.zeros(5, 64, device=DEV), ids, 10, accumulate=True),
                lambda: sip.sip_embed_backward(torch.zeros(5, 64, device=DEV), ids, 10, grad_weight=torch.zeros(9, 64, device=DEV))):
        with pytest.raises(TypeError):
            bad()
    for bad in (lambda: sip.sip_embed(torch.zeros(10, 60, device=DEV), ids), lambda: sip.sip_embed(torch.zeros(10, 68, device=DEV)[:, :64][:, 2:58], ids),
                lambda: sip.sip_embed_backward(torch.zeros(5, 64, device=DEV), ids, 10, workspace=torch.zeros(64, dtype=torch.uint8, device=DEV)),
                lambda: sip.sip_embed_backward(torch.zeros(5, 64, device=DEV), ids, 0)):
        with pytest.raises(sip.SipError):
            bad()
