"""sip_head_adapt() against its formula in 64 bits.

Tolerance of a new logit, with S = sum_j |up| sum_d |down| |hidden| |scale|: two nested sums of D and rank terms in fp32 in whatever order
err by (D + rank + 4) 2^-24 S at most (products included), the addition by 2^-24 and the rounding by half a step of the result."""
import math

import pytest
import torch

import paper_2506_22033_amd as sip

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
F32, BF16 = torch.float32, torch.bfloat16
U = 2.0 ** -24


def _inputs(B, A, r, V, D, xt, zt, seed=0, pad=0):
    g = torch.Generator(device=DEV).manual_seed(seed + B + V)
    hidden = torch.empty(B, D + pad, dtype=xt, device=DEV)[:, :D]
    hidden.copy_(torch.randn(B, D, generator=g, device=DEV))
    down = (torch.randn(A, r, D, generator=g, device=DEV) / math.sqrt(D)).to(BF16)
    up = (torch.randn(A, V, r, generator=g, device=DEV) / math.sqrt(r)).to(BF16)
    scales = torch.rand(A, generator=g, device=DEV) * 2 - 0.5
    which = torch.randint(-1, A, (B,), generator=g, device=DEV, dtype=torch.int32)
    logits = torch.randn(B, V, generator=g, device=DEV).to(zt)
    return logits, hidden, down, up, which, scales


def _check(got, logits, hidden, down, up, which, scales=None):
    A, r, D = down.shape
    for b in range(logits.shape[0]):
        a = int(which[b])
        if not 0 <= a < A:
            assert torch.equal(got[b].view(torch.uint8), logits[b].view(torch.uint8)), b
            continue
        s = 1.0 if scales is None else float(scales[a])
        x, y, u = hidden[b].double(), down[a].double(), up[a].double()
        want = logits[b].double() + s * (u @ (y @ x))
        size = abs(s) * (u.abs() @ (y.abs() @ x.abs()))
        tol = (D + r + 4) * U * size * 1.01 + want.abs() * (U + torch.finfo(got.dtype).eps / 2) * 1.01 + 1e-37
        off = (got[b].double() - want).abs()
        assert (off <= tol).all(), (b, float((off / tol).max()))


@pytest.mark.parametrize("xt,zt", [(BF16, F32), (F32, F32), (BF16, BF16), (F32, BF16)])
@pytest.mark.parametrize("B,A,r,V,D", [
    (1, 1, 8, 1, 8), (1, 3, 16, 1000, 64), (5, 2, 8, 33, 72), (17, 1, 64, 300, 128), (16, 4, 24, 5001, 520), (40, 3, 128, 257, 256),
    (64, 64, 16, 700, 512), (256, 7, 32, 129, 64), (3, 2, 56, 2000, 8192), (33, 2, 40, 50257, 64), (100, 1, 16, 4099, 1024)])
def test_adapters(B, A, r, V, D, xt, zt):
    logits, hidden, down, up, which, scales = _inputs(B, A, r, V, D, xt, zt)
    got = logits.clone()
    assert sip.sip_head_adapt(got, hidden, down, up, which, scales) is got
    _check(got, logits, hidden, down, up, which, scales)


def test_without_scales_every_row_one_adapter_and_none():
    logits, hidden, down, up, which, _ = _inputs(50, 4, 16, 900, 256, BF16, F32)
    for rows in (torch.full_like(which, 2), torch.full_like(which, -1), torch.full_like(which, 4), torch.arange(50, device=DEV).int() % 4):
        got = logits.clone()
        sip.sip_head_adapt(got, hidden, down, up, rows)
        _check(got, logits, hidden, down, up, rows)


def test_rows_without_an_adapter_are_not_touched_whatever_they_hold():
    logits, hidden, down, up, which, scales = _inputs(20, 3, 16, 900, 256, BF16, F32)
    which[::2] = torch.tensor([-1, 3, -2 ** 31, 2 ** 31 - 1, -1, 3, 3, 3, -5, 99], dtype=torch.int32, device=DEV)
    which[1::2] = 1
    clean = logits.clone()
    sip.sip_head_adapt(clean, hidden, down, up, which, scales)
    hidden[::2] = math.nan
    logits[::2] = math.nan
    got = logits.clone()
    down[0], up[0] = math.nan, math.inf                    # nobody's
    scales[2] = math.nan
    sip.sip_head_adapt(got, hidden, down, up, which, scales)
    assert got[::2].isnan().all() and torch.equal(got[1::2], clean[1::2])


def test_a_bad_row_spoils_itself_alone():
    logits, hidden, down, up, which, scales = _inputs(20, 1, 16, 900, 256, BF16, F32)
    which[:] = 0
    clean = logits.clone()
    sip.sip_head_adapt(clean, hidden, down, up, which, scales)
    hidden[7, 3], hidden[9, 0] = math.nan, math.inf
    sip.sip_head_adapt(logits, hidden, down, up, which, scales)
    rest = [b for b in range(20) if b not in (7, 9)]
    assert torch.equal(logits[rest], clean[rest]) and not torch.isfinite(logits[7]).any() and not torch.isfinite(logits[9]).any()


@pytest.mark.parametrize("zt", [F32, BF16])
def test_strides_alignment_and_no_writes_beside(zt):
    B, V = 19, 777
    logits, hidden, down, up, which, scales = _inputs(B, 3, 16, V, 128, F32, zt, pad=20)
    room = torch.full((B, 1001), 5.0, dtype=zt, device=DEV)
    got = room[:, 3:3 + V]                                 # aligned to an element only
    got.copy_(logits)
    need = sip.sip_head_adapt_workspace_bytes(B, 3, 16, 128)
    ws = torch.full((need + 256,), 0x33, dtype=torch.uint8, device=DEV)
    sip.sip_head_adapt(got, hidden, down, up, which, scales, workspace=ws[:need])
    _check(got.contiguous(), logits, hidden, down, up, which, scales)
    assert (room[:, :3] == 5.0).all() and (room[:, 3 + V:] == 5.0).all() and (ws[need:] == 0x33).all()


def test_many_adapters_and_rows():
    logits, hidden, down, up, which, scales = _inputs(3000, 1500, 8, 40, 16, BF16, F32)
    got = logits.clone()
    sip.sip_head_adapt(got, hidden, down, up, which, scales)
    ok = which >= 0
    a = which.long().clamp(min=0)
    t = torch.bmm(down[a].double(), hidden.double()[:, :, None].contiguous())
    add = torch.bmm(up[a].double(), t)[:, :, 0] * scales.double()[a][:, None]
    want = torch.where(ok[:, None], logits.double() + add, logits.double())
    assert (got.double() - want).abs().max() <= 1e-4       # (a row or adapter that is another's is off by 1)
    _check(got[:40], logits[:40], hidden[:40], down, up, which[:40], scales)


def test_adapters_beyond_32_bits():
    """An adapter that starts past 2^31 bytes of the stack."""
    A, r, V, D = 9, 128, 200000, 64
    up = torch.empty(A, V, r, dtype=BF16, device=DEV)
    g = torch.Generator(device=DEV).manual_seed(3)
    up[-1] = torch.randn(V, r, generator=g, device=DEV).to(BF16)
    down = torch.randn(A, r, D, generator=g, device=DEV).to(BF16)
    hidden = torch.randn(2, D, generator=g, device=DEV).to(BF16)
    which = torch.tensor([A - 1, -1], dtype=torch.int32, device=DEV)
    logits = torch.randn(2, V, generator=g, device=DEV)
    got = logits.clone()
    sip.sip_head_adapt(got, hidden, down, up, which)
    _check(got, logits, hidden, down, up, which)


def test_a_workspace_serves_fewer_rows():
    for A, r, D in ((1, 8, 8), (32, 64, 4096), (4096, 128, 16384)):
        sizes = [sip.sip_head_adapt_workspace_bytes(B, A, r, D) for B in list(range(1, 400)) + [1000, 4096, 65536]]
        assert sizes == sorted(sizes)


def test_the_same_bits_every_time_and_in_a_graph():
    logits, hidden, down, up, which, scales = _inputs(37, 5, 32, 6000, 512, BF16, F32)
    want = sip.sip_head_adapt(logits.clone(), hidden, down, up, which, scales)
    got = logits.clone()
    ws = torch.empty(sip.sip_head_adapt_workspace_bytes(37, 5, 32, 512), dtype=torch.uint8, device=DEV)
    side, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    sip.sip_init()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph, stream=side):
        sip.sip_head_adapt(got, hidden, down, up, which, scales, workspace=ws)
    for turn in range(4):
        got.copy_(logits)
        ws.fill_(turn * 37)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(got, want)
        assert torch.equal(sip.sip_head_adapt(logits.clone(), hidden, down, up, which, scales), want)


def test_refusals():
    logits, hidden, down, up, which, scales = _inputs(6, 2, 16, 100, 64, BF16, F32)
    for bad in (lambda: sip.sip_head_adapt(logits.half(), hidden, down, up, which), lambda: sip.sip_head_adapt(logits, hidden[:5], down, up, which),
                lambda: sip.sip_head_adapt(logits, hidden, down.float(), up, which), lambda: sip.sip_head_adapt(logits, hidden, down, up[:, :99], which),
                lambda: sip.sip_head_adapt(logits, hidden, down[:1], up, which), lambda: sip.sip_head_adapt(logits, hidden, down, up, which.long()),
                lambda: sip.sip_head_adapt(logits, hidden, down, up, which, scales[:1]), lambda: sip.sip_head_adapt(logits, hidden, down[0], up, which)):
        with pytest.raises(TypeError):
            bad()
    with pytest.raises(sip.SipError):
        sip.sip_head_adapt(logits, hidden, down[:, :12].contiguous(), up[:, :, :12].contiguous(), which)
    with pytest.raises(sip.SipError):
        sip.sip_head_adapt(logits, hidden, down, up, which, workspace=torch.empty(16, dtype=torch.uint8, device=DEV))
