"""The vocabulary head's binding: what it takes, what it refuses, and what its options mean."""
import pytest
import torch

import paper_2506_22033_amd as sip

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
BF16 = torch.bfloat16


def test_clipping_refuses_memory_that_the_device_cannot_reach():
    """Raised before anything is enqueued."""
    g = torch.ones(8, device=DEV)
    need = sip.sip_grad_clip_workspace_bytes(1)
    for kw in (dict(workspace=torch.empty(need, dtype=torch.uint8)), dict(norm=torch.empty(1)),
               dict(workspace=torch.empty(1, dtype=torch.uint8, device=DEV).expand(need))):
        with pytest.raises(TypeError):
            sip.sip_grad_clip([g], 0.5, **kw)
    assert (g == 1.0).all()


def test_a_workspace_is_contiguous_device_memory():
    h, w, t = torch.zeros(2, 64, dtype=BF16, device=DEV), torch.zeros(9, 64, dtype=BF16, device=DEV), torch.zeros(
        2, dtype=torch.int32, device=DEV)
    loss, lse = sip.sip_xent_forward(h, w, t)
    codes, scales, zeros = sip.sip_head_quantize(w, 64)
    for ws in (torch.empty(1 << 20, dtype=torch.uint8), torch.empty(1, dtype=torch.uint8, device=DEV).expand(1 << 20),
               torch.empty(1 << 21, dtype=torch.uint8, device=DEV)[::2]):
        for call in (lambda: sip.sip_xent_forward(h, w, t, workspace=ws),
                     lambda: sip.sip_xent_backward(h, w, t, loss, lse, workspace=ws),
                     lambda: sip.sip_head_logits(h, codes, scales, zeros, workspace=ws)):
            with pytest.raises(TypeError):
                call()


def test_zero_points_are_made_unless_both_outputs_are_there_without_them():
    w = (torch.randn(40, 128, generator=torch.Generator().manual_seed(0)) + 1.0).to(DEV, BF16)
    want = sip.sip_head_quantize(w, 64)
    assert want[2] is not None
    codes, scales, zeros = (torch.empty_like(x) for x in want)
    for kw in (dict(codes=codes), dict(scales=scales), dict(zeros=zeros), dict(codes=codes, zeros=zeros),
               dict(codes=codes, scales=scales, zeros=zeros)):
        got = sip.sip_head_quantize(w, 64, **kw)
        assert all(torch.equal(a, b) for a, b in zip(got, want)), kw.keys()
        for k, v in kw.items():
            assert got[("codes", "scales", "zeros").index(k)] is v
    plain = sip.sip_head_quantize(w, 64, use_zeros=False)
    assert plain[2] is None and not torch.equal(plain[0], want[0])
    for kw in (dict(codes=codes, scales=scales), dict(codes=codes, use_zeros=False), dict(scales=scales, use_zeros=False)):
        got = sip.sip_head_quantize(w, 64, **kw)
        assert got[2] is None and torch.equal(got[0], plain[0]) and torch.equal(got[1], plain[1])


def _single(t, pad):
    """The one row of `t` as a row of a matrix whose row stride is its width and `pad`; aligned to 16 bytes."""
    wide = torch.zeros(17, t.shape[1] + pad, dtype=t.dtype, device=DEV)
    wide[16, :t.shape[1]] = t[0]
    return wide[16:17, :t.shape[1]]


def test_the_stride_of_a_single_row_says_nothing():
    """One row of a matrix of an odd width."""
    g = torch.Generator().manual_seed(3)
    h, w = torch.randn(1, 64, generator=g).to(DEV, BF16), torch.randn(1, 64, generator=g).to(DEV, BF16)
    many = torch.randn(50, 64, generator=g).to(DEV, BF16)
    t = torch.zeros(1, dtype=torch.int32, device=DEV)
    for pad in (3, 4):
        for x, y in ((h, many), (h, w)):
            xs, ys = _single(x, pad), y if y.shape[0] > 1 else _single(y, pad)
            want = sip.sip_xent_forward(x, y, t)
            assert all(torch.equal(a, b) for a, b in zip(sip.sip_xent_forward(xs, ys, t), want))
            grads = sip.sip_xent_backward(x, y, t, *want)
            for a, b in zip(sip.sip_xent_backward(xs, ys, t, *want, grad_hidden=_single(h, pad)), grads):
                assert torch.equal(a, b)
        codes, scales, zeros = sip.sip_head_quantize(many, 32)
        assert torch.equal(sip.sip_head_logits(_single(h, pad), codes, scales, zeros), sip.sip_head_logits(h, codes, scales, zeros))
        one = sip.sip_head_quantize(w, 32)
        got = sip.sip_head_quantize(_single(w, pad), 32, codes=_single(one[0], pad))
        assert all(torch.equal(a, b) for a, b in zip(got, one))
        assert torch.equal(sip.sip_head_logits(h, _single(one[0], pad), *one[1:]), sip.sip_head_logits(h, *one))


def test_errors_name_the_call():
    h, w, t = torch.zeros(2, 12, dtype=BF16, device=DEV), torch.zeros(9, 12, dtype=BF16, device=DEV), torch.zeros(
        2, dtype=torch.int32, device=DEV)
    x = torch.zeros(2, device=DEV)
    with pytest.raises(sip.SipError, match="sip_xent_forward failed"):
        sip.sip_xent_forward(h, w, t)
    with pytest.raises(sip.SipError, match="sip_xent_backward failed"):
        sip.sip_xent_backward(h, w, t, x, x)
    with pytest.raises(sip.SipError, match="sip_grad_clip failed"):
        sip.sip_grad_clip([x], -1.0)
    with pytest.raises(sip.SipError, match="sip_head_quantize failed"):
        sip.sip_head_quantize(torch.zeros(4, 48, dtype=BF16, device=DEV), 16)
    with pytest.raises(sip.SipError, match="sip_head_logits failed"):
        sip.sip_head_logits(torch.zeros(2, 48, dtype=BF16, device=DEV), torch.zeros(4, 24, dtype=torch.uint8, device=DEV), torch.ones(4, 3, device=DEV))
    assert "sip_sample failed" in str(sip.SipError(1))


def test_the_tensors_device_is_the_current_one_during_a_call(monkeypatch):
    """With another device current, a device's default stream would be that other's.  (On one device: the current one is said to
    be another.)"""
    w = torch.ones(8, 64, dtype=BF16, device=DEV)
    want = sip.sip_head_quantize(w, 64)
    entered = []

    class Recorded(torch.cuda.device):
        def __enter__(self):
            entered.append(self.idx)
            return super().__enter__()

    monkeypatch.setattr(torch.cuda, "device", Recorded)
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 1)
    got = sip.sip_head_quantize(w, 64)
    monkeypatch.undo()
    assert entered == [w.device.index]
    sip.sip_head_quantize(w, 64)
    assert all(torch.equal(a, b) for a, b in zip(got, want))
