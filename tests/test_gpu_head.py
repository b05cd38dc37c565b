"""The 4-bit head: its quantiser, and its product with hidden states, against the definitions."""
import math

import pytest
import torch

import paper_2506_22033_amd as sip

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
F32, BF16 = torch.float32, torch.bfloat16


def make(B, V, D, group, zeros, hidden=BF16, scales=BF16, seed=0, x_scale=1.0):
    g = torch.Generator(device=DEV).manual_seed(seed)
    x = (torch.randn(B, D, generator=g, device=DEV) * x_scale).to(hidden)
    codes = torch.randint(0, 256, (V, D // 2), generator=g, device=DEV, dtype=torch.uint8)
    s = ((torch.rand(V, D // group, generator=g, device=DEV) + 0.5) * 0.02).to(scales)
    z = torch.randint(0, 16, (V, D // group), generator=g, device=DEV, dtype=torch.uint8) if zeros else None
    return x, codes, s, z


def unpack(codes):
    return torch.stack((codes & 15, codes >> 4), dim=2).flatten(1)


def weights(codes, scales, zeros):
    group = codes.shape[1] * 2 // scales.shape[1]
    q = unpack(codes).double()
    z = 8.0 if zeros is None else zeros.double().repeat_interleave(group, 1)
    return (q - z) * scales.double().repeat_interleave(group, 1)


def check(x, codes, scales, zeros, dtype, out=None):
    got = sip.sip_head_logits(x, codes, scales, zeros, dtype=dtype, out=out)
    w = weights(codes, scales, zeros)
    want = x.double() @ w.t()
    # a group's sum runs over values of up to 16 + 15 in place of q - zero, and the zero point's share is taken off
    # after it: roundings of 2^-24 of the magnitudes 31 |x| s, sqrt(D) of them, four times allowed; then the result's own
    D = x.shape[1]
    group = D // scales.shape[1]
    terms = x.double().abs() @ (31.0 * scales.double().abs().repeat_interleave(group, 1)).t()
    allow = 4 * 2.0 ** -24 * math.sqrt(D) * terms + (2.0 ** -8 if dtype == BF16 else 2.0 ** -22) * want.abs() + 1e-30
    assert got.dtype == dtype and got.shape == want.shape
    assert ((got.double() - want).abs() <= allow).all(), float(((got.double() - want).abs() - allow).max())
    bits = 2.0 ** -8 if dtype == BF16 else 2e-6
    assert float((got.double() - want).norm()) <= bits * float(want.norm()) + 1e-30
    return got


@pytest.mark.parametrize("B,V,D,group", [
    (1, 1, 32, 32), (1, 17, 64, 64), (1, 1000, 128, 128), (2, 333, 96, 32), (3, 15, 160, 32), (5, 129, 1056, 32),
    (7, 1001, 2080, 32), (15, 64, 192, 64), (16, 4097, 256, 128), (17, 300, 384, 128), (31, 1023, 64, 32),
    (33, 511, 512, 64), (48, 200, 640, 128), (64, 777, 1024, 64), (65, 130, 128, 32), (100, 259, 320, 64),
    (129, 1000, 256, 32), (200, 515, 192, 64), (257, 300, 128, 128), (1, 5000, 8192, 128), (4, 2000, 16384, 64),
    (300, 33, 4096, 32)])
@pytest.mark.parametrize("zeros", [False, True])
def test_logits(B, V, D, group, zeros):
    for hidden in (BF16, F32):
        for dtype in (BF16, F32):
            for scales in (BF16, F32):
                check(*make(B, V, D, group, zeros, hidden, scales, seed=B + V + D), dtype)


def test_fp32_hidden_states_enter_with_all_their_bits():
    """One element of a hidden state, picked out by q - zero = 1 under a scale of 1.  The sums hold 25 x and 24 x, rounded
    to 24 bits each, so the difference is x to within 2^-24 (25 + 24) x; a state rounded to 8 or 16 bits would be off by up to
    2^-8 or 2^-16."""
    D = 64
    x = torch.zeros(9, D, device=DEV)
    x[:, 5] = torch.randn(9, generator=torch.Generator().manual_seed(1)).to(DEV) * torch.logspace(-20, 20, 9, device=DEV)
    q = torch.full((D, D), 8, dtype=torch.uint8, device=DEV)
    q[torch.arange(D), torch.arange(D)] = 9
    codes = q[:, 0::2] | (q[:, 1::2] << 4)
    got = sip.sip_head_logits(x, codes, torch.ones(D, D // 32, device=DEV))
    assert ((got - x).abs() <= 2.0 ** -18 * x[:, 5:6].abs()).all()


def test_extreme_codes_zeros_and_scales():
    for code in (0x00, 0xFF, 0x0F, 0xF0):
        for zero in (0, 15):
            x, codes, s, z = make(3, 40, 256, 64, True, seed=1)
            check(x, torch.full_like(codes, code), s, torch.full_like(z, zero), F32)
    x, codes, s, z = make(3, 40, 256, 64, True, scales=F32, seed=1)
    s[::3] = 0.0
    s[1::3] = -s[1::3]
    check(x, codes, s, z, F32)


def test_strides_of_hidden_codes_and_logits():
    B, V, D, group = 6, 203, 160, 32
    x, codes, s, z = make(B, V, D, group, True, seed=3)
    xs = torch.full((B, D + 24), 5.0, dtype=BF16, device=DEV)
    xs[:, :D] = x
    cs = torch.full((V, D // 2 + 48), 0x5A, dtype=torch.uint8, device=DEV)
    cs[:, :D // 2] = codes
    wide = torch.full((B, V + 13), 7.0, device=DEV)
    codes16 = cs.as_strided((V, D // 2), (D // 2 + 48, 1))
    got = check(xs[:, :D], codes16, s, z, F32, out=wide[:, :V])
    assert (wide[:, V:] == 7.0).all()
    assert torch.equal(got, sip.sip_head_logits(x, codes, s, z))


def test_rows_do_not_touch_each_other():
    """A row of NaN or infinities leaves the others' bits as they are."""
    for B in (5, 40, 130):
        x, codes, s, z = make(B, 300, 256, 64, True, seed=7)
        want = sip.sip_head_logits(x, codes, s, z)
        bad = x.clone()
        bad[2], bad[B - 1] = math.nan, math.inf
        got = sip.sip_head_logits(bad, codes, s, z)
        keep = [i for i in range(B) if i not in (2, B - 1)]
        assert torch.equal(got[keep], want[keep]) and got[2].isnan().all() and not got[B - 1].isfinite().any()


def test_default_output_feeds_the_sampler():
    x, codes, s, z = make(12, 1003, 128, 32, True, seed=2)
    logits = sip.sip_head_logits(x, codes, s, z)
    ids, _, lp = sip.sip_sample(logits, {"temperature": torch.zeros(12, device=DEV)}, None, None, 1, 0, 0)
    assert torch.equal(ids.long(), logits.argmax(1))
    want = logits.double().log_softmax(1).gather(1, ids.long()[:, None])
    assert ((lp.double() - want).abs() <= 1e-5).all()


def test_same_bits_on_every_call_and_on_another_stream():
    for B in (1, 20, 130):
        x, codes, s, z = make(B, 3001, 512, 64, True, seed=5)
        first = sip.sip_head_logits(x, codes, s, z)
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        for _ in range(3):
            with torch.cuda.stream(side):
                again = sip.sip_head_logits(x, codes, s, z)
            side.synchronize()
            assert torch.equal(first, again)


def test_outputs_and_workspace_stay_within_their_bounds():
    for B, V, D in ((1, 1001, 128), (37, 515, 256), (140, 130, 128)):
        x, codes, s, z = make(B, V, D, 32, True, hidden=F32, seed=2)
        need = sip.sip_head_workspace_bytes(B, V, D, 32)
        buf = torch.full((need + 1024,), 0xA5, dtype=torch.uint8, device=DEV)
        out = torch.full((B * V + 256,), 7.0, device=DEV)
        sip.sip_head_logits(x, codes, s, z, out=out[:B * V].view(B, V), workspace=buf[:need])
        assert (buf[need:] == 0xA5).all() and (out[B * V:] == 7.0).all()
        assert torch.equal(out[:B * V].view(B, V), sip.sip_head_logits(x, codes, s, z))


def test_recorded_in_a_graph():
    x, codes, s, z = make(9, 700, 256, 64, True, hidden=F32)
    out = torch.empty(9, 700, device=DEV)
    ws = torch.empty(sip.sip_head_workspace_bytes(9, 700, 256, 64), dtype=torch.uint8, device=DEV)
    sip.sip_head_logits(x, codes, s, z, out=out, workspace=ws)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        sip.sip_head_logits(x, codes, s, z, out=out, workspace=ws)
    for seed in range(3):
        x.copy_(torch.randn(9, 256, device=DEV, generator=torch.Generator(device=DEV).manual_seed(seed)))
        graph.replay()
        torch.cuda.synchronize()
        got = out.clone()
        assert torch.equal(got, sip.sip_head_logits(x, codes, s, z))


def test_logits_beyond_two_to_the_32_bytes():
    """1100 rows of 2^20 + 8 places in bf16: the last row starts beyond 2^31 bytes; codes of 2^32 bytes and more."""
    B, V, D = 1100, 1000, 64
    x, codes, s, z = make(B, V, D, 32, True, seed=5)
    out = torch.zeros(B, (1 << 21) + 8, dtype=BF16, device=DEV)
    sip.sip_head_logits(x, codes, s, z, out=out[:, :V])
    assert torch.equal(out[:, :V], sip.sip_head_logits(x, codes, s, z, dtype=BF16)) and not out[:, V:V + 64].any()
    V, D = (1 << 19), 16384
    codes = torch.zeros(V, D // 2, dtype=torch.uint8, device=DEV)
    codes[V - 1] = 0x99
    x = torch.ones(2, D, dtype=BF16, device=DEV)
    got = sip.sip_head_logits(x, codes, torch.ones(V, D // 128, device=DEV))
    assert (got[:, V - 1] == D).all() and (got[:, :V - 1] == -8.0 * D).all()


# ---- the quantiser

def quantized(weight, group, zeros, scales_dtype):
    """The definition, in fp32 as it says (divisors as tensors: by a number torch multiplies with the reciprocal)."""
    w = weight.float().unflatten(1, (-1, group))
    hi, lo = w.amax(2).clamp(min=0.0), w.amin(2).clamp(max=0.0)
    s = (hi - lo) / torch.full_like(lo, 15.0) if zeros else torch.maximum(hi, -lo) / torch.full_like(lo, 7.0)
    s = s.to(scales_dtype).float()
    s[s == 0] = 1.0
    z = (-lo / s).round().clamp(0.0, 15.0) if zeros else torch.full_like(s, 8.0)
    q = ((w / s[..., None]).round() + z[..., None]).clamp(0.0, 15.0).to(torch.uint8).flatten(1)
    return q[:, 0::2] | (q[:, 1::2] << 4), s.to(scales_dtype), z.to(torch.uint8) if zeros else None


@pytest.mark.parametrize("V,D,group", [(1, 32, 32), (3, 64, 64), (5, 128, 128), (257, 96, 32), (130, 2080, 32), (77, 1152, 128),
                                       (1000, 448, 64), (33, 16384, 128), (4000, 32, 32)])
@pytest.mark.parametrize("zeros", [False, True])
@pytest.mark.parametrize("scales", [BF16, F32])
def test_quantizer(V, D, group, zeros, scales):
    g = torch.Generator(device=DEV).manual_seed(V)
    w = (torch.randn(V, D, generator=g, device=DEV) * 0.02).bfloat16()
    w[0] = 0.0                                         # groups of zeros, of one sign, of one value
    if V > 4:
        w[1], w[2], w[3] = w[1].abs(), -w[2].abs(), 0.5
        w[4, ::7] = 3.0e38
    got = sip.sip_head_quantize(w, group, use_zeros=zeros, scales_dtype=scales)
    for a, b in zip(got, quantized(w, group, zeros, scales)):
        assert (a is None and b is None) or torch.equal(a, b)


def test_quantizer_on_strided_rows_and_back():
    w = (torch.randn(300, 256 + 40, device=DEV) * 0.02).bfloat16()[:, :256]
    codes, s, z = sip.sip_head_quantize(w, 64)
    want = quantized(w, 64, True, BF16)
    assert all(torch.equal(a, b) for a, b in zip((codes, s, z), want))
    # half a step for the rounding of a weight, half for the zero point's, the scale's rounding to bf16 over 15 steps
    step = s.double().repeat_interleave(64, 1)
    assert ((weights(codes, s, z) - w.double()).abs() <= step * (1.0 + 15 * 2.0 ** -8)).all()
    small = torch.full((4, 64), 1e-40, device=DEV).bfloat16()
    assert torch.equal(sip.sip_head_quantize(small, 32)[0], quantized(small, 32, True, BF16)[0])


def test_what_the_binding_refuses():
    x, codes, s, z = make(2, 16, 64, 32, True)
    for args in ((x.half(), codes, s, z), (x[:, :32], codes, s, z), (x, codes.to(torch.int8), s, z), (x, codes, s[:8], z),
                 (x, codes, s, z[:, :1]), (x.cpu(), codes, s, z), (x, codes, s.half(), z)):
        with pytest.raises(TypeError):
            sip.sip_head_logits(*args)
    with pytest.raises(sip.SipError):                  # a group of 16
        sip.sip_head_logits(x, codes, torch.ones(16, 4, device=DEV))
    with pytest.raises(TypeError):
        sip.sip_head_quantize(torch.zeros(4, 48, dtype=BF16, device=DEV), 32)
    with pytest.raises(TypeError):
        sip.sip_head_quantize(torch.zeros(4, 64, device=DEV), 32)


@pytest.mark.parametrize("B,V,D,group", [(40, 66000, 512, 64), (40, 65537, 96, 32), (200, 33001, 2048, 32), (300, 23000, 640, 128),
                                         (150, 33300, 1088, 64)])
@pytest.mark.parametrize("hidden", [BF16, F32])
def test_many_rows_over_many_tiles(B, V, D, group, hidden):
    for scales in (BF16, F32):
        check(*make(B, V, D, group, True, hidden, scales, seed=B), F32)


@pytest.mark.parametrize("B,V,D,group", [(2, 301, 512, 32), (40, 301, 512, 32), (70, 66000, 256, 32), (40, 130, 2048, 64), (40, 130, 160, 32)])
def test_scales_and_zeros_at_any_element(B, V, D, group):
    """Bases that are aligned to an element only give the bits that aligned ones do."""
    for dtype in (BF16, F32):
        x, codes, s, z = make(B, V, D, group, True, scales=dtype, seed=6)
        want = check(x, codes, s, z, F32)
        for by in (1, 2, 3):
            s_room = torch.full((s.numel() + 8,), math.nan, dtype=dtype, device=DEV)
            z_room = torch.full((z.numel() + 8,), 255, dtype=torch.uint8, device=DEV)
            s_there = s_room[by:by + s.numel()].view_as(s).copy_(s)
            z_there = z_room[by:by + z.numel()].view_as(z).copy_(z)
            assert torch.equal(sip.sip_head_logits(x, codes, s_there, z_there), want)


@pytest.mark.parametrize("exponent", [-100, -62, -50, 50, 62, 100])
def test_quantizer_far_from_one(exponent):
    """Quotients by scales at either end of fp32's range and around 2^+-60 are the division's, bit for bit."""
    g = torch.Generator(device=DEV).manual_seed(9)
    w = torch.ldexp(torch.randn(400, 512, generator=g, device=DEV), torch.tensor(exponent, device=DEV)).bfloat16()
    for group in (32, 64, 128):
        for zeros in (False, True):
            for scales in (BF16, F32):
                for a, b in zip(sip.sip_head_quantize(w, group, use_zeros=zeros, scales_dtype=scales), quantized(w, group, zeros, scales)):
                    assert (a is None and b is None) or torch.equal(a, b)
