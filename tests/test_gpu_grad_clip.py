"""Global gradient norm and clipping against 64 bits."""
import math

import pytest
import torch

import paper_2506_22033_amd as sip

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def make(sizes, seed=0, scale=0.01, offset=0):
    """Tensors of the given sizes, fp32 and bf16 in turn, cut from one buffer each that begins `offset` elements in."""
    g = torch.Generator(device=DEV).manual_seed(seed)
    out, kinds = [], (torch.float32, torch.bfloat16)
    for kind in kinds:
        mine = [n for i, n in enumerate(sizes) if kinds[i % 2] == kind]
        flat = (torch.randn(sum(mine) + offset, generator=g, device=DEV) * scale).to(kind)[offset:]
        out.append(list(flat.split(mine)) if mine else [])
    return [out[i % 2][i // 2] for i in range(len(sizes))]


def check(grads, max_norm, eps=1e-6, in_place=False):
    norm64 = math.sqrt(sum(float(t.double().square().sum()) for t in grads))
    f = min(1.0, max_norm / (norm64 + eps))
    want = [t.double() * f for t in grads]
    outs = grads if in_place else [torch.full_like(t, 7.0) for t in grads]
    norm = sip.sip_grad_clip(sip.GradTable(grads, outs), max_norm, eps=eps)
    # fp64 sums: the norm is off by its rounding to fp32; the factor by a few of those, the product by one more and, for
    # bf16, by the result's
    assert abs(float(norm) - norm64) <= 2.0 ** -23 * norm64 + 1e-30
    for o, w in zip(outs, want):
        bits = 2.0 ** -8 if o.dtype == torch.bfloat16 else 0.0
        assert ((o.double() - w).abs() <= (2.0 ** -20 + bits) * w.abs() + 1e-38).all()
    return outs


@pytest.mark.parametrize("sizes", [[1], [0, 3], [7, 0, 9], [8192, 8193], [100003], [5, 65536, 17, 131073, 1, 1, 40000],
                                   [3] * 500, [1 + 13 * i for i in range(130)], [0, 0]])
@pytest.mark.parametrize("offset", [0, 1, 3])
def test_norm_and_clipped_values(sizes, offset):
    grads = make(sizes, seed=len(sizes), offset=offset)
    total = math.sqrt(sum(sizes)) * 0.01
    check(grads, 0.25 * total + 1e-4)
    check(grads, 4.0 * total + 1.0)
    check(grads, 0.25 * total + 1e-4, in_place=True)


def test_outputs_of_another_alignment():
    for shift in range(8):
        g = make([5000], seed=1)[0]
        o = torch.full((5016,), 7.0, device=DEV)
        out = o[shift:shift + 5000]
        norm = sip.sip_grad_clip(sip.GradTable([g], [out]), 0.1)
        assert torch.allclose(out, g * (0.1 / (norm + 1e-6)), rtol=1e-6, atol=0)
        assert (o[:shift] == 7.0).all() and (o[shift + 5000:] == 7.0).all()
        b = g.bfloat16()
        o = torch.full((5016,), 7.0, dtype=torch.bfloat16, device=DEV)
        sip.sip_grad_clip(sip.GradTable([b], [o[shift:shift + 5000]]), math.inf)
        assert torch.equal(o[shift:shift + 5000], b) and (o[:shift] == 7.0).all() and (o[shift + 5000:] == 7.0).all()


def test_no_tensors_and_no_elements():
    assert float(sip.sip_grad_clip([], 1.0)) == 0.0
    assert float(sip.sip_grad_clip([torch.empty(0, device=DEV)], 1.0)) == 0.0


def test_a_norm_below_the_bound_changes_nothing():
    grads = make([1000, 777, 3], seed=4)
    keep = [t.clone() for t in grads]
    sip.sip_grad_clip(grads, 1e6)
    assert all(torch.equal(a, b) for a, b in zip(grads, keep))
    sip.sip_grad_clip(grads, math.inf)
    assert all(torch.equal(a, b) for a, b in zip(grads, keep))


def test_nan_and_infinite_norms():
    for bad in (math.nan, math.inf):
        grads = make([1000, 777], seed=5)
        grads[1][500] = bad
        norm = sip.sip_grad_clip(grads, 1.0)
        assert (norm.isnan() if bad != bad else norm.isinf())
        if bad != bad:
            assert all(t.isnan().all() for t in grads)
        else:
            assert not grads[0].any() and grads[1][500].isnan() and int(grads[1].isnan().sum()) == 1


def test_squares_that_leave_the_range_of_fp32():
    """2^70 and 2^-70 squared lie outside fp32; the norm does not."""
    for x in (2.0 ** 70, 2.0 ** -70):
        g = torch.full((10000,), x, device=DEV)
        norm = sip.sip_grad_clip([g], math.inf)
        assert abs(float(norm) / (100.0 * x) - 1.0) <= 2.0 ** -23


def test_same_bits_on_every_call_and_on_another_stream():
    grads = make([50001, 1023, 400000, 7], seed=9)
    outs = [torch.empty_like(t) for t in grads]
    table = sip.GradTable(grads, outs)
    first = sip.sip_grad_clip(table, 0.3).clone(), [t.clone() for t in outs]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    for _ in range(3):
        with torch.cuda.stream(side):
            norm = sip.sip_grad_clip(table, 0.3)
        side.synchronize()
        assert torch.equal(norm, first[0]) and all(torch.equal(a, b) for a, b in zip(outs, first[1]))


def test_recorded_in_a_graph():
    grads = make([3001, 500], seed=1)
    outs = [torch.empty_like(t) for t in grads]
    table, norm = sip.GradTable(grads, outs), torch.empty((), device=DEV)
    ws = torch.empty(sip.sip_grad_clip_workspace_bytes(2), dtype=torch.uint8, device=DEV)
    sip.sip_grad_clip(table, 0.1, norm=norm, workspace=ws)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        sip.sip_grad_clip(table, 0.1, norm=norm, workspace=ws)
    for seed in range(3):
        for t, x in zip(grads, make([3001, 500], seed=10 + seed)):
            t.copy_(x)
        graph.replay()
        torch.cuda.synchronize()
        got = norm.clone(), [o.clone() for o in outs]
        want = sip.sip_grad_clip(table, 0.1)
        assert torch.equal(got[0], want) and all(torch.equal(a, b) for a, b in zip(got[1], outs))


def test_workspace_stays_within_its_bounds():
    grads = make([7000, 123], seed=2)
    need = sip.sip_grad_clip_workspace_bytes(2)
    buf = torch.full((need + 1024,), 0xA5, dtype=torch.uint8, device=DEV)
    sip.sip_grad_clip(grads, 0.1, workspace=buf[:need])
    torch.cuda.synchronize()
    assert (buf[need:] == 0xA5).all()


def test_one_tensor_of_more_than_two_to_the_32_elements():
    n = 2 ** 32 + 12345
    g = torch.zeros(n, dtype=torch.bfloat16, device=DEV)
    g[5], g[n - 1], g[2 ** 31 + 7] = 3.0, 4.0, 12.0
    norm = sip.sip_grad_clip([g], 6.5, eps=0.0)
    assert float(norm) == 13.0 and float(g[5]) == 1.5 and float(g[n - 1]) == 2.0 and float(g[2 ** 31 + 7]) == 6.0


def test_what_the_binding_refuses():
    a = torch.zeros(8, device=DEV)
    for bad in (a.half(), a.cpu(), torch.zeros(4, 4, device=DEV).t()):
        with pytest.raises(TypeError):
            sip.GradTable([bad])
    for out in (a.bfloat16(), torch.zeros(9, device=DEV)):
        with pytest.raises(TypeError):
            sip.GradTable([a], [out])
    with pytest.raises(TypeError):
        sip.GradTable([a], [a, a])
    with pytest.raises(sip.SipError):
        sip.sip_grad_clip([a], -1.0)
    with pytest.raises(sip.SipError):
        sip.sip_grad_clip([a], math.nan)
