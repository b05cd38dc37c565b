"""Host-side checks of include/sip_beam.h and of the adapters' and embedding's part of include/sip_head.h that need no GPU: the headers
are plain C, the bindings mirror them, and bad arguments are found before anything is enqueued."""
import os
import subprocess

import pytest

import paper_2506_22033_amd as sip
from paper_2506_22033_amd import beam, binding, head

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
INVALID, UNSUPPORTED, WORKSPACE = binding.SIP_ERR_INVALID_ARG, binding.SIP_ERR_UNSUPPORTED, binding.SIP_ERR_WORKSPACE


def test_header_is_c99_and_the_limits_are_the_binding_s(tmp_path):
    src, exe = tmp_path / "t.c", tmp_path / "t"
    src.write_text('#include "sip_beam.h"\n#include "sip_head.h"\n#include <stdio.h>\nint main(void) { printf("%d %d %d %d\\n", '
                   'SIP_MAX_BEAMS, SIP_MAX_CONTINUATIONS, SIP_MAX_RANK, SIP_MAX_ADAPTERS); return 0; }\n')
    subprocess.run(["gcc", "-std=c99", "-Wall", "-Wextra", "-Werror", "-pedantic", "-I", os.path.join(ROOT, "include"), "-o",
                    str(exe), str(src)], check=True, capture_output=True, text=True)
    got = [int(x) for x in subprocess.run([str(exe)], check=True, capture_output=True, text=True).stdout.split()]
    assert got == [sip.SIP_MAX_BEAMS, sip.SIP_MAX_CONTINUATIONS, sip.SIP_MAX_RANK, sip.SIP_MAX_ADAPTERS]


def test_every_function_of_the_header_has_a_signature():
    text = open(os.path.join(ROOT, "include", "sip_beam.h")).read()
    lib = beam._load()
    for name in beam._SIGNATURES:
        assert name + "(" in text and getattr(lib, name).argtypes is not None


def test_workspace_queries():
    assert sip.sip_beam_workspace_bytes(1, 1, 1, 1) > 0
    for bad in ((0, 1, 9, 1), (1, 0, 9, 1), (1, 1, 0, 1), (1, 1, 9, 0), (-1, 1, 9, 1), (1, sip.SIP_MAX_BEAMS + 1, 9, 1),
                (1, 1, sip.SIP_MAX_V + 1, 1), (1, 1, 9, sip.SIP_MAX_CONTINUATIONS + 1), (1 << 20, 2, 9, 1)):
        assert sip.sip_beam_workspace_bytes(*bad) == 0
    assert sip.sip_embed_workspace_bytes(0, 1, 8) > 0
    for bad in ((-1, 9, 8), (sip.SIP_MAX_TOKENS + 1, 9, 8), (9, 0, 8), (9, 9, 12), (9, 9, sip.SIP_MAX_D + 8), (9, sip.SIP_MAX_V + 1, 8)):
        assert sip.sip_embed_workspace_bytes(*bad) == 0
    assert sip.sip_head_adapt_workspace_bytes(1, 1, 8, 8) > 0
    for bad in ((0, 1, 8, 8), (1, 0, 8, 8), (1, 1, 12, 8), (1, 1, 8, 12), (1, 1, sip.SIP_MAX_RANK + 8, 8), (1, sip.SIP_MAX_ADAPTERS + 1, 8, 8),
                (sip.SIP_MAX_TOKENS + 1, 1, 8, 8)):
        assert sip.sip_head_adapt_workspace_bytes(*bad) == 0


def _select(**over):
    a = dict(logits=0x10000, groups=2, width=3, V=100, stride=104, dtype=0, scale=1.0, scores=0x20000, finished=None, end=5, rank=None, n=3,
             tokens=0x30000, parents=0x40000, out=0x50000, ws=0x100000, ws_bytes=1 << 24)
    a.update(over)
    return beam._load().sip_beam_select(a["logits"], a["groups"], a["width"], a["V"], a["stride"], a["dtype"], a["scale"], a["scores"],
                                        a["finished"], a["end"], a["rank"], a["n"], a["tokens"], a["parents"], a["out"], a["ws"],
                                        a["ws_bytes"], None)


@pytest.mark.parametrize("over,want", [
    (dict(logits=None), INVALID), (dict(scores=None), INVALID), (dict(tokens=None), INVALID), (dict(parents=None), INVALID),
    (dict(out=None), INVALID), (dict(groups=0), INVALID), (dict(width=0), INVALID), (dict(V=0), INVALID), (dict(n=0), INVALID),
    (dict(dtype=2), INVALID), (dict(stride=99), INVALID), (dict(stride=101), INVALID), (dict(stride=100, dtype=1), INVALID),
    (dict(logits=0x10004), INVALID), (dict(scale=0.0), INVALID), (dict(scale=-1.0), INVALID), (dict(scale=float("inf")), INVALID),
    (dict(scale=float("nan")), INVALID), (dict(scale=1e-31), INVALID), (dict(finished=0x60000, end=-1), INVALID),
    (dict(finished=0x60000, end=100), INVALID), (dict(width=sip.SIP_MAX_BEAMS + 1), UNSUPPORTED),
    (dict(n=sip.SIP_MAX_CONTINUATIONS + 1), UNSUPPORTED), (dict(V=sip.SIP_MAX_V + 1, stride=sip.SIP_MAX_V + 8), UNSUPPORTED),
    (dict(groups=1 << 20), UNSUPPORTED), (dict(stride=1 << 33), UNSUPPORTED), (dict(ws=None), WORKSPACE), (dict(ws=0x100040), WORKSPACE),
    (dict(ws_bytes=64), WORKSPACE)])
def test_select_refuses(over, want):
    assert _select(**over) == want


def _reorder(**over):
    a = dict(state=0x100000, bytes=sip.sip_state_bytes(8, 16), slots=8, L=16, groups=2, width=4, rows=0x20000, parents=0x30000, tokens=None)
    a.update(over)
    return beam._load().sip_state_reorder(a["state"], a["bytes"], a["slots"], a["L"], a["groups"], a["width"], a["rows"], a["parents"],
                                          a["tokens"], None)


@pytest.mark.parametrize("over,want", [
    (dict(slots=0), INVALID), (dict(L=0), INVALID), (dict(slots=sip.SIP_MAX_SLOTS + 1), INVALID), (dict(L=sip.SIP_MAX_L + 1), INVALID),
    (dict(groups=-1), INVALID), (dict(width=0), INVALID), (dict(rows=None), INVALID), (dict(parents=None), INVALID),
    (dict(width=65), UNSUPPORTED), (dict(groups=1 << 20), UNSUPPORTED), (dict(state=None), WORKSPACE), (dict(state=0x100010), WORKSPACE),
    (dict(bytes=sip.sip_state_bytes(8, 16) - 1), WORKSPACE), (dict(groups=0, rows=None, parents=None), binding.SIP_OK)])
def test_reorder_refuses(over, want):
    assert _reorder(**over) == want


def _embed(**over):
    a = dict(weight=0x10000, wt=1, V=10, D=64, stride=64, ids=0x20000, N=4, out=0x30000, os=64, ot=1)
    a.update(over)
    return head._load().sip_embed(a["weight"], a["wt"], a["V"], a["D"], a["stride"], a["ids"], a["N"], 1.0, a["out"], a["os"], a["ot"], None)


def _embed_codes(**over):
    a = dict(codes=0x10000, cs=32, scales=0x40000, st=1, zeros=None, group=32, V=10, D=64, ids=0x20000, N=4, out=0x30000, os=64, ot=1)
    a.update(over)
    return head._load().sip_embed_codes(a["codes"], a["cs"], a["scales"], a["st"], a["zeros"], a["group"], a["V"], a["D"], a["ids"], a["N"],
                                        1.0, a["out"], a["os"], a["ot"], None)


LOOKUP_BAD = [
    (dict(V=0), INVALID), (dict(D=0), INVALID), (dict(ids=None), INVALID), (dict(N=-1), INVALID), (dict(out=None), INVALID), (dict(os=56), INVALID),
    (dict(os=68), INVALID), (dict(out=0x30008), INVALID), (dict(ot=2), INVALID), (dict(V=sip.SIP_MAX_V + 1), UNSUPPORTED),
    (dict(N=(1 << 20) + 1), UNSUPPORTED), (dict(os=1 << 33), UNSUPPORTED), (dict(N=0, ids=None, out=None), binding.SIP_OK)]


@pytest.mark.parametrize("over,want", LOOKUP_BAD + [
    (dict(weight=None), INVALID), (dict(wt=-1), INVALID), (dict(stride=56), INVALID), (dict(stride=66), INVALID), (dict(weight=0x10002), INVALID),
    (dict(D=60), INVALID), (dict(stride=1 << 33), UNSUPPORTED)])
def test_lookup_refuses(over, want):
    assert _embed(**over) == want


@pytest.mark.parametrize("over,want", LOOKUP_BAD + [
    (dict(codes=None), INVALID), (dict(scales=None), INVALID), (dict(st=2), INVALID), (dict(group=0), INVALID), (dict(group=16), UNSUPPORTED),
    (dict(group=128), INVALID), (dict(cs=16), INVALID), (dict(cs=40), INVALID), (dict(codes=0x10008), INVALID), (dict(scales=0x40001), INVALID),
    (dict(scales=0x40002, st=0), INVALID), (dict(cs=1 << 33), UNSUPPORTED)])
def test_lookup_from_codes_refuses(over, want):
    assert _embed_codes(**over) == want


def _gradient(**over):
    a = dict(grad=0x10000, gs=64, gt=1, ids=0x20000, N=4, V=10, D=64, acc=0, gw=0x30000, ws_=64, wt=0, ws=0x100000, ws_bytes=1 << 24)
    a.update(over)
    return head._load().sip_embed_backward(a["grad"], a["gs"], a["gt"], a["ids"], a["N"], a["V"], a["D"], 1.0, a["acc"], a["gw"], a["ws_"],
                                           a["wt"], a["ws"], a["ws_bytes"], None)


@pytest.mark.parametrize("over,want", [
    (dict(grad=None), INVALID), (dict(gs=56), INVALID), (dict(gs=68), INVALID), (dict(grad=0x10004), INVALID), (dict(gt=2), INVALID),
    (dict(ids=None), INVALID), (dict(N=-1), INVALID), (dict(V=0), INVALID), (dict(D=0), INVALID), (dict(D=60), INVALID), (dict(gw=None), INVALID),
    (dict(gw=0x30008), INVALID), (dict(ws_=60), INVALID), (dict(ws_=66), INVALID), (dict(wt=3), INVALID), (dict(N=sip.SIP_MAX_TOKENS + 1), UNSUPPORTED),
    (dict(V=sip.SIP_MAX_V + 1), UNSUPPORTED), (dict(D=sip.SIP_MAX_D + 8, gs=sip.SIP_MAX_D + 8, ws_=sip.SIP_MAX_D + 8), UNSUPPORTED),
    (dict(gs=1 << 33), UNSUPPORTED), (dict(ws_=1 << 33), UNSUPPORTED), (dict(ws=None), WORKSPACE), (dict(ws=0x100001), WORKSPACE),
    (dict(ws_bytes=100), WORKSPACE), (dict(N=0, acc=1, ids=None, grad=None), binding.SIP_OK)])
def test_gradient_refuses(over, want):
    assert _gradient(**over) == want


def _adapt(**over):
    a = dict(hidden=0x10000, B=2, D=64, hs=64, ht=1, down=0x20000, up=0x30000, A=3, r=16, rows=0x40000, scales=None, V=10, logits=0x50000, ls=10, lt=0,
             ws=0x100000, ws_bytes=1 << 24)
    a.update(over)
    return head._load().sip_head_adapt(a["hidden"], a["B"], a["D"], a["hs"], a["ht"], a["down"], a["up"], a["A"], a["r"], a["rows"], a["scales"], a["V"],
                                       a["logits"], a["ls"], a["lt"], a["ws"], a["ws_bytes"], None)


@pytest.mark.parametrize("over,want", [
    (dict(hidden=None), INVALID), (dict(B=0), INVALID), (dict(D=0), INVALID), (dict(D=60, hs=64), INVALID), (dict(hs=56), INVALID), (dict(hs=68), INVALID),
    (dict(hidden=0x10008), INVALID), (dict(ht=2), INVALID), (dict(down=None), INVALID), (dict(up=None), INVALID), (dict(down=0x20008), INVALID),
    (dict(up=0x30002), INVALID), (dict(A=0), INVALID), (dict(r=0), INVALID), (dict(r=12), INVALID), (dict(rows=None), INVALID), (dict(V=0), INVALID),
    (dict(logits=None), INVALID), (dict(ls=9), INVALID), (dict(logits=0x50002), INVALID), (dict(lt=1, logits=0x50001), INVALID), (dict(lt=7), INVALID),
    (dict(B=sip.SIP_MAX_TOKENS + 1), UNSUPPORTED), (dict(A=sip.SIP_MAX_ADAPTERS + 1), UNSUPPORTED), (dict(r=sip.SIP_MAX_RANK + 8), UNSUPPORTED),
    (dict(V=sip.SIP_MAX_V + 1, ls=sip.SIP_MAX_V + 1), UNSUPPORTED), (dict(hs=1 << 33), UNSUPPORTED), (dict(ls=1 << 33), UNSUPPORTED),
    (dict(ws=None), WORKSPACE), (dict(ws=0x100080), WORKSPACE), (dict(ws_bytes=100), WORKSPACE)])
def test_adapt_refuses(over, want):
    assert _adapt(**over) == want
