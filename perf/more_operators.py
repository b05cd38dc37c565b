"""More operators whose speed this repository answers for: those on the way from hidden states to tokens and back.

A case is one pass through an operator as a program that searches with beams, serves adapters or trains an embedding makes
it: ``beam`` (the best continuations of every group of beams), ``reorder`` (the sampler state's slots take their parents'
histories), ``embed`` (rows of the embedding, or of a tied 4-bit head, by token), ``embed_grad`` (the embedding's gradient) and
``adapt`` (every request's own low-rank addition to its logits).  Vocabularies are those of ``workloads/`` and of the tests,
widths are generic.
"""
from __future__ import annotations

import math

import numpy as np
import torch

own = False                                            # True: through the library's entry points

DEV = "cuda:0"
INF = math.inf


def _case(op, name, **kw):
    c = {"op": op}
    if name:
        c["name"] = name
    c.update(kw)
    return c


def listed():
    return [
        # one request, four beams, a small vocabulary: the smallest call, latency only
        _case("beam", "beam_one", groups=1, width=4, V=32000, n=4, dtype="f32", finished=0.0, normalised=False, first=False),
        # a full batch of requests of four beams, twice as many candidates as beams, some of them finished
        _case("beam", "beam_batch", groups=64, width=4, V=152064, n=8, dtype="f32", finished=0.1, normalised=True, first=False),
        # few requests of many beams, a vocabulary that is not a round number, 16 bits
        _case("beam", "beam_wide", groups=7, width=32, V=151643, n=64, dtype="bf16", finished=0.0, normalised=False, first=False),
        # the histories of one request's beams
        _case("reorder", "reorder_one", groups=1, width=4, L_max=512),
        # those of a full batch, long ones
        _case("reorder", "reorder_batch", groups=64, width=8, L_max=4096),
        # the tokens of a decode step, from the codes of a tied 4-bit head
        _case("embed", "embed_step", N=32, V=128256, D=4096, source="codes", group=128, zeros=True, out="bf16", masked=0.0, zipf=1.0),
        # a batch of prompts, padded
        _case("embed", "embed_prompt", N=16000, V=128256, D=4096, source="bf16", group=0, zeros=False, out="bf16", masked=0.1,
              zipf=1.0),
        # a training step of a small model with a small vocabulary
        _case("embed_grad", "grad_small", N=384, V=4096, D=512, grad="f32", out="f32", add=False, masked=0.0, zipf=1.0),
        # a training step on 8192 tokens, added to the gradient of the head that shares the matrix
        _case("embed_grad", "grad_tied", N=8192, V=128256, D=4096, grad="bf16", out="bf16", add=True, masked=0.1, zipf=1.0),
        # the most tokens, a gradient in 32 bits
        _case("embed_grad", "grad_long", N=65536, V=151643, D=2048, grad="bf16", out="f32", add=False, masked=0.0, zipf=1.1),
        # one interactive user with an adapter
        _case("adapt", "adapt_one", B=1, adapters=8, rank=16, V=128256, D=4096, hidden="bf16", logits="f32", plain=0.0),
        # a full decode batch, every eighth row without an adapter
        _case("adapt", "adapt_batch", B=256, adapters=32, rank=64, V=128256, D=4096, hidden="bf16", logits="f32", plain=0.125),
    ]


MOST_ROWS_V = 256 * 152064                             # of the largest listed cases
MOST_VD = 128256 * 4096
MOST_ND = 65536 * 2048
MOST_UP = 32 * 128256 * 64


def draw(rng):
    """One more case: 1 to 1024 beams in groups of 1 to 64 over vocabularies from 1000 to 2^18 entries, states of up to 1024
    slots, 1 to 65536 tokens, widths from 64 to 8192, ranks from 8 to 128 of up to 64 adapters, every type and option."""
    def log(lo, hi, unit=1):
        return max(unit, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi))))) // unit * unit)

    op = rng.choice(["beam", "beam", "reorder", "embed", "embed_grad", "embed_grad", "adapt"])
    V = log(1000, 262144)
    if op == "beam":
        width = log(1, 64)
        groups = log(1, max(1, min(1024, MOST_ROWS_V // V) // width))
        return _case(op, "", groups=groups, width=width, V=V, n=rng.choice([width, 2 * width, rng.randint(1, 2 * width)]),
                     dtype=rng.choice(["bf16", "f32"]), finished=rng.choice([0.0, 0.0, rng.uniform(0.05, 0.9)]),
                     normalised=rng.random() < 0.4, first=rng.random() < 0.2)
    if op == "reorder":
        width = log(1, 64)
        return _case(op, "", groups=log(1, max(1, 512 // width)), width=width, L_max=log(16, 4096))
    zipf = rng.choice([0.0, 1.0, 1.2])
    masked = rng.choice([0.0, 0.0, rng.uniform(0.05, 0.95)])
    if op == "embed":
        source = rng.choice(["bf16", "bf16", "f32", "codes"])
        group = rng.choice([32, 64, 128]) if source == "codes" else 0
        D = log(64, min(8192, MOST_VD // V), max(group, 8))
        return _case(op, "", N=log(1, min(65536, MOST_ND // 2 // D)), V=V, D=D, source=source, group=group,
                     zeros=rng.random() < 0.5, out=rng.choice(["bf16", "bf16", "f32"]), masked=masked, zipf=zipf)
    if op == "embed_grad":
        D = log(64, min(8192, MOST_VD // 2 // V), 8)
        return _case(op, "", N=log(1, min(65536, MOST_ND // 2 // D)), V=V, D=D, grad=rng.choice(["bf16", "bf16", "f32"]),
                     out=rng.choice(["bf16", "f32"]), add=rng.random() < 0.5, masked=masked, zipf=zipf)
    D = log(64, 8192, 8)
    rank = log(8, 128, 8)
    adapters = log(1, max(1, min(64, MOST_UP // (V * rank))))
    return _case(op, "", B=log(1, 256), adapters=adapters, rank=rank, V=V, D=D, hidden=rng.choice(["bf16", "bf16", "f32"]),
                 logits=rng.choice(["bf16", "f32"]), plain=rng.choice([0.0, rng.uniform(0.05, 0.95)]))


# ---------------------------------------------------------------- inputs

_DTYPE = {"bf16": torch.bfloat16, "f32": torch.float32}
TABLE = 4096                                           # entries of a slot's table of multiplicities, in buckets of four


def _gen(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    return g


def _normal(g, n, m, scale, dtype):
    """[n, m] normal values, drawn a piece at a time."""
    out = torch.empty(n, m, dtype=dtype, device=DEV)
    step = max(1, (1 << 27) // m)
    for i in range(0, n, step):
        out[i:i + step] = torch.randn(min(step, n - i), m, generator=g, device=DEV) * scale
    return out


def _share(V, a):
    """Probabilities of the vocabulary's entries by rank: r^-a."""
    p = np.arange(1, V + 1, dtype=np.float64) ** -a
    return p / p.sum()


def _tokens(g, n, V, a):
    """Token ids as text has them: a few that are everywhere, most of them rare, in no order."""
    if a == 0.0:
        return torch.randint(0, V, (n,), generator=g, device=DEV, dtype=torch.int32)
    cdf = torch.from_numpy(np.cumsum(_share(V, a))).to(DEV)
    rank = torch.searchsorted(cdf, torch.rand(n, generator=g, device=DEV, dtype=torch.float64)).clamp(max=V - 1)
    return torch.randperm(V, generator=g, device=DEV)[rank].to(torch.int32)


def _masked_tokens(g, case):
    t = _tokens(g, case["N"], case["V"], case["zipf"])
    return torch.where(torch.rand(case["N"], generator=g, device=DEV) < case["masked"], -1, t).to(torch.int32)


def _round_256(n):
    return (n + 255) // 256 * 256


def _state_views(state, slots, L_max):
    """(length, distinct, tokens, keys, counts) of a sampler state's buffer, by the layout that include/sip.h documents."""
    def view(at, *shape):
        return state[at:at + 4 * math.prod(shape)].view(torch.int32).view(*shape)
    row = _round_256(4 * slots)
    table = view(256 + 2 * row + _round_256(4 * slots * L_max), slots, 2, TABLE)
    return view(256, slots), view(256 + row, slots), view(256 + 2 * row, slots, L_max), table[:, 0], table[:, 1]


def _home(token):
    return ((token.long() * 0x9E3779B1) & 0xFFFFFFFF) >> 22


def _fill_tables(length, distinct, tokens, keys, counts):
    """The tables of the histories: every distinct token in the first bucket from its home on that has room for it."""
    slots, L = tokens.shape
    live = torch.arange(L, device=DEV) < length[:, None]
    pair = (torch.arange(slots, device=DEV)[:, None] << 32 | tokens.long())[live]
    pair, n = torch.unique(pair, return_counts=True)
    slot, token = pair >> 32, pair & 0xFFFFFFFF
    distinct.copy_(torch.bincount(slot, minlength=slots))
    keys.fill_(-1)
    counts.zero_()
    bucket = _home(token)
    used = torch.zeros(slots * (TABLE // 4), dtype=torch.int64, device=DEV)
    while slot.numel():
        at = slot * (TABLE // 4) + bucket
        order = torch.sort(at, stable=True).indices
        at, slot, token, n, bucket = at[order], slot[order], token[order], n[order], bucket[order]
        here = torch.arange(at.numel(), device=DEV)
        first = torch.searchsorted(at, at)             # of those that come to the same bucket
        place = used[at] + here - first
        fits = place < 4
        keys[slot[fits], bucket[fits] * 4 + place[fits]] = token[fits].to(torch.int32)
        counts[slot[fits], bucket[fits] * 4 + place[fits]] = n[fits].to(torch.int32)
        used += torch.bincount(at[fits], minlength=used.numel())
        slot, token, n, bucket = slot[~fits], token[~fits], n[~fits], (bucket[~fits] + 1) % (TABLE // 4)


def prepare(case, seed):
    g = _gen(seed)
    s = {"case": case}
    if own:
        import paper_2506_22033_amd as sip
    scratch = lambda n: torch.empty(max(n, 256), dtype=torch.uint8, device=DEV)          # noqa: E731
    if case["op"] == "beam":
        G, K, V, n = case["groups"], case["width"], case["V"], case["n"]
        stride = (V + 7) // 8 * 8                      # rows that the sampler takes: whole 16-byte groups
        s["logits"] = _normal(g, G * K, stride, 2.5, _DTYPE[case["dtype"]])[:, :V]
        # beams of one request lie within a few nats of one another, requests anywhere
        base, each = torch.rand(G, 1, generator=g, device=DEV) * 60.0, torch.rand(G, K, generator=g, device=DEV) * 3.0
        score = -(base + each)
        if case["first"]:                              # before the first step there is one beam
            score[:, 1:] = -INF
        s["scores"] = score.reshape(-1).contiguous()
        s["finished"] = None
        if case["finished"] > 0.0:
            s["finished"] = (torch.rand(G * K, generator=g, device=DEV) < case["finished"]).to(torch.uint8)
        s["rank_scale"] = None
        if case["normalised"]:                         # 1 / length
            s["rank_scale"] = 1.0 / torch.randint(5, 200, (G * K,), generator=g, device=DEV).float()
        s["end_token"] = V // 3
        for name, dt in (("tokens", torch.int32), ("parents", torch.int32), ("out_scores", torch.float32)):
            s[name] = torch.empty(G, n, dtype=dt, device=DEV)
        if own:
            s["workspace"] = scratch(sip.sip_beam_workspace_bytes(G, K, V, n))
    elif case["op"] == "reorder":
        G, K, L = case["groups"], case["width"], case["L_max"]
        slots = G * K + 3
        s["slots"], row = slots, _round_256(4 * slots)
        s["state"] = torch.zeros(256 + 2 * row + _round_256(4 * slots * L) + slots * 2 * TABLE * 4, dtype=torch.uint8, device=DEV)
        s["views"] = _state_views(s["state"], slots, L)
        length, distinct, tokens, keys, counts = s["views"]
        # the beams of a request are about as long as one another; the last steps of a search
        long = torch.randint((L + 1) // 2, L + 1, (G,), generator=g, device=DEV, dtype=torch.int32).repeat_interleave(K)
        s["slot_of_row"] = torch.randperm(slots, generator=g, device=DEV)[:G * K].to(torch.int32)
        length[s["slot_of_row"].long()] = long
        tokens.copy_(_tokens(g, slots * L, 32000, 1.0).view(slots, L))
        _fill_tables(length, distinct, tokens, keys, counts)
        # the best beam has more children than the others, and the parents come in no order
        s["parents"] = (torch.rand(G * K, generator=g, device=DEV).square() * K).long().clamp(max=K - 1).to(torch.int32)
        s["tokens"] = _tokens(g, G * K, 32000, 1.0)
    elif case["op"] == "embed":
        V, D, N = case["V"], case["D"], case["N"]
        s["ids"] = _masked_tokens(g, case)
        s["scale"] = math.sqrt(D)
        if case["source"] == "codes":
            s["codes"] = torch.randint(0, 256, (V, D // 2), generator=g, device=DEV, dtype=torch.uint8)
            s["scales"] = (torch.rand(V, D // case["group"], generator=g, device=DEV) + 0.5).mul_(0.3 / math.sqrt(D)).bfloat16()
            s["zeros"] = torch.randint(5, 11, s["scales"].shape, generator=g, device=DEV,
                                       dtype=torch.uint8) if case["zeros"] else None
        else:
            s["weight"] = _normal(g, V, D, 1.0 / math.sqrt(D), _DTYPE[case["source"]])
        s["out"] = torch.empty(N, D, dtype=_DTYPE[case["out"]], device=DEV)
    elif case["op"] == "embed_grad":
        N, V, D = case["N"], case["V"], case["D"]
        s["ids"] = _masked_tokens(g, case)
        s["scale"] = math.sqrt(D)
        s["grad_out"] = _normal(g, N, D, 1e-3, _DTYPE[case["grad"]])
        s["grad_weight"] = _normal(g, V, D, 1e-2, _DTYPE[case["out"]])       # (what the head's gradient left there)
        if own:
            s["workspace"] = scratch(sip.sip_embed_workspace_bytes(N, V, D))
    else:
        B, A, r, V, D = case["B"], case["adapters"], case["rank"], case["V"], case["D"]
        s["hidden"] = _normal(g, B, D, 1.0, _DTYPE[case["hidden"]])
        s["down"] = _normal(g, A * r, D, 1.0 / math.sqrt(D), torch.bfloat16).view(A, r, D)
        s["up"] = _normal(g, A * V, r, 0.5 / math.sqrt(r), torch.bfloat16).view(A, V, r)
        s["scales"] = torch.rand(A, generator=g, device=DEV) + 0.5
        which = torch.randint(0, A, (B,), generator=g, device=DEV, dtype=torch.int32)
        s["adapter_of_row"] = torch.where(torch.rand(B, generator=g, device=DEV) < case["plain"], -1, which).to(torch.int32)
        stride = (V + 7) // 8 * 8
        s["logits"] = _normal(g, B, stride, 2.0, _DTYPE[case["logits"]])[:, :V]
        if own:
            s["workspace"] = scratch(sip.sip_head_adapt_workspace_bytes(B, A, r, D))
    return s


# ---------------------------------------------------------------- one pass

def run(s):
    if own:
        return _run_own(s)
    return {"beam": _plain_beam, "reorder": _plain_reorder, "embed": _plain_embed, "embed_grad": _plain_embed_grad,
            "adapt": _plain_adapt}[s["case"]["op"]](s)


def _run_own(s):
    import paper_2506_22033_amd as sip
    case = s["case"]
    if case["op"] == "beam":
        sip.sip_beam_select(s["logits"], s["scores"], case["width"], case["n"], finished=s["finished"], rank_scale=s["rank_scale"],
                            end_token=s["end_token"], tokens=s["tokens"], parents=s["parents"], out_scores=s["out_scores"],
                            workspace=s["workspace"])
        return {"tokens": s["tokens"], "parents": s["parents"], "scores": s["out_scores"]}
    if case["op"] == "reorder":
        sip.sip_state_reorder(s["state"], s["slots"], case["L_max"], s["slot_of_row"], s["parents"], case["width"], s["tokens"])
        return dict(zip(("length", "distinct", "tokens", "keys", "counts"), s["views"]))
    if case["op"] == "embed":
        if case["source"] == "codes":
            sip.sip_embed_codes(s["codes"], s["scales"], s["zeros"], s["ids"], s["scale"], out=s["out"])
        else:
            sip.sip_embed(s["weight"], s["ids"], s["scale"], out=s["out"])
        return {"out": s["out"]}
    if case["op"] == "embed_grad":
        sip.sip_embed_backward(s["grad_out"], s["ids"], case["V"], s["scale"], grad_weight=s["grad_weight"], accumulate=case["add"],
                               workspace=s["workspace"])
        return {"grad_weight": s["grad_weight"]}
    sip.sip_head_adapt(s["logits"], s["hidden"], s["down"], s["up"], s["adapter_of_row"], s["scales"], workspace=s["workspace"])
    return {"logits": s["logits"]}


def _plain_beam(s):
    """In 64 bits: two continuations may lie as near to one another as they like."""
    G, K, V, n = (s["case"][k] for k in ("groups", "width", "V", "n"))
    score, z32 = s["scores"].double(), s["logits"].float() + 0.0             # (+ 0.0: one zero)
    z = z32.double()
    top = z.amax(1, keepdim=True)
    lse = top + (z - top).exp_().sum(1, keepdim=True).log()
    # the n first of every row, by logit and then by token: whole numbers that order alike
    bits = z32.view(torch.int32).long()
    order = torch.where(bits < 0, -2147483648 - bits, bits)
    m = min(n, V)
    token = (V - 1) - (order * 1048576 + torch.arange(V - 1, -1, -1, device=DEV)).topk(m, dim=1).values % 1048576
    total = score[:, None] + (z.gather(1, token) - lse)
    total = torch.where(score[:, None] > -INF, total, -INF)
    if s["finished"] is not None:                      # one continuation, which costs nothing
        done = (s["finished"] != 0)[:, None]
        alone = (torch.arange(m, device=DEV) == 0)[None, :]
        total = torch.where(done, torch.where(alone, score[:, None], -INF), total)
        token = torch.where(done, s["end_token"], token)
    rank = total if s["rank_scale"] is None else total * s["rank_scale"].double()[:, None]
    rank, at = rank.view(G, K * m).sort(dim=1, descending=True, stable=True)
    at, rank = at[:, :n], rank[:, :n]
    live = rank > -INF
    pad = n - at.shape[1]                              # (fewer continuations than are asked for)
    out = {"tokens": torch.where(live, token.view(G, K * m).gather(1, at), -1).to(torch.int32),
           "parents": torch.where(live, at // m, -1).to(torch.int32),
           "scores": total.view(G, K * m).gather(1, at).float()}
    if pad:
        out = {k: torch.cat((v, v.new_full((G, pad), -INF if v.is_floating_point() else -1)), dim=1) for k, v in out.items()}
    return out


def _plain_reorder(s):
    K, L = s["case"]["width"], s["case"]["L_max"]
    length, distinct, tokens, keys, counts = s["views"]
    rows = torch.arange(s["slot_of_row"].numel(), device=DEV)
    to, parent = s["slot_of_row"].long(), rows // K * K + s["parents"].long()
    of = to[parent]
    n, d, key, count, t = length[of], distinct[of], keys[of], counts[of], s["tokens"]
    place = torch.arange(L, device=DEV)[None, :]
    new = torch.where(place < n[:, None], tokens[of], tokens[to])
    new = torch.where(place == n[:, None], t[:, None], new)
    # the table: the token's entry, or the first free one, in the buckets from its home on
    room = n < L
    step = (torch.arange(TABLE, device=DEV)[None, :] - 4 * _home(t)[:, None]) % TABLE
    here, free = key == t[:, None], key == -1
    entry = torch.where(here | free, step + TABLE * (~here), 3 * TABLE).argmin(dim=1)[:, None]
    fresh = ~here.any(dim=1)
    key.scatter_(1, entry, torch.where(room[:, None], t[:, None], key.gather(1, entry)))
    count.scatter_(1, entry, count.gather(1, entry) + room[:, None].int())
    length[to] = n + room.int()
    distinct[to] = d + (fresh & room).int()
    tokens[to], keys[to], counts[to] = new, key, count
    return dict(zip(("length", "distinct", "tokens", "keys", "counts"), s["views"]))


def _live(s):
    valid = (s["ids"] >= 0) & (s["ids"] < s["case"]["V"])
    return valid[:, None], s["ids"].long().clamp(0, s["case"]["V"] - 1)


def _plain_embed(s):
    valid, at = _live(s)
    if s["case"]["source"] == "codes":
        q = torch.stack((s["codes"][at] & 15, s["codes"][at] >> 4), dim=2).flatten(1).float().unflatten(1, (-1, s["case"]["group"]))
        zero = 8.0 if s["zeros"] is None else s["zeros"][at].float()[:, :, None]
        row = ((q - zero) * s["scales"][at].float()[:, :, None]).flatten(1)
    else:
        row = s["weight"][at].float()
    return {"out": torch.where(valid, row * s["scale"], 0.0).to(s["out"].dtype)}


def _plain_embed_grad(s):
    valid, at = _live(s)
    total = torch.zeros(s["grad_weight"].shape, dtype=torch.float32, device=DEV)
    total.index_add_(0, at, torch.where(valid, s["grad_out"].float(), 0.0))
    total *= s["scale"]
    if s["case"]["add"]:
        total += s["grad_weight"].float()
    s["grad_weight"].copy_(total)
    return {"grad_weight": s["grad_weight"]}


def _plain_adapt(s):
    """All adapters for all rows, those that are not a row's own as zeros."""
    A, r, D = s["down"].shape
    mine = s["adapter_of_row"][:, None] == torch.arange(A, device=DEV)[None, :]
    t = (s["hidden"].float() @ s["down"].float().reshape(A * r, D).t()).view(-1, A, r)
    t = torch.where(mine[:, :, None], t * s["scales"][None, :, None], 0.0).flatten(1)
    up = s["up"].float().transpose(1, 2).reshape(A * r, -1)
    s["logits"].copy_(s["logits"].float() + t @ up)
    return {"logits": s["logits"]}


# ---------------------------------------------------------------- what a pass cannot do without

_SIZE = {"bf16": 2, "f32": 4}


def _distinct(case):
    """How many different tokens there are, on average."""
    live = case["N"] * (1.0 - case["masked"])
    return float(-np.expm1(live * np.log1p(-np.minimum(_share(case["V"], case["zipf"]), 0.999999))).sum())


def work(case):
    """Every input read once, every output written once: histories and tables that change, rows of the embedding that are asked
    for, adapters that a row has."""
    if case["op"] == "beam":
        R, V = case["groups"] * case["width"], case["V"]
        live = (1 if case["first"] else case["width"]) * case["groups"] * (1.0 - case["finished"])
        return {"bytes": live * V * _SIZE[case["dtype"]] + 4 * R + 12 * case["groups"] * case["n"], "flops": 4 * live * V}
    if case["op"] == "reorder":
        K = case["width"]
        lower = (np.arange(K) / K) ** 0.5
        share = np.diff(np.append(lower, 1.0))         # of parent k
        moved = K - share.sum()                        # rows whose parent is another
        read = (1.0 - (1.0 - share) ** (K - 1)).sum()
        each = 3 * case["L_max"] + 8 * TABLE           # (of a history, three quarters of L_max tokens on average)
        return {"bytes": float(case["groups"] * ((moved + read) * each + K * 28)), "flops": 0}
    if case["op"] == "embed":
        D = case["D"]
        row = D * _SIZE[case["source"]] if case["group"] == 0 else D // 2 + D // case["group"] * (3 if case["zeros"] else 2)
        return {"bytes": _distinct(case) * row + case["N"] * (4 + D * _SIZE[case["out"]]), "flops": case["N"] * D}
    if case["op"] == "embed_grad":
        D, e = case["D"], _SIZE[case["out"]]
        rows = 2 * _distinct(case) if case["add"] else case["V"]
        live = case["N"] * (1.0 - case["masked"])
        return {"bytes": live * D * _SIZE[case["grad"]] + rows * D * e + 4 * case["N"], "flops": live * D}
    B, A, r, V, D = case["B"], case["adapters"], case["rank"], case["V"], case["D"]
    live = B * (1.0 - case["plain"])
    used = A * (1.0 - (1.0 - 1.0 / A) ** live)
    return {"bytes": 2 * used * r * (V + D) + live * (2 * V * _SIZE[case["logits"]] + D * _SIZE[case["hidden"]]),
            "flops": 2 * live * r * (V + D)}


# ---------------------------------------------------------------- the definitions in 64 bits

def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] == "beam":
        out = []
        for g in range(case["groups"]):
            rows = slice(g * case["width"], (g + 1) * case["width"])
            lp = torch.log_softmax(s["logits"][rows].double(), dim=1) + s["scores"][rows].double()[:, None]
            if s["finished"] is not None:
                done = s["finished"][rows].bool()
                lp[done] = -INF
                lp[done, s["end_token"]] = s["scores"][rows][done].double()
            rank = lp if s["rank_scale"] is None else lp * s["rank_scale"][rows].double()[:, None]
            best = rank.flatten().topk(min(case["n"], rank.numel()))
            row = lp.flatten()[best.indices]
            out.append(torch.cat((row, row.new_full((case["n"] - row.numel(),), -INF))))
        return {"tokens": None, "parents": None, "scores": torch.stack(out)}
    if case["op"] == "reorder":
        return None                                    # (whole numbers)
    if case["op"] == "adapt":
        z = s["logits"].double()
        for b, a in enumerate(s["adapter_of_row"].tolist()):
            if a >= 0:
                t = s["down"][a].double() @ s["hidden"][b].double()
                z[b] += s["up"][a].double() @ (t * s["scales"][a].double())
        return {"logits": z}
    ids = s["ids"].long()
    live = ((ids >= 0) & (ids < case["V"])).nonzero()[:, 0]
    if case["op"] == "embed":
        out = torch.zeros(case["N"], case["D"], dtype=torch.float64, device=DEV)
        v = ids[live]
        if case["source"] == "codes":
            G = case["group"]
            w = torch.empty(v.numel(), case["D"], dtype=torch.float64, device=DEV)
            w[:, 0::2], w[:, 1::2] = (s["codes"][v] & 15).double(), (s["codes"][v] >> 4).double()
            w -= 8.0 if s["zeros"] is None else s["zeros"][v].double().repeat_interleave(G, dim=1)
            w *= s["scales"][v].double().repeat_interleave(G, dim=1)
        else:
            w = s["weight"][v].double()
        out[live] = w * s["scale"]
        return {"out": out}
    total = torch.zeros(case["V"], case["D"], dtype=torch.float64, device=DEV)
    total.index_put_((ids[live],), s["grad_out"][live].double(), accumulate=True)
    total *= s["scale"]
    return {"grad_weight": total + s["grad_weight"].double() if case["add"] else total}
