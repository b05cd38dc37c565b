"""The vocabulary head's operators whose speed this repository answers for.

A case is one pass through an operator as a program that trains or serves a model's vocabulary head makes it:
``score`` (log-probabilities of given tokens), ``train`` (loss and gradients), ``clip`` (global gradient norm and
clipping), ``quantise`` (4-bit codes with group scales from bf16 weights) and ``head`` (logits of a decode step from
4-bit weights).  Vocabularies are those of ``workloads/`` and of the tests, widths are generic.
"""
from __future__ import annotations

import math

import torch

own = False                                            # True: through the library's entry points

DEV = "cuda:0"
EPS = 1e-6                                             # beside the norm that a gradient is divided by


def _case(op, name, **kw):
    c = {"op": op}
    if name:
        c["name"] = name
    c.update(kw)
    return c


def listed():
    return [
        # the log-probability of one token, a small head: the smallest call, latency only
        _case("score", "score_one", N=1, V=32000, D=1024, masked=0.0, weighted=False),
        # scoring a long prompt, a vocabulary that is not a round number
        _case("score", "score_prompt", N=2000, V=151643, D=2048, masked=0.0, weighted=False),
        # a training step of a small model with a small vocabulary
        _case("train", "train_small", N=384, V=4096, D=512, masked=0.0, weighted=False),
        # sampled replies with an advantage per token, the prompts' tokens (a little over half) masked
        _case("train", "train_replies", N=2048, V=128256, D=2048, masked=0.55, weighted=True),
        # a training step on 8192 tokens
        _case("train", "train_large", N=8192, V=128256, D=4096, masked=0.0, weighted=False),
        # one interactive user
        _case("head", "head_one", B=1, V=128256, D=4096, group=128, zeros=False, hidden="bf16", logits="bf16",
              scales="bf16"),
        # a few users, odd sizes, 32 bits in and out
        _case("head", "head_odd", B=7, V=151643, D=2080, group=32, zeros=True, hidden="f32", logits="f32",
              scales="f32"),
        # a full decode batch
        _case("head", "head_batch", B=256, V=152064, D=4096, group=64, zeros=True, hidden="bf16", logits="f32",
              scales="bf16"),
        # the gradients of a small model, most of them vectors
        _case("clip", "clip_small", tensors=40, total=1000003, f32=0.5, clipped=True),
        # the gradients of a large one
        _case("clip", "clip_large", tensors=290, total=800000001, f32=0.2, clipped=True),
        # a small head
        _case("quantise", "quantise_small", V=4096, D=512, group=32, zeros=True, scales="f32"),
        # the largest vocabulary
        _case("quantise", "quantise_large", V=256000, D=4096, group=128, zeros=False, scales="bf16"),
    ]


MOST_NVD = 8192 * 128256 * 4096                        # of the largest listed case


def draw(rng):
    """One more case: 1 to 8192 tokens or 1 to 256 rows, vocabularies from 1000 to 2^18 entries, widths from 64 to
    8192, one to 400 tensors of a thousand to 8e8 elements together, every type and option."""
    def log(lo, hi, unit=1):
        n = max(unit, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi))))) // unit * unit)
        return n if n != 3072 else n + unit

    op = rng.choice(["score", "train", "train", "head", "head", "clip", "quantise"])
    V = log(1000, 262144)
    if op in ("score", "train"):
        D = log(64, 8192, 8)
        N = log(1, max(1, min(8192, MOST_NVD // (V * D))))
        return _case(op, "", N=N, V=V, D=D, masked=rng.choice([0.0, 0.0, rng.uniform(0.05, 0.95)]),
                     weighted=rng.random() < 0.5)
    group = rng.choice([32, 64, 128])
    D = log(64, 8192, group)
    if op == "head":
        return _case(op, "", B=log(1, 256), V=V, D=D, group=group, zeros=rng.random() < 0.5,
                     hidden=rng.choice(["bf16", "bf16", "f32"]), logits=rng.choice(["bf16", "f32"]),
                     scales=rng.choice(["bf16", "f32"]))
    if op == "clip":
        total = log(1000, 800000000)
        return _case(op, "", tensors=min(total, log(1, 400)), total=total, f32=rng.choice([0.0, 1.0, rng.random()]),
                     clipped=rng.random() < 0.75)
    return _case(op, "", V=V, D=D, group=group, zeros=rng.random() < 0.5, scales=rng.choice(["bf16", "f32"]))


# ---------------------------------------------------------------- inputs

_DTYPE = {"bf16": torch.bfloat16, "f32": torch.float32}


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


def prepare(case, seed):
    g = _gen(seed)
    s = {"case": case}
    if own:
        import paper_2506_22033_amd as sip
    scratch = lambda n: torch.empty(max(n, 256), dtype=torch.uint8, device=DEV)          # noqa: E731
    if case["op"] in ("score", "train"):
        N, V, D = case["N"], case["V"], case["D"]
        w = _normal(g, V, D, 1.3 / math.sqrt(D), torch.bfloat16)
        t = torch.randint(0, V, (N,), generator=g, device=DEV, dtype=torch.int32)
        h = torch.randn(N, D, generator=g, device=DEV)
        # a model that knows something: the token's logit stands out, by 10 on average and not always
        wt = w[t.long()].float()
        lift = 10.0 + 4.0 * torch.randn(N, 1, generator=g, device=DEV)
        s["hidden"] = (h + lift * wt / wt.square().sum(1, keepdim=True)).bfloat16()
        off = torch.rand(N, generator=g, device=DEV) < case["masked"]
        s["targets"] = torch.where(off, -100, t).to(torch.int32)
        s["weight"] = w
        s["grad_loss"] = torch.randn(N, generator=g, device=DEV) if case["weighted"] else None
        s["scale"] = 1.0 / N                           # the mean over the batch's tokens
        if own:
            s["workspace"] = scratch(sip.sip_xent_workspace_bytes(N, V, D, case["op"] == "train"))
        if case["op"] == "train":
            s["grad_hidden"], s["grad_weight"] = torch.empty_like(s["hidden"]), torch.empty_like(w)
    elif case["op"] == "head":
        B, V, D, G = case["B"], case["V"], case["D"], case["group"]
        s["hidden"] = _normal(g, B, D, 1.0, _DTYPE[case["hidden"]])
        s["codes"] = torch.randint(0, 256, (V, D // 2), generator=g, device=DEV, dtype=torch.uint8)
        s["scales"] = (torch.rand(V, D // G, generator=g, device=DEV) + 0.5).mul_(0.3 / math.sqrt(D)).to(
            _DTYPE[case["scales"]])
        s["zeros"] = torch.randint(5, 11, (V, D // G), generator=g, device=DEV,
                                   dtype=torch.uint8) if case["zeros"] else None
        stride = (V + 7) // 8 * 8                      # rows that the sampler takes: whole 16-byte groups
        s["logits"] = torch.empty(B, stride, dtype=_DTYPE[case["logits"]], device=DEV)[:, :V]
        if own:
            s["workspace"] = scratch(sip.sip_head_workspace_bytes(B, V, D, G))
    elif case["op"] == "clip":
        n, total = case["tensors"], case["total"]
        # sizes from vectors to matrices, cut from one buffer for each type, as a bucketed optimizer keeps them
        share = torch.rand(n, generator=torch.Generator().manual_seed(total), dtype=torch.float64).mul_(5.0).exp_()
        cuts = [0] + [int(x) for x in (share.cumsum(0) / share.sum() * total).round()]
        is_f32 = [(i * 0.618034) % 1.0 < case["f32"] for i in range(n)]
        s["flat"], s["out"], s["grads"], s["outs"] = {}, {}, [None] * n, [None] * n
        for name, dt in _DTYPE.items():
            mine = [i for i in range(n) if is_f32[i] == (name == "f32")]
            size = [cuts[i + 1] - cuts[i] for i in mine]
            s["flat"][name] = _normal(g, 1, sum(size), 0.01, dt)[0] if sum(size) else torch.empty(0, dtype=dt, device=DEV)
            s["out"][name] = torch.empty_like(s["flat"][name])
            for i, a, b in zip(mine, s["flat"][name].split(size), s["out"][name].split(size)):
                s["grads"][i], s["outs"][i] = a, b
        s["max_norm"] = 0.01 * math.sqrt(total) * (0.3 if case["clipped"] else 3.0)
        if own:
            s["table"] = sip.GradTable(s["grads"], s["outs"])
            s["workspace"] = scratch(sip.sip_grad_clip_workspace_bytes(n))
    else:
        V, D, G = case["V"], case["D"], case["group"]
        s["weight"] = _normal(g, V, D, 0.02, torch.bfloat16)
        s["codes"] = torch.empty(V, D // 2, dtype=torch.uint8, device=DEV)
        s["scales"] = torch.empty(V, D // G, dtype=_DTYPE[case["scales"]], device=DEV)
        s["zeros"] = torch.empty(V, D // G, dtype=torch.uint8, device=DEV) if case["zeros"] else None
    return s


# ---------------------------------------------------------------- one pass

def run(s):
    if own:
        return _run_own(s)
    return {"score": _plain_xent, "train": _plain_xent, "head": _plain_head, "clip": _plain_clip,
            "quantise": _plain_quantise}[s["case"]["op"]](s)


def _run_own(s):
    import paper_2506_22033_amd as sip
    op = s["case"]["op"]
    if op in ("score", "train"):
        loss, lse = sip.sip_xent_forward(s["hidden"], s["weight"], s["targets"], workspace=s["workspace"])
        if op == "score":
            return {"loss": loss, "lse": lse}
        sip.sip_xent_backward(s["hidden"], s["weight"], s["targets"], loss, lse, s["grad_loss"], s["scale"],
                              grad_hidden=s["grad_hidden"], grad_weight=s["grad_weight"], workspace=s["workspace"])
        return {"loss": loss, "grad_hidden": s["grad_hidden"], "grad_weight": s["grad_weight"]}
    if op == "head":
        sip.sip_head_logits(s["hidden"], s["codes"], s["scales"], s["zeros"], out=s["logits"],
                            workspace=s["workspace"])
        return {"logits": s["logits"]}
    if op == "clip":
        norm = sip.sip_grad_clip(s["table"], s["max_norm"], eps=EPS, workspace=s["workspace"])
        return {"norm": norm, "out": s["out"]}
    sip.sip_head_quantize(s["weight"], s["case"]["group"], codes=s["codes"], scales=s["scales"], zeros=s["zeros"])
    return {"codes": s["codes"], "scales": s["scales"], "zeros": s["zeros"]}


def _plain_xent(s):
    h, w, t = s["hidden"].float(), s["weight"].float(), s["targets"].long()
    valid = (t >= 0) & (t < w.shape[0])
    at = t.clamp(0, w.shape[0] - 1)[:, None]
    z = h @ w.t()
    zt = z.gather(1, at)
    # loss = ln(1 + sum over the others of exp(z - z_t)): exact for a token that is nearly certain too
    rest = z.scatter(1, at, -math.inf)
    top = rest.amax(1, keepdim=True)
    gap = top + (rest - top).exp_().sum(1, keepdim=True).log() - zt
    every = gap.clamp(min=0.0) + (-gap.abs()).exp().log1p()
    lse = zt + every
    zero = torch.zeros_like(lse)
    loss = torch.where(valid[:, None], every, zero)[:, 0]
    if s["case"]["op"] == "score":
        return {"loss": loss, "lse": torch.where(valid[:, None], lse, zero)[:, 0]}
    g = valid.float() * s["scale"]
    if s["grad_loss"] is not None:
        g = g * s["grad_loss"]
    p = z.sub_(lse).exp_()
    p.scatter_(1, at, torch.expm1(-every))     # p_t - 1
    p.mul_(g[:, None])
    return {"loss": loss, "grad_hidden": (p @ w).bfloat16(), "grad_weight": (p.t() @ h).bfloat16()}


def _unpacked(codes):
    """[V, D] of the codes: byte j holds entry 2 j in its low half and 2 j + 1 in its high half."""
    return torch.stack((codes & 15, codes >> 4), dim=2).flatten(1)


def _plain_head(s):
    G = s["case"]["group"]
    q = _unpacked(s["codes"]).float().unflatten(1, (-1, G))
    zero = 8.0 if s["zeros"] is None else s["zeros"].float()[:, :, None]
    w = ((q - zero) * s["scales"].float()[:, :, None]).flatten(1)
    return {"logits": (s["hidden"].float() @ w.t()).to(s["logits"].dtype)}


def _plain_clip(s):
    norm = torch.stack([t.float().square().sum() for t in s["grads"]]).sum().sqrt()
    factor = (s["max_norm"] / (norm + EPS)).clamp(max=1.0)
    return {"norm": norm, "out": {k: (v.float() * factor).to(v.dtype) for k, v in s["flat"].items()}}


def _plain_quantise(s):
    w = s["weight"].float().unflatten(1, (-1, s["case"]["group"]))
    if s["zeros"] is None:
        scale = w.abs().amax(2)
        scale = scale / torch.full_like(scale, 7.0)    # (torch multiplies by the reciprocal of a plain number)
    else:
        low = w.amin(2).clamp(max=0.0)
        scale = (w.amax(2).clamp(min=0.0) - low) / torch.full_like(low, 15.0)
    scale = scale.to(s["scales"].dtype).float()
    scale = torch.where(scale == 0.0, torch.ones_like(scale), scale)
    zero = torch.full_like(scale, 8.0) if s["zeros"] is None else (-low / scale).round().clamp(0.0, 15.0)
    q = ((w / scale[:, :, None]).round() + zero[:, :, None]).clamp(0.0, 15.0).to(torch.uint8).flatten(1)
    return {"codes": q[:, 0::2] | (q[:, 1::2] << 4), "scales": scale.to(s["scales"].dtype),
            "zeros": None if s["zeros"] is None else zero.to(torch.uint8)}


# ---------------------------------------------------------------- what a pass cannot do without

def work(case):
    """Every input read once, every output written once.  ``train``: logits, their gradient's two products."""
    if case["op"] in ("score", "train"):
        N, V, D = case["N"], case["V"], case["D"]
        live = N * (1.0 - case["masked"])
        train = case["op"] == "train"
        size = 2 * D * (live + V)
        return {"bytes": (2 if train else 1) * size + 12 * N, "flops": (6 if train else 2) * live * V * D}
    if case["op"] == "head":
        B, V, D, G = case["B"], case["V"], case["D"], case["group"]
        e = {"bf16": 2, "f32": 4}
        size = V * D // 2 + V * (D // G) * (e[case["scales"]] + (1 if case["zeros"] else 0))
        return {"bytes": size + B * D * e[case["hidden"]] + B * V * e[case["logits"]], "flops": 2 * B * V * D}
    if case["op"] == "clip":
        return {"bytes": 2 * case["total"] * (2 + 2 * case["f32"]) + 4, "flops": 3 * case["total"]}
    V, D, G = case["V"], case["D"], case["group"]
    size = 2 * V * D + V * D // 2 + V * (D // G) * ((4 if case["scales"] == "f32" else 2) + (1 if case["zeros"] else 0))
    return {"bytes": size, "flops": 5 * V * D}


# ---------------------------------------------------------------- the definitions in 64 bits

def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] in ("score", "train"):
        return _exact_xent(s)
    if case["op"] == "head":
        V, D, G = case["V"], case["D"], case["group"]
        x, out = s["hidden"].double(), []
        for v in range(0, V, 16384):
            c = s["codes"][v:v + 16384]
            w = torch.empty(c.shape[0], D, dtype=torch.float64, device=DEV)
            w[:, 0::2], w[:, 1::2] = (c & 15).double(), (c >> 4).double()
            w -= 8.0 if s["zeros"] is None else s["zeros"][v:v + 16384].double().repeat_interleave(G, dim=1)
            w *= s["scales"][v:v + 16384].double().repeat_interleave(G, dim=1)
            out.append(x @ w.t())
        return {"logits": torch.cat(out, dim=1)}
    if case["op"] == "clip":
        norm = math.sqrt(sum(float(t.double().square().sum()) for t in s["grads"]))
        factor = min(1.0, s["max_norm"] / (norm + EPS))
        return {"norm": torch.tensor(norm, dtype=torch.float64),
                "out": {k: v.double() * factor for k, v in s["flat"].items()}}
    G, out = case["group"], []
    for v in range(0, case["V"], 16384):
        w = s["weight"][v:v + 16384].double().reshape(-1, case["D"] // G, G)
        hi, lo = w.max(dim=2).values, w.min(dim=2).values
        out.append(torch.maximum(hi, -lo) / 7 if s["zeros"] is None else (hi.clamp(min=0) - lo.clamp(max=0)) / 15)
    return {"codes": None, "scales": torch.cat(out), "zeros": None}


def _exact_xent(s):
    case = s["case"]
    N, V, D = case["N"], case["V"], case["D"]
    rows = ((s["targets"] >= 0) & (s["targets"] < V)).nonzero()[:, 0]
    h, t = s["hidden"][rows].double(), s["targets"][rows].long()
    step = max(256, (1 << 28) // max(1, rows.numel()))
    lse = torch.full((rows.numel(),), -math.inf, dtype=torch.float64, device=DEV)
    for v in range(0, V, step):
        lse = torch.logaddexp(lse, torch.logsumexp(h @ s["weight"][v:v + step].double().t(), dim=1))
    target = (h * s["weight"][t].double()).sum(1)
    whole = lambda x: torch.zeros(N, *x.shape[1:], dtype=torch.float64, device=DEV).index_copy_(0, rows, x)  # noqa: E731
    if case["op"] == "score":
        return {"loss": whole(lse - target), "lse": whole(lse)}
    g = torch.full((rows.numel(), 1), s["scale"], dtype=torch.float64, device=DEV)
    if s["grad_loss"] is not None:
        g = g * s["grad_loss"][rows].double()[:, None]
    dh, dw = torch.zeros_like(h), torch.empty(V, D, dtype=torch.float64, device=DEV)
    for v in range(0, V, step):
        w = s["weight"][v:v + step].double()
        dz = (h @ w.t() - lse[:, None]).exp()
        mine = ((t >= v) & (t < v + w.shape[0])).nonzero()[:, 0]
        dz[mine, t[mine] - v] -= 1.0
        dz *= g
        dh += dz @ w
        dw[v:v + step] = dz.t() @ h
    return {"loss": whole(lse - target), "grad_hidden": whole(dh), "grad_weight": dw}
