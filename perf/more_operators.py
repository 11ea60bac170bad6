"""Performance cases of the routing operators and of the low-rank adapters.

Routing: a layer's router gives every token one logit per expert.  Scores are
their softmax or sigmoid; a bias that balances the experts' load joins the
scores for the choice alone; experts stand in groups, of which the best few are
kept; the k best experts of those are taken, with their scores (renormalised or
not, times a factor) as weights (``moe.route_scores``; its gradient
``moe.route_scores_backward``).

Adapters: a batch holds rows of many requests, each with a low-rank adapter of
its own (or none) beside a projection that all share:
y = base + scale * (x A^T) B^T (``moe.adapter_rows``; its gradient
``moe.adapter_backward``).  Rows are ordered by adapter once per batch, as
``moe.permute`` orders tokens by expert.
"""
import math

import torch

own = False

_TYPE = {"bf16": torch.bfloat16, "f32": torch.float32}


def listed():
    return [
        # ---- routing
        # one sequence being decoded: sigmoid scores, bias, groups judged by their two best
        {"name": "route_decode_1", "op": "route", "tokens": 1, "experts": 256, "top_k": 8,
         "score": "sigmoid", "bias": True, "groups": 8, "top_groups": 4, "pair": True,
         "renorm": True, "scale": 2.5, "type": "f32", "masked": 0},
        # an odd prompt batch of the DeepSeekV2 share: softmax, groups judged by their best
        {"name": "route_dsv2_997", "op": "route", "tokens": 997, "experts": 160, "top_k": 6,
         "score": "softmax", "bias": False, "groups": 8, "top_groups": 3, "pair": False,
         "renorm": False, "scale": 16.0, "type": "f32", "masked": 0},
        # few experts, bf16 logits full of ties, one expert switched off
        {"name": "route_8_experts_4099", "op": "route", "tokens": 4099, "experts": 8, "top_k": 2,
         "score": "softmax", "bias": False, "groups": 1, "top_groups": 1, "pair": False,
         "renorm": True, "scale": 1.0, "type": "bf16", "masked": 1},
        # the largest prefill batch
        {"name": "route_prefill_65536", "op": "route", "tokens": 65536, "experts": 256,
         "top_k": 8, "score": "sigmoid", "bias": True, "groups": 8, "top_groups": 4,
         "pair": True, "renorm": True, "scale": 2.5, "type": "f32", "masked": 0},
        # ---- its gradient
        # softmax over all experts: every logit of a token gets a gradient
        {"name": "route_back_1501", "op": "route_back", "tokens": 1501, "experts": 160,
         "top_k": 6, "score": "softmax", "bias": False, "groups": 8, "top_groups": 3,
         "pair": False, "renorm": False, "scale": 16.0, "type": "bf16", "masked": 0},
        # a training step's tokens: sigmoid scores, gradients at the chosen experts only
        {"name": "route_back_65536", "op": "route_back", "tokens": 65536, "experts": 256,
         "top_k": 8, "score": "sigmoid", "bias": True, "groups": 8, "top_groups": 4,
         "pair": True, "renorm": True, "scale": 2.5, "type": "f32", "masked": 0},
        # ---- adapters
        # one token of one request: latency
        {"name": "adapter_decode_1", "op": "adapter", "rows": 1, "n": 4096, "k": 4096,
         "rank": 16, "count": 4, "alpha": 0.0, "none": 0.0, "base": True, "type": "bf16"},
        # a decode batch, a request a row, most adapters of the pool in use
        {"name": "adapter_decode_64", "op": "adapter", "rows": 64, "n": 1344, "k": 6144,
         "rank": 32, "count": 64, "alpha": 0.0, "none": 0.0, "base": True, "type": "bf16"},
        # prompts of a few requests, some without an adapter, beside an fp32 output
        {"name": "adapter_prompt_1501", "op": "adapter", "rows": 1501, "n": 6144, "k": 1344,
         "rank": 8, "count": 7, "alpha": 0.6, "none": 0.2, "base": True, "type": "f32"},
        # a prefill batch of long prompts
        {"name": "adapter_prefill_16384", "op": "adapter", "rows": 16384, "n": 4096, "k": 4096,
         "rank": 64, "count": 8, "alpha": 0.0, "none": 0.0, "base": True, "type": "bf16"},
        # ---- their gradient
        # a small step over a few adapters
        {"name": "adapter_back_997", "op": "adapter_back", "rows": 997, "n": 3584, "k": 4096,
         "rank": 16, "count": 5, "alpha": 0.6, "none": 0.1, "base": True, "type": "bf16"},
        # a fine-tuning step of two adapters trained side by side
        {"name": "adapter_back_8192", "op": "adapter_back", "rows": 8192, "n": 4096, "k": 4096,
         "rank": 32, "count": 2, "alpha": 0.0, "none": 0.0, "base": True, "type": "bf16"},
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi + 0.5)))))))


def draw(rng):
    op = rng.choice(["route", "route_back", "adapter", "adapter_back"])
    if op.startswith("route"):
        experts, groups, top_groups, top_k = rng.choice(
            [(8, 1, 1, 2), (16, 1, 1, 4), (60, 1, 1, 4), (64, 1, 1, 6), (96, 4, 2, 6),
             (128, 1, 1, 8), (160, 8, 3, 6), (161, 7, 3, 5), (200, 5, 2, 3), (256, 8, 4, 8),
             (256, 16, 1, 7), (256, 1, 1, 1)])
        score = rng.choice(["softmax", "sigmoid"])
        return {"op": op, "tokens": _log_int(rng, 1, 65536), "experts": experts, "top_k": top_k,
                "score": score, "bias": rng.random() < 0.6, "groups": groups,
                "top_groups": top_groups, "pair": groups > 1 and rng.random() < 0.5,
                "renorm": top_k > 1 and rng.random() < 0.6,
                "scale": rng.choice([1.0, 2.5, 16.0]), "type": rng.choice(["bf16", "f32"]),
                "masked": rng.choice([0, 0, 1, experts // 8])}
    return {"op": op, "rows": _log_int(rng, 1, 8192 if op == "adapter" else 4096),
            "n": 64 * _log_int(rng, 4, 64), "k": 64 * _log_int(rng, 4, 64),
            "rank": rng.choice([8, 16, 16, 24, 32, 32, 64]), "count": _log_int(rng, 1, 64),
            "alpha": rng.choice([0.0, 0.6, 1.0]), "none": rng.choice([0.0, 0.0, 0.3]),
            "base": rng.random() < 0.75, "type": rng.choice(["bf16", "f32"])}


# --------------------------------------------------------------------------
# inputs


def _logits(case, gen):
    """Logits whose experts differ in popularity; some experts switched off."""
    T, E = case["tokens"], case["experts"]
    z = torch.randn((T, E), generator=gen, device="cuda")
    z += 0.4 * torch.randn(E, generator=gen, device="cuda")
    if case["score"] == "sigmoid":
        z -= 1.0
    off = torch.randperm(E, generator=gen, device="cuda")[:case["masked"]]
    z[:, off] = -math.inf
    return z.to(_TYPE[case["type"]])


def _popularity(case):
    p = torch.arange(1, case["count"] + 1, dtype=torch.float64) ** -case["alpha"]
    return (1 - case["none"]) * p / p.sum()


def _dispatch(case, gen):
    """Rows ordered by (adapter, row), as moe.permute gives them for adapter
    ids (-1: none): offsets, row of each place, place of each row or -1."""
    R, C = case["rows"], case["count"]
    edge = _popularity(case).cumsum(0).cuda()
    u = torch.rand(R, generator=gen, device="cuda", dtype=torch.float64)
    ids = torch.searchsorted(edge, u, right=True)  # C: none
    order = torch.argsort(ids, stable=True)
    counts = torch.bincount(ids, minlength=C + 1)[:C]
    offsets = torch.zeros(C + 1, dtype=torch.int32, device="cuda")
    offsets[1:] = counts.cumsum(0).int()
    place = torch.empty(R, dtype=torch.int32, device="cuda")
    place[order] = torch.arange(R, dtype=torch.int32, device="cuda")
    place[ids == C] = -1
    return {"offsets": offsets, "sorted_slot": order.int().contiguous(), "slot_row": place,
            "most": max(1, int(counts.max()))}


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    st = {"case": case}

    def normal(*shape, size=1.0, dtype=torch.bfloat16):
        return (torch.randn(shape, generator=gen, device="cuda") * size).to(dtype)
    if case["op"].startswith("route"):
        T, E, k = case["tokens"], case["experts"], case["top_k"]
        st["logits"] = _logits(case, gen)
        st["bias"] = normal(E, size=0.1, dtype=torch.float32) if case["bias"] else None
        if case["op"] == "route":
            st["ids"] = torch.empty((T, k), dtype=torch.int32, device="cuda")
            st["w"] = torch.empty((T, k), dtype=torch.float32, device="cuda")
        else:
            st["ids"] = _choose(st)  # the forward pass' choice
            st["dw"] = normal(T, k, dtype=torch.float32)
            st["dlogits"] = torch.empty_like(st["logits"])
        return st
    st |= _dispatch(case, gen)
    R, N, K, r, C = (case[i] for i in ("rows", "n", "k", "rank", "count"))
    wide = _TYPE[case["type"]]
    st["x"] = normal(R, K)
    st["a"] = normal(C, r, K, size=K ** -0.5)
    st["b"] = normal(C, N, r, size=0.02)
    st["scale"] = 0.25 + 2 * torch.rand(C, generator=gen, device="cuda")
    if case["op"] == "adapter":
        st["base"] = normal(R, N, dtype=wide) if case["base"] else None
        st["y"] = torch.empty((R, N), dtype=wide, device="cuda")
    else:
        st["dy"] = normal(R, N, size=0.1)
        st["base"] = normal(R, K, size=0.1, dtype=wide) if case["base"] else None
        st["dx"] = torch.empty((R, K), dtype=wide, device="cuda")
        st["da"] = torch.empty((C, r, K), dtype=torch.float32, device="cuda")
        st["db"] = torch.empty((C, N, r), dtype=torch.float32, device="cuda")
    return st


# --------------------------------------------------------------------------
# the plain forms


def _scores(st, z):
    if st["case"]["score"] == "softmax":
        e = torch.exp(z - z.amax(-1, keepdim=True))
        return e / e.sum(-1, keepdim=True)
    return 1 / (1 + torch.exp(-z))


def _choose(st):
    """The chosen experts, in 64 bits: choices next to each other are common
    among many tokens.  Without a bias the scores' order is the logits'."""
    case, z = st["case"], st["logits"].double()
    c = _scores(st, z)
    if st["bias"] is not None:
        c = c + st["bias"].double()
    c = torch.where(z == -math.inf, z, c)  # switched off: never chosen
    order = z if st["bias"] is None else c
    if case["groups"] > 1:
        best = (c if case["pair"] else order).unflatten(-1, (case["groups"], -1))
        best = torch.sort(best, dim=-1, descending=True).values
        if case["pair"] and best.shape[-1] > 1:
            second = best[..., 1]
            best = best[..., 0] + torch.where(second == -math.inf, 0.0, second)
        else:
            best = best[..., 0]
        kept = torch.sort(best, dim=-1, descending=True, stable=True).indices[:, :case["top_groups"]]
        keep = torch.zeros_like(best, dtype=torch.bool).scatter_(1, kept, True)
        keep = keep.repeat_interleave(case["experts"] // case["groups"], -1)
        order = torch.where(keep, order, -math.inf)
    top = torch.sort(order, dim=-1, descending=True, stable=True)
    k = case["top_k"]
    return torch.where(top.values[:, :k] == -math.inf, -1, top.indices[:, :k]).int()


def _route_plain(st):
    case = st["case"]
    ids = _choose(st)
    s = _scores(st, st["logits"].double())
    w = s.gather(1, ids.clamp(min=0).long()) * (ids >= 0)
    if case["renorm"]:
        w = w / w.sum(-1, keepdim=True)
    return {"ids": ids, "w": (w * case["scale"]).float()}


def _route_back_plain(st):
    case, ids = st["case"], st["ids"]
    at = ids.clamp(min=0).long()
    g = st["dw"] * case["scale"] * (ids >= 0)
    s = _scores(st, st["logits"].float())
    chosen = s.gather(1, at) * (ids >= 0)
    if case["renorm"]:  # w = s / sum
        total = chosen.sum(-1, keepdim=True)
        g = (g - (g * chosen).sum(-1, keepdim=True) / total) / total
    ds = torch.zeros_like(s).scatter_add_(1, at, g * (ids >= 0))
    if case["score"] == "softmax":
        dz = s * (ds - (ds * s).sum(-1, keepdim=True))
    else:
        dz = ds * s * (1 - s)
    return dz.to(st["logits"].dtype)


def _places(st):
    off = st["offsets"].long()
    at = off[:-1, None] + torch.arange(st["most"], device="cuda")
    ok = at < off[1:, None]
    return st["sorted_slot"].long()[at.clamp(max=st["case"]["rows"] - 1)], ok


def _spread(st, per_adapter, at, ok):
    """[count, most, cols] to rows; rows of no adapter get zeros."""
    out = torch.zeros((st["case"]["rows"], per_adapter.shape[-1]), device="cuda")
    out[at[ok]] = per_adapter[ok]
    return out


def _adapter_plain(st):
    at, ok = _places(st)
    x = st["x"].float()[at] * ok[..., None]
    u = torch.bmm(x, st["a"].float().transpose(1, 2).contiguous())
    d = torch.bmm(u, st["b"].float().transpose(1, 2).contiguous()) * st["scale"][:, None, None]
    y = _spread(st, d, at, ok)
    if st["base"] is not None:
        y = y + st["base"].float()
    return y.to(st["y"].dtype)


def _adapter_back_plain(st):
    at, ok = _places(st)
    x = st["x"].float()[at] * ok[..., None]
    dy = st["dy"].float()[at] * ok[..., None] * st["scale"][:, None, None]
    a, b = st["a"].float(), st["b"].float()
    u = torch.bmm(x, a.transpose(1, 2).contiguous())
    v = torch.bmm(dy, b)
    dx = _spread(st, torch.bmm(v, a), at, ok)
    if st["base"] is not None:
        dx = dx + st["base"].float()
    return {"dx": dx.to(st["dx"].dtype), "da": torch.bmm(v.transpose(1, 2).contiguous(), x),
            "db": torch.bmm(dy.transpose(1, 2).contiguous(), u)}


def run(st):
    if own:
        return _run_own(st)
    return {"route": _route_plain, "route_back": _route_back_plain, "adapter": _adapter_plain,
            "adapter_back": _adapter_back_plain}[st["case"]["op"]](st)


# --------------------------------------------------------------------------
# the framework's calls


def _plan(st):
    """What a program sets up once: the dims and the routing, or the adapters'
    handle and the workspace."""
    if "plan" not in st:
        from paper_2410_12247_amd import moe
        c = st["case"]
        if c["op"].startswith("route"):
            st["plan"] = (
                moe.dims(c["tokens"], 64, 64, c["experts"], c["top_k"], renormalize=c["renorm"]),
                moe.routing(moe.SCORE_SIGMOID if c["score"] == "sigmoid" else moe.SCORE_SOFTMAX,
                            c["groups"], c["top_groups"],
                            moe.GROUP_TOP_TWO if c["pair"] else moe.GROUP_MAX, c["scale"]))
        else:
            ad = moe.adapters(st["a"], st["b"], st["scale"])
            need = (moe.adapter_workspace_bytes if c["op"] == "adapter"
                    else moe.adapter_backward_bytes)(c["rows"], ad)
            st["plan"] = ad, torch.empty(need, dtype=torch.uint8, device="cuda")
    return st["plan"]


def _run_own(st):
    from paper_2410_12247_amd import moe
    op = st["case"]["op"]
    if op == "route":
        d, r = _plan(st)
        moe.route_scores(d, r, st["logits"], st["bias"], st["ids"], st["w"])
        return {"ids": st["ids"], "w": st["w"]}
    if op == "route_back":
        d, r = _plan(st)
        moe.route_scores_backward(d, r, st["logits"], st["ids"], st["dw"], st["dlogits"])
        return st["dlogits"]
    ad, ws = _plan(st)
    order = st["offsets"], st["sorted_slot"], st["slot_row"]
    if op == "adapter":
        moe.adapter_rows(ad, *order, st["x"], st["base"], st["y"], ws)
        return st["y"]
    moe.adapter_backward(ad, *order, st["x"], st["dy"], st["base"], st["dx"], st["da"], st["db"],
                         ws)
    return {"dx": st["dx"], "da": st["da"], "db": st["db"]}


# --------------------------------------------------------------------------
# what a pass cannot do without


def work(case):
    size = 2 if case["type"] == "bf16" else 4
    if case["op"].startswith("route"):
        T, E, k = case["tokens"], case["experts"], case["top_k"]
        if case["op"] == "route":
            return {"bytes": T * (E * size + 8 * k) + (4 * E if case["bias"] else 0),
                    "flops": T * E * 8}
        # a softmax over all experts needs every logit, the others the chosen ones
        read = E if case["score"] == "softmax" and not case["renorm"] else k
        return {"bytes": T * (read * size + 8 * k + E * size), "flops": T * read * 8}
    R, N, K, r = case["rows"], case["n"], case["k"], case["rank"]
    active = float((1 - (1 - _popularity(case)) ** R).sum())  # expected
    rows = R * (1 - case["none"])
    sides = 2 if case["base"] else 1
    weights = 2 * active * (N + K) * r
    if case["op"] == "adapter":
        return {"bytes": 2 * rows * K + weights + sides * R * N * size + 8 * R,
                "flops": 2 * rows * r * (N + K)}
    return {"bytes": 2 * rows * (K + N) + weights + sides * R * K * size
            + 4 * case["count"] * (N + K) * r + 8 * R, "flops": 2 * rows * r * (3 * K + 2 * N)}


# --------------------------------------------------------------------------
# the operators' definitions in 64 bits


def _best(v, taken):
    """The first position of the largest v that is not taken, per row."""
    v = torch.where(taken, -math.inf, v)
    top = v.max(-1, keepdim=True).values
    at = torch.arange(v.shape[-1], device=v.device).expand_as(v)
    at = torch.where((v == top) & ~taken, at, v.shape[-1]).min(-1).values
    return at, top[:, 0]


def _route_64(st):
    case, z = st["case"], st["logits"].double()
    T, E, G = case["tokens"], case["experts"], case["groups"]
    bias = torch.zeros(E, device="cuda") if st["bias"] is None else st["bias"]
    s = torch.softmax(z, -1) if case["score"] == "softmax" else torch.sigmoid(z)
    off = z == -math.inf
    c = s + bias.double()
    out = off.clone()
    if G > 1:
        value = torch.empty((T, G), dtype=torch.float64, device="cuda")
        for g in range(G):
            part = slice(g * (E // G), (g + 1) * (E // G))
            gone = off[:, part].clone()
            at, value[:, g] = _best(c[:, part], gone)
            if case["pair"] and E > G:
                gone.scatter_(1, at.clamp(max=E // G - 1)[:, None], True)
                second = _best(c[:, part], gone)[1]
                value[:, g] += torch.where(second == -math.inf, 0.0, second)
        kept = torch.zeros((T, G), dtype=torch.bool, device="cuda")
        for _ in range(case["top_groups"]):
            kept.scatter_(1, _best(value, kept)[0].clamp(max=G - 1)[:, None], True)
        out |= ~kept[:, torch.arange(E, device="cuda") // (E // G)]
    ids, w = [], []
    for _ in range(case["top_k"]):
        at, _top = _best(z if st["bias"] is None else c, out)
        none = at == E
        at = at.clamp(max=E - 1)
        out.scatter_(1, at[:, None], True)
        ids.append(torch.where(none, -1, at))
        w.append(torch.where(none, 0.0, s[torch.arange(T, device="cuda"), at]))
    ids, w = torch.stack(ids, 1).int(), torch.stack(w, 1)
    if case["renorm"]:
        w = w / w.sum(1, keepdim=True)
    return ids, w * case["scale"]


def _route_back_64(st):
    """Through the derivative of each weight by each score, and of each score
    by each logit."""
    case, z, ids = st["case"], st["logits"].double(), st["ids"].long()
    there = (ids >= 0).double()
    g = st["dw"].double() * there * case["scale"]
    one = torch.zeros((case["tokens"], case["top_k"], 1), device="cuda")
    s = torch.softmax(z, -1) if case["score"] == "softmax" else torch.sigmoid(z)
    chosen = torch.stack([s.gather(1, ids[:, j:j + 1].clamp(min=0))[:, 0] * there[:, j]
                          for j in range(case["top_k"])], 1)
    if case["renorm"]:
        S = chosen.sum(1)
        # dw_j / ds_i = (j == i) / S - s_j / S^2
        g = g / S[:, None] - ((g * chosen).sum(1) / S ** 2)[:, None] * (one[..., 0] + there)
    dz = torch.zeros_like(z)
    for j in range(case["top_k"]):
        at = ids[:, j:j + 1].clamp(min=0)
        p = chosen[:, j:j + 1]
        if case["score"] == "softmax":
            # ds_j / dz_e = s_j ((j == e) - s_e)
            dz -= (g[:, j:j + 1] * there[:, j:j + 1]) * p * s
            dz.scatter_add_(1, at, g[:, j:j + 1] * there[:, j:j + 1] * p)
        else:
            dz.scatter_add_(1, at, g[:, j:j + 1] * there[:, j:j + 1] * p * (1 - p))
    return dz


def exact(case, seed):
    st = prepare(case, seed)
    if case["op"] == "route":
        ids, w = _route_64(st)
        return {"ids": ids, "w": w}
    if case["op"] == "route_back":
        return _route_back_64(st)
    R, N, K = case["rows"], case["n"], case["k"]
    off = [int(v) for v in st["offsets"]]
    forward = case["op"] == "adapter"
    out = torch.zeros((R, N if forward else K), dtype=torch.float64, device="cuda")
    if st["base"] is not None:
        out += st["base"]
    if not forward:
        da = torch.zeros(st["a"].shape, dtype=torch.float64, device="cuda")
        db = torch.zeros(st["b"].shape, dtype=torch.float64, device="cuda")
    for e in range(case["count"]):
        rows = st["sorted_slot"][off[e]:off[e + 1]].long()
        if not len(rows):
            continue
        a, b, f = st["a"][e].double(), st["b"][e].double(), st["scale"][e].double()
        x = st["x"][rows].double()
        u = x @ a.t()
        if forward:
            out[rows] += f * (u @ b.t())
            continue
        dy = st["dy"][rows].double()
        v = dy @ b
        out[rows] += f * (v @ a)
        da[e] = f * (v.t() @ x)
        db[e] = f * (dy.t() @ u)
    return out if forward else {"dx": out, "da": da, "db": db}
