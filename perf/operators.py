"""Products whose rows choose their right operand, as cases to be timed and compared: routing to experts, the experts'
products with their gradients, the weighted sum of a token's experts, and low-rank adapters beside a shared projection.

run() computes a case in its plain form, elementary torch operations in 32 bits rounded once at the end, or, where `own` is
true, by the calls that a program makes of this library.  exact() is the definition in 64 bits.
"""
import math

import torch

own = False  # whether run() makes the library's calls

F32, F16, BF16 = "f32", "f16", "bf16"
TORCH = {F32: torch.float32, F16: torch.float16, BF16: torch.bfloat16}
# operand and result type of a kind
KINDS = {"f32": (F32, F32), "f16f32": (F16, F32), "f16f16": (F16, F16), "bf16f32": (BF16, F32), "bf16bf16": (BF16, BF16)}
BYTES = {F32: 4, F16: 2, BF16: 2}

# what a drawn case may cost: no more than the largest listed ones
MOST_FLOPS, MOST_BYTES = 5.6e11, 1.3e9


def _route(name, tokens, experts, top_k, type, score, bias=False, groups=1, top_groups=1, group_top=1, renormalise=True, scale=1.0):
    return {"name": name, "op": "route", "tokens": tokens, "experts": experts, "top_k": top_k, "type": type, "score": score, "bias": bias,
            "groups": groups, "top_groups": top_groups, "group_top": group_top, "renormalise": renormalise, "scale": scale}


def _route_backward(name, tokens, experts, top_k, type, score, renormalise=True, scale=1.0):
    return {"name": name, "op": "route_backward", "tokens": tokens, "experts": experts, "top_k": top_k, "type": type, "score": score,
            "renormalise": renormalise, "scale": scale}


def _grouped(name, kind, tokens, top_k, experts, N, K, layout, gather=True):
    return {"name": name, "op": "grouped", "kind": kind, "tokens": tokens, "top_k": top_k, "experts": experts, "N": N, "K": K,
            "layout": layout, "gather": gather}


def _wgrad(name, kind, tokens, top_k, experts, M, N, layout, gather=True):
    return {"name": name, "op": "wgrad", "kind": kind, "tokens": tokens, "top_k": top_k, "experts": experts, "M": M, "N": N,
            "layout": layout, "gather": gather}


def _combine(name, kind, tokens, top_k, N, backward):
    return {"name": name, "op": "combine", "kind": kind, "tokens": tokens, "top_k": top_k, "N": N, "backward": backward}


def _adapters(name, kind, rows, N, K, adapters, rank, layout, run):
    return {"name": name, "op": "adapters", "kind": kind, "rows": rows, "N": N, "K": K, "adapters": adapters, "rank": rank,
            "layout": layout, "run": run}


def listed():
    return [
        # one step of serving 64 requests: the router's scores, whose latency every layer waits for
        _route("route_serving", 64, 128, 8, F32, "softmax"),
        # a training batch on many experts in groups, with the bias that balances them
        _route("route_grouped_batch", 16384, 256, 8, BF16, "sigmoid", True, 8, 4, 2, True, 2.5),
        # the router's gradient of a training batch
        _route_backward("route_backward_batch", 16384, 128, 8, F32, "softmax"),
        # and on odd numbers of tokens and experts, weights left as they are
        _route_backward("route_backward_odd", 1001, 60, 4, BF16, "sigmoid", False, 1.5),
        # serving 64 requests: a few rows for each of many experts, the weights are what is read
        _grouped("grouped_serving", "bf16bf16", 64, 8, 128, 1536, 2048, "col"),
        # a prompt or training batch: hundreds of rows for each expert (also the size of its operand's gradient)
        _grouped("grouped_batch", "bf16bf16", 8192, 8, 64, 2048, 2048, "col"),
        # the experts' weight gradients of a training batch, rows of the tokens gathered
        _wgrad("wgrad_batch", "bf16f32", 8192, 4, 32, 2048, 1024, "row"),
        # the same on odd sizes, stored as the weights of a column-major product are
        _wgrad("wgrad_odd", "f16f16", 1500, 2, 7, 515, 334, "col", False),
        # the sum of a token's experts after a prompt
        _combine("combine_batch", "bf16bf16", 8192, 8, 2048, False),
        # its gradient in a small training step
        _combine("combine_backward", "f16f16", 2048, 4, 1000, True),
        # one token of each of 64 requests, any of 32 adapters or none
        _adapters("adapters_serving", "bf16bf16", 64, 4096, 4096, 32, 16, "col", 1),
        # prompts of some hundred tokens, an adapter each
        _adapters("adapters_prompts", "f16f32", 8192, 4096, 4096, 8, 64, "col", 300),
    ]


def _size(rng, lo, hi, step=1):
    x = math.exp(rng.uniform(math.log(lo), math.log(hi)))
    return min(hi, max(lo, int(round(x / step)) * step))


def _draw(rng):
    op = rng.choice(("route", "route_backward", "grouped", "grouped", "wgrad", "combine", "adapters", "adapters"))
    kind = rng.choice(("bf16bf16", "bf16bf16", "bf16f32", "f16f16", "f16f32", "f32"))
    step = rng.choice((1, 8, 64))  # odd extents, whole 16-byte granules, whole tiles
    layout = rng.choice(("row", "col"))
    if op in ("route", "route_backward"):
        groups = rng.choice((1, 1, 4, 8)) if op == "route" else 1
        experts = groups * _size(rng, 8 if groups == 1 else 4, 256 // groups)
        top_groups = rng.randint(max(1, groups // 2), groups)
        top_k = rng.randint(1, min(8, top_groups * (experts // groups)))
        type, score, renormalise = rng.choice((F32, BF16, F16)), rng.choice(("softmax", "sigmoid")), rng.random() < 0.7
        tokens, scale = _size(rng, 1, 16384), rng.choice((1.0, 2.5))
        if op == "route":
            return _route("", tokens, experts, top_k, type, score, rng.random() < 0.5, groups, top_groups, rng.choice((1, 2)), renormalise, scale)
        return _route_backward("", tokens, experts, top_k, type, score, renormalise, scale)
    top_k = rng.randint(1, 8)
    if op == "grouped":
        experts = _size(rng, 8, 128)
        return _grouped("", kind, _size(rng, 1, 8192), top_k, experts, _size(rng, 256, 2048, step), _size(rng, 256, 2048, step), layout,
                        rng.random() < 0.6)
    if op == "wgrad":
        return _wgrad("", kind, _size(rng, 64, 8192), top_k, _size(rng, 8, 64), _size(rng, 256, 2048, step), _size(rng, 256, 2048, step),
                      layout, rng.random() < 0.6)
    if op == "combine":
        return _combine("", kind, _size(rng, 1, 8192), top_k, _size(rng, 256, 2048, step), kind in ("f32", "f16f16", "bf16bf16") and rng.random() < 0.5)
    run = rng.choice((1, 1, 300))
    rows = _size(rng, 1, 256) if run == 1 else _size(rng, 256, 8192)
    return _adapters("", kind, rows, _size(rng, 512, 4096, step), _size(rng, 512, 4096, step), _size(rng, 1, 32),
                     rng.choice((8, 16, 32, 64, rng.randint(3, 64))), layout, run)


def draw(rng):
    while True:
        case = _draw(rng)
        del case["name"]
        w = work(case)
        if w["flops"] <= MOST_FLOPS * (0.05 if case.get("kind") == "f32" else 1.0) and w["bytes"] <= MOST_BYTES:
            return case


# ---------------------------------------------------------------------------- inputs
def _gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def _normal(gen, shape, type, scale=1.0):
    return (torch.randn(shape, generator=gen, device="cuda") * scale).to(TORCH[type])


def _logits(gen, tokens, experts):
    """A router's scores: some experts are preferred to others."""
    return torch.randn((tokens, experts), generator=gen, device="cuda") * 1.2 + torch.randn((experts,), generator=gen, device="cuda") * 0.6


def _eligible(case, logits, bias):
    """Scores and choice values in 64 bits, those of experts that no chosen group holds at minus infinity."""
    score = torch.softmax(logits.double(), 1) if case["score"] == "softmax" else torch.sigmoid(logits.double())
    choice = score if bias is None else score + bias.double()
    G = case.get("groups", 1)
    if G > 1:
        per = choice.view(choice.shape[0], G, -1)
        rank = per.topk(min(case["group_top"], per.shape[2]), 2).values.sum(2)
        order = rank.argsort(dim=1, descending=True, stable=True)[:, :case["top_groups"]]
        kept = torch.zeros_like(rank, dtype=torch.bool).scatter_(1, order, True)
        choice = torch.where(kept.unsqueeze(2), per, -math.inf).flatten(1)
        return score, choice, rank
    return score, choice, None


def _undecided(case, logits, bias):
    """Rows in which the rounding of 32-bit scores may decide which expert comes first: choice values (or those of groups)
    nearer than some units in the last place, and not of equal logits that every evaluation finds equal."""
    _, choice, rank = _eligible(case, logits, bias)
    k = min(case["top_k"] + 1, choice.shape[1])
    val, idx = choice.sort(dim=1, descending=True, stable=True)
    val = val[:, :k]
    gap = val[:, :-1] - val[:, 1:]
    close = gap <= 4e-6 * val[:, :-1].abs()
    if bias is None:
        at = logits.gather(1, idx[:, :k])
        close &= at[:, :-1] != at[:, 1:]
    bad = close.any(1)
    if rank is not None:
        val = rank.sort(dim=1, descending=True).values
        n = case["top_groups"]
        if n < case["groups"]:
            bad |= val[:, n - 1] - val[:, n] <= 4e-6 * val[:, n - 1].abs()
    return bad


def _routing(gen, case, tokens, experts, type):
    """A router's logits and balancing bias.  Which experts are chosen has to be the same for every evaluation in 32 bits, so
    tokens whose choice hangs on a rounding are drawn again."""
    bias = torch.randn((experts,), generator=gen, device="cuda") * 0.02 if case.get("bias") else None
    logits = _logits(gen, tokens, experts).to(TORCH[type])
    for _ in range(12):
        bad = _undecided(case, logits, bias)
        again = _logits(gen, tokens, experts).to(TORCH[type])
        logits = torch.where(bad.unsqueeze(1), again, logits)
    return logits, bias


def _sorted_entries(indices, experts):
    """offsets, token of a slot, slot of a token's entry, for the experts chosen by each token."""
    tokens, k = indices.shape
    flat = indices.flatten().long()
    order = flat.argsort(stable=True)
    slot_of = torch.empty_like(order)
    slot_of[order] = torch.arange(order.numel(), device="cuda")
    counts = (flat.unsqueeze(0) == torch.arange(experts, device="cuda").unsqueeze(1)).sum(1)
    offsets = torch.cat([torch.zeros(1, dtype=torch.long, device="cuda"), counts.cumsum(0)])
    return offsets.int(), (order // k).int(), slot_of.view(tokens, k).int()


def _assignment(gen, case):
    tokens, experts, k = case["tokens"], case["experts"], min(case["top_k"], case["experts"])
    return _sorted_entries(_logits(gen, tokens, experts).topk(k, 1).indices, experts)


def prepare(case, seed):
    gen = _gen(seed)
    s = {"case": case}
    op = case["op"]
    if op in ("route", "route_backward"):
        T, E, k = case["tokens"], case["experts"], case["top_k"]
        s["logits"], s["bias"] = _routing(gen, case, T, E, case["type"])
        if op == "route":
            s["weights"] = torch.empty((T, k), device="cuda")
            s["indices"] = torch.empty((T, k), dtype=torch.int32, device="cuda")
            s["offsets"] = torch.empty(E + 1, dtype=torch.int32, device="cuda")
            s["token_of"] = torch.empty(T * k, dtype=torch.int32, device="cuda")
            s["slot_of"] = torch.empty((T, k), dtype=torch.int32, device="cuda")
        else:
            s["indices"] = s["logits"].double().topk(k, 1).indices.int()
            s["d_weights"] = torch.randn((T, k), generator=gen, device="cuda")
            s["d_logits"] = torch.empty_like(s["logits"])
    elif op in ("grouped", "wgrad"):
        a, c = KINDS[case["kind"]]
        s["offsets"], token_of, _ = _assignment(gen, case)
        s["bounds"] = s["offsets"].tolist()
        rows, E, N = token_of.numel(), case["experts"], case["N"]
        s["rows"], s["map"] = rows, token_of if case["gather"] else None
        width = case["K"] if op == "grouped" else case["M"]
        s["A"] = _normal(gen, (case["tokens"] if case["gather"] else rows, width), a)
        if op == "grouped":
            s["B"] = _normal(gen, (E, width, N) if case["layout"] == "row" else (E, N, width), a, width ** -0.5)
            s["C"] = torch.empty((rows, N), dtype=TORCH[c], device="cuda")
        else:
            s["D"] = _normal(gen, (rows, N), a)
            s["C"] = torch.empty((E, width, N) if case["layout"] == "row" else (E, N, width), dtype=TORCH[c], device="cuda")
    elif op == "combine":
        a, c = KINDS[case["kind"]]
        T, k, N = case["tokens"], case["top_k"], case["N"]
        s["slot_of"] = torch.randperm(T * k, generator=gen, device="cuda").int().view(T, k)
        s["weights"] = torch.softmax(torch.randn((T, k), generator=gen, device="cuda"), 1)
        s["Y"] = _normal(gen, (T * k, N), a)
        if case["backward"]:
            s["d_out"] = _normal(gen, (T, N), a)
            s["dY"], s["d_weights"] = torch.empty_like(s["Y"]), torch.empty((T, k), device="cuda")
        else:
            s["out"] = torch.empty((T, N), dtype=TORCH[c], device="cuda")
    else:
        a, c = KINDS[case["kind"]]
        rows, N, K, n, r = case["rows"], case["N"], case["K"], case["adapters"], case["rank"]
        s["A"] = _normal(gen, (rows, K), a)
        s["B"] = _normal(gen, (K, N) if case["layout"] == "row" else (N, K), a, K ** -0.5)
        s["down"] = _normal(gen, (n, r, K), a, K ** -0.5)
        s["up"] = _normal(gen, (n, N, r), a, 0.5 * r ** -0.5)
        s["scales"] = torch.rand((n,), generator=gen, device="cuda") + 0.5
        # runs of rows of one request each, every eighth or so without an adapter
        runs = -(-rows // case["run"]) * 2 + 1
        of = torch.randint(0, n, (runs,), generator=gen, device="cuda")
        of = torch.where(torch.rand((runs,), generator=gen, device="cuda") < 0.125, torch.full_like(of, -1), of)
        if case["run"] == 1:
            s["adapter_of"] = of[:rows].int()
        else:
            starts = torch.randint(0, rows, (runs - 1,), generator=gen, device="cuda").sort().values
            s["adapter_of"] = of[(torch.arange(rows, device="cuda").unsqueeze(0) >= starts.unsqueeze(1)).sum(0)].int()
        s["C"] = torch.empty((rows, N), dtype=TORCH[c], device="cuda")
    if own:
        _prepare_calls(s)
    return s


# ---------------------------------------------------------------------------- the library's calls
def _prepare_calls(s):
    """The library's functions and their arguments, as a program that owns its buffers keeps them."""
    import paper_2003_06324_amd as g
    case, op = s["case"], s["case"]["op"]
    stream = torch.cuda.current_stream().cuda_stream
    elem = {F32: g.ELEM_F32, F16: g.ELEM_F16, BF16: g.ELEM_BF16}
    kind = {"f32": g.KIND_F32, "f16f32": g.KIND_F16F32, "f16f16": g.KIND_F16F16, "bf16f32": g.KIND_BF16F32, "bf16bf16": g.KIND_BF16BF16}
    lay = {"row": g.ROW_MAJOR, "col": g.COL_MAJOR}
    score = {"softmax": g.SCORE_SOFTMAX, "sigmoid": g.SCORE_SIGMOID}
    if op == "route":
        T, E, k = case["tokens"], case["experts"], case["top_k"]
        s["calls"] = ((g.gemm_route, (elem[case["type"]], T, E, s["logits"], 0, s["bias"], score[case["score"]], case["groups"], case["top_groups"],
                                      case["group_top"], k, int(case["renormalise"]), case["scale"], s["weights"], s["indices"], stream)),
                      (g.gemm_route_plan, (T, k, E, s["indices"], s["offsets"], s["token_of"], s["slot_of"], stream)))
        s["result"] = (s["weights"], s["indices"], s["offsets"], s["token_of"], s["slot_of"])
    elif op == "route_backward":
        s["calls"] = ((g.gemm_route_backward, (elem[case["type"]], case["tokens"], case["experts"], s["logits"], 0, score[case["score"]],
                                               case["top_k"], int(case["renormalise"]), case["scale"], s["indices"], s["d_weights"],
                                               s["d_logits"], 0, stream)),)
        s["result"] = (s["d_logits"],)
    elif op == "grouped":
        s["calls"] = ((g.gemm_grouped, (kind[case["kind"]], case["experts"], s["offsets"], s["rows"], case["N"], case["K"], s["A"],
                                        s["A"].shape[0], 0, s["map"], s["B"], lay[case["layout"]], 0, 0, s["C"], 0, stream)),)
        s["result"] = (s["C"],)
    elif op == "wgrad":
        s["calls"] = ((g.gemm_grouped_wgrad, (kind[case["kind"]], case["experts"], s["offsets"], s["rows"], case["M"], case["N"], s["A"],
                                              s["A"].shape[0], 0, s["map"], s["D"], 0, s["C"], lay[case["layout"]], 0, 0, stream)),)
        s["result"] = (s["C"],)
    elif op == "combine":
        T, k, N = case["tokens"], case["top_k"], case["N"]
        if case["backward"]:
            s["calls"] = ((g.gemm_combine_backward, (elem[KINDS[case["kind"]][0]], T, k, N, s["d_out"], 0, s["Y"], T * k, 0, s["slot_of"],
                                                     s["weights"], s["dY"], 0, s["d_weights"], stream)),)
            s["result"] = (s["dY"], s["d_weights"])
        else:
            s["calls"] = ((g.gemm_combine, (kind[case["kind"]], T, k, N, s["Y"], T * k, 0, s["slot_of"], s["weights"], s["out"], 0, stream)),)
            s["result"] = (s["out"],)
    else:
        s["calls"] = ((g.gemm_adapters, (kind[case["kind"]], case["rows"], case["N"], case["K"], s["A"], 0, s["B"], lay[case["layout"]], 0,
                                         case["adapters"], case["rank"], s["adapter_of"], s["scales"], s["down"], g.COL_MAJOR, 0, 0,
                                         s["up"], g.COL_MAJOR, 0, 0, s["C"], 0, stream)),)
        s["result"] = (s["C"],)


def run(state):
    if own:
        for fn, args in state["calls"]:
            fn(*args)
        return state["result"]
    return _PLAIN[state["case"]["op"]](state["case"], state)


# ---------------------------------------------------------------------------- plain forms
def _scores32(case, logits):
    l = logits.float()
    if case["score"] == "sigmoid":
        return 1.0 / (1.0 + torch.exp(-l))
    e = torch.exp(l - l.amax(1, keepdim=True))
    return e / e.sum(1, keepdim=True)


def _plain_route(case, s):
    T, E, k, G = case["tokens"], case["experts"], case["top_k"], case["groups"]
    score = _scores32(case, s["logits"])
    choice = score if s["bias"] is None else score + s["bias"]
    if G > 1:
        per = choice.view(T, G, E // G)
        best = per.sort(dim=2, descending=True).values
        rank = best[:, :, 0] + best[:, :, 1] if case["group_top"] == 2 and E // G > 1 else best[:, :, 0]
        kept = torch.zeros((T, G), dtype=torch.bool, device=rank.device)
        kept.scatter_(1, rank.sort(dim=1, descending=True, stable=True).indices[:, :case["top_groups"]], True)
        choice = torch.where(kept.repeat_interleave(E // G, 1), choice, torch.full_like(choice, -math.inf))
    indices = choice.sort(dim=1, descending=True, stable=True).indices[:, :k]
    w = score.gather(1, indices)
    if case["renormalise"]:
        w = w / w.sum(1, keepdim=True)
    flat = indices.flatten()
    order = flat.sort(stable=True).indices
    slot_of = torch.empty_like(order)
    slot_of[order] = torch.arange(T * k, device=order.device)
    offsets = torch.zeros(E + 1, dtype=torch.int64, device=order.device)
    offsets[1:] = torch.zeros(E, dtype=torch.int64, device=order.device).index_add_(0, flat, torch.ones_like(flat)).cumsum(0)
    return w * case["scale"], indices.int(), offsets.int(), (order // k).int(), slot_of.view(T, k).int()


def _plain_route_backward(case, s):
    score, at, dw = _scores32(case, s["logits"]), s["indices"].long(), s["d_weights"]
    chosen = score.gather(1, at)
    if case["renormalise"]:
        total = chosen.sum(1, keepdim=True)
        ds = case["scale"] / total * (dw - (dw * chosen).sum(1, keepdim=True) / total)
    else:
        ds = case["scale"] * dw
    full = torch.zeros_like(score).scatter_(1, at, ds)
    if case["score"] == "softmax":
        dl = score * (full - (full * score).sum(1, keepdim=True))
    else:
        dl = full * score * (1.0 - score)
    return (dl.to(TORCH[case["type"]]),)


def _plain_grouped(case, s):
    a = s["A"].float()
    if s["map"] is not None:
        a = a[s["map"].long()]
    out = torch.empty((s["rows"], case["N"]), device=a.device)
    for e in range(case["experts"]):
        lo, hi = s["bounds"][e], s["bounds"][e + 1]
        if hi > lo:
            b = s["B"][e].float()
            out[lo:hi] = torch.mm(a[lo:hi], b if case["layout"] == "row" else b.t())
    return (out.to(s["C"].dtype),)


def _plain_wgrad(case, s):
    a, d = s["A"].float(), s["D"].float()
    if s["map"] is not None:
        a = a[s["map"].long()]
    out = torch.zeros(s["C"].shape, device=a.device)
    for e in range(case["experts"]):
        lo, hi = s["bounds"][e], s["bounds"][e + 1]
        if hi > lo:
            out[e] = torch.mm(a[lo:hi].t(), d[lo:hi]) if case["layout"] == "row" else torch.mm(d[lo:hi].t(), a[lo:hi])
    return (out.to(s["C"].dtype),)


def _plain_combine(case, s):
    y, at, w = s["Y"].float(), s["slot_of"].long(), s["weights"]
    if not case["backward"]:
        out = torch.zeros((case["tokens"], case["N"]), device=y.device)
        for j in range(case["top_k"]):
            out += w[:, j:j + 1] * y[at[:, j]]
        return (out.to(s["out"].dtype),)
    d = s["d_out"].float()
    dy, dw = torch.empty_like(y), torch.empty_like(w)
    for j in range(case["top_k"]):
        dy[at[:, j]] = w[:, j:j + 1] * d
        dw[:, j] = (d * y[at[:, j]]).sum(1)
    return dy.to(s["Y"].dtype), dw


def _plain_adapters(case, s):
    n, r, N, K = case["adapters"], case["rank"], case["N"], case["K"]
    a, b = s["A"].float(), s["B"].float()
    out = torch.mm(a, b if case["layout"] == "row" else b.t())
    # every adapter's down projection of every row, zero where it is not the row's own
    mine = (s["adapter_of"].unsqueeze(1) == torch.arange(n, device=a.device)) * s["scales"]
    t = torch.mm(a, s["down"].float().view(n * r, K).t()) * mine.repeat_interleave(r, 1)
    out += torch.mm(t, s["up"].float().transpose(1, 2).reshape(n * r, N))
    return (out.to(s["C"].dtype),)


_PLAIN = {"route": _plain_route, "route_backward": _plain_route_backward, "grouped": _plain_grouped, "wgrad": _plain_wgrad,
          "combine": _plain_combine, "adapters": _plain_adapters}


# ---------------------------------------------------------------------------- bytes and operations
def work(case):
    op = case["op"]
    if op in ("route", "route_backward"):
        T, E, k, esz = case["tokens"], case["experts"], case["top_k"], BYTES[case["type"]]
        if op == "route":  # logits, bias; weights, indices, the plan
            return {"bytes": T * E * esz + E * 4 * case["bias"] + T * k * 16 + (E + 1) * 4, "flops": 5.0 * T * E}
        return {"bytes": 2 * T * E * esz + T * k * 8, "flops": 8.0 * T * E}
    a, c = (BYTES[x] for x in KINDS[case["kind"]])
    if op in ("grouped", "wgrad"):
        T, E, N = case["tokens"], case["experts"], case["N"]
        rows = T * min(case["top_k"], E)
        a_rows = T if case["gather"] else rows
        plan = (E + 1) * 4 + rows * 4 * case["gather"]
        if op == "grouped":  # every expert that some row chose (about: of rows dealt out evenly), its weights once
            K, touched = case["K"], E * (1.0 - (1.0 - 1.0 / E) ** rows)
            return {"bytes": a_rows * K * a + touched * K * N * a + rows * N * c + plan, "flops": 2.0 * rows * N * K}
        M = case["M"]
        return {"bytes": a_rows * M * a + rows * N * a + E * M * N * c + plan, "flops": 2.0 * rows * M * N}
    if op == "combine":
        T, k, N = case["tokens"], case["top_k"], case["N"]
        if case["backward"]:
            return {"bytes": T * N * a + 2 * T * k * N * a + T * k * 12, "flops": 3.0 * T * k * N}
        return {"bytes": T * k * N * a + T * N * c + T * k * 8, "flops": 2.0 * T * k * N}
    rows, N, K, n, r = case["rows"], case["N"], case["K"], case["adapters"], case["rank"]
    requests = max(1, round(rows / case["run"]))
    used = n * (1.0 - (1.0 - 1.0 / n) ** (0.875 * requests))
    return {"bytes": rows * K * a + K * N * a + used * r * (K + N) * a + rows * N * c + rows * 4 + n * 4,
            "flops": 2.0 * rows * N * K + 0.875 * 2.0 * rows * r * (N + K)}


# ---------------------------------------------------------------------------- the definition in 64 bits
def exact(case, seed):
    s = prepare(case, seed)
    op = case["op"]
    if op == "route":
        score, choice, _ = _eligible(case, s["logits"], s["bias"])
        indices = choice.argsort(dim=1, descending=True, stable=True)[:, :case["top_k"]]
        w = torch.take_along_dim(score, indices, 1) * case["scale"]
        if case["renormalise"]:
            w = w / torch.take_along_dim(score, indices, 1).sum(1, True)
        return (w, indices.int()) + _sorted_entries(indices, case["experts"])
    if op == "route_backward":
        l, at, dw = s["logits"].double(), s["indices"].long(), s["d_weights"].double()
        score = torch.softmax(l, 1) if case["score"] == "softmax" else torch.sigmoid(l)
        w = score.gather(1, at)
        if case["renormalise"]:
            w = w / w.sum(1, True)
        # weights as functions of the logits: derivatives entry by entry, d w_j / d l_i summed over j
        eye = torch.zeros_like(score).unsqueeze(1).repeat(1, at.shape[1], 1).scatter_(2, at.unsqueeze(2), 1.0)  # [t, j, e]
        chosen = eye.sum(1)
        if case["score"] == "softmax":
            d = eye - ((chosen * score / score.gather(1, at).sum(1, True)) if case["renormalise"] else score).unsqueeze(1)
        else:
            d = eye * (1.0 - score).unsqueeze(1)
            if case["renormalise"]:
                d = d - (chosen * score * (1.0 - score) / score.gather(1, at).sum(1, True)).unsqueeze(1)
        return ((case["scale"] * dw * w).unsqueeze(1).matmul(d).squeeze(1),)
    if op in ("grouped", "wgrad"):
        rows = torch.arange(s["rows"], device="cuda") if s["map"] is None else s["map"].long()
        out = torch.zeros(s["C"].shape, dtype=torch.float64, device="cuda")
        for e in range(case["experts"]):
            mine = slice(s["bounds"][e], s["bounds"][e + 1])
            a = s["A"].index_select(0, rows[mine]).double()
            if op == "grouped":
                b = s["B"][e].double()
                out[mine] = a @ (b if case["layout"] == "row" else b.t())
            else:
                g = a.t() @ s["D"][mine].double()
                out[e] = g if case["layout"] == "row" else g.t()
        return (out,)
    if op == "combine":
        w, at = s["weights"].double(), s["slot_of"].long()
        if not case["backward"]:
            return (sum(w[:, j, None] * s["Y"].index_select(0, at[:, j]).double() for j in range(case["top_k"])),)
        d = s["d_out"].double()
        dy = torch.zeros(s["Y"].shape, dtype=torch.float64, device="cuda")
        dy[at.flatten()] = (w.unsqueeze(2) * d.unsqueeze(1)).flatten(0, 1)
        return dy, (s["Y"].double()[at] * d.unsqueeze(1)).sum(2)
    a, b = s["A"].double(), s["B"].double()
    out = a @ (b if case["layout"] == "row" else b.t())
    for i in range(case["adapters"]):
        rows = (s["adapter_of"] == i).nonzero().flatten()
        if rows.numel():
            out[rows] += s["scales"][i].double() * (a[rows] @ s["down"][i].double().t() @ s["up"][i].double().t())
    return (out,)
