"""The operators of a mixture of experts between and around the integer products, as measurable cases.

``route``    each token's experts from its scores (softmax or sigmoid, a bias for balance, groups of experts, the
             largest few, weights renormalised), and the token's rows sorted by expert;
``experts``  8-bit rows through the 8-bit weights of the expert each belongs to, scales, bias and activation in the
             write-back, gated or not;
``join``     the end of a block: its rows (of several experts, by weight) summed, normed, gated, scaled and added to the
             residual stream, and the norm in front of the next block, as real numbers or in 8 bits.

``prepare`` makes what a serving program holds before a call, ``run`` is one pass: the plain form in torch operations, or,
where ``own`` is set, the calls into this library.  ``exact`` is the same pass from the definitions, in 64 bits.
"""
import math

import torch

own = False

DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
EPS = 1e-6


# ---------------------------------------------------------------------------
# cases
# ---------------------------------------------------------------------------

def _route(name, tokens, experts, top, dtype="f32", scoring="softmax", bias=False, groups=1, top_groups=1, best=1,
           normalise=True, scale=1.0, pad=0):
    return {"name": name, "kind": "route", "tokens": tokens, "experts": experts, "top": top, "dtype": dtype,
            "scoring": scoring, "bias": bias, "groups": groups, "top_groups": top_groups, "best": best,
            "normalise": normalise, "scale": scale, "pad": pad}


def _experts(name, tokens, experts, top, n, k, gated=False, act="none", dtype="bf16", bias=False, gather=True, pad=0):
    """gather: A holds the tokens and each sorted row names one (the products behind the router); else A holds the sorted
    rows themselves (the second products).  pad: added to every smallest leading dimension."""
    return {"name": name, "kind": "experts", "tokens": tokens, "experts": experts, "top": top, "n": n, "k": k,
            "gated": gated, "act": act, "dtype": dtype, "bias": bias, "gather": gather, "pad": pad}


def _join(name, rows, cols, parts, dtype="bf16", post="none", gate_rows=0, residual=True, norm="rms", real=True, codes=False,
          scale=1.0, pad=0):
    """gate_rows: consecutive rows that share a row of gates (0: no gate)."""
    return {"name": name, "kind": "join", "rows": rows, "cols": cols, "parts": parts, "dtype": dtype, "post": post,
            "gate_rows": gate_rows, "residual": residual, "norm": norm, "real": real, "codes": codes, "scale": scale, "pad": pad}


def listed():
    return [
        # one token of one request: latency
        _route("route_1_token", 1, 128, 8),
        # a ragged batch of half-precision scores with no renormalisation, experts that are no power of two
        _route("route_odd", 517, 60, 4, dtype="bf16", normalise=False, pad=3),
        # a prompt over many experts in groups, with the bias that balances them
        _route("route_prompt_groups", 8192, 256, 8, scoring="sigmoid", bias=True, groups=8, top_groups=4, best=2, scale=2.5),
        # one token through the first products of its eight experts: latency, and eight experts' weights
        _experts("experts_1_token", 1, 64, 8, 1024, 2048, gated=True, act="silu"),
        # thirty-two requests decoding together through the second products: all experts' weights for a few rows each
        _experts("experts_32_tokens", 32, 64, 8, 2048, 1024, gather=False),
        # rows of no convenient number, length or distance, with biases
        _experts("experts_odd", 203, 12, 3, 515, 777, act="gelu", dtype="f32", bias=True, pad=3),
        # a prompt through the first products of many small experts
        _experts("experts_prompt", 4096, 64, 8, 1024, 2048, gated=True, act="silu"),
        # a prompt through the second products of a few large experts, a long k
        _experts("experts_prompt_few", 2048, 8, 2, 4096, 11008, gather=False),
        # one token's eight experts into the residual stream and the next norm, in both forms: latency
        _join("join_1_token", 1, 4096, 8, codes=True),
        # an encoder's ragged batch: the norm behind the addition, mean subtracted
        _join("join_odd", 517, 1027, 1, dtype="f16", norm="layer", pad=3),
        # a prompt between norms on both sides of a block, gated by sequence
        _join("join_prompt", 8192, 4096, 1, post="rms", gate_rows=2048),
        # a prompt's eight experts each, by weight
        _join("join_prompt_experts", 8192, 2048, 8, scale=0.5),
    ]


def _size(rng, lo, hi):
    """Log-uniform in lo .. hi; a third of them multiples of 64, a third of 16, a third as drawn."""
    x = int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))
    unit = rng.choice((64, 16, 1))
    if x >= unit:
        x = x // unit * unit
    return max(lo, min(hi, x))


def draw(rng):
    kind = rng.choice(("route", "experts", "experts", "join"))
    if kind == "route":
        groups = rng.choice((1, 1, 2, 4, 8))
        each = _size(rng, 4, 512 // groups)
        experts = groups * each
        top_groups = rng.randint(1, groups)
        top = rng.randint(1, min(8, top_groups * each))
        case = _route("", _size(rng, 1, 8192), experts, top, rng.choice(("f32", "f32", "bf16", "f16")),
                      rng.choice(("softmax", "sigmoid")), rng.random() < 0.5, groups, top_groups, rng.choice((1, 2)),
                      rng.random() < 0.7, rng.choice((1.0, 2.5)), rng.choice((0, 0, 3)))
        while case["tokens"] * experts > 8192 * 256:
            case["tokens"] //= 2
    elif kind == "experts":
        experts = rng.choice((4, 8, 12, 16, 32, 60, 64, 128, 160))
        top, gated = rng.randint(1, min(8, experts)), rng.random() < 0.5
        n, k = _size(rng, 64, 4096), _size(rng, 64, 11008)
        tokens = _size(rng, 1, 4096)
        while experts * n * k * (2 if gated else 1) > 8 * 4096 * 11008:
            n, k = (max(64, n // 2), k) if n > k else (n, max(64, k // 2))
        while tokens > 1 and tokens * top * n * k * (2 if gated else 1) > 4096 * 4096 * 11008:
            tokens //= 2
        case = _experts("", tokens, experts, top, n, k, gated, rng.choice(("silu", "gelu", "gelu_tanh", "relu")) if gated or rng.random() < 0.4 else "none",
                        rng.choice(("bf16", "bf16", "f16", "f32")), rng.random() < 0.3, rng.random() < 0.5, rng.choice((0, 0, 16, 5)))
    else:
        parts = rng.choice((1, 1, 2, 4, 8, rng.randint(3, 8)))
        rows, cols = _size(rng, 1, 8192), _size(rng, 64, 8192)
        while rows * cols * (parts + 3) > 8192 * 2048 * 11:
            rows = max(1, rows // 2)
        dtype = rng.choice(("bf16", "bf16", "f16", "f32"))
        codes = dtype != "f32" and rng.random() < 0.4
        case = _join("", rows, cols, parts, dtype, rng.choice(("none", "rms", "layer")),
                     rng.choice((0, rows, max(1, rows // 3), 1)), rng.random() < 0.9, rng.choice(("rms", "rms", "layer", "none")),
                     not codes or rng.random() < 0.5, codes, rng.choice((1.0, 0.22)), rng.choice((0, 0, 8, 5)))
    case.pop("name", None)
    return case


def _outputs(case):
    """Columns of an expert's weights."""
    return case["n"] * (2 if case["gated"] else 1)


def work(case):
    size = {"f32": 4, "bf16": 2, "f16": 2}[case["dtype"]]
    if case["kind"] == "route":
        t, e, top = case["tokens"], case["experts"], case["top"]
        return {"bytes": t * e * size + 16 * t * top + 4 * (e + 1) + (4 * e if case["bias"] else 0), "flops": 4 * t * e}
    if case["kind"] == "experts":
        rows, k = case["tokens"] * case["top"], case["k"]
        hit = min(case["experts"], rows)  # (a few fewer where tokens meet in one)
        return {"bytes": hit * _outputs(case) * (k + (8 if case["bias"] else 4))
                + (case["tokens"] if case["gather"] else rows) * (k + 4) + rows * (case["n"] * size + 4),
                "flops": 2 * rows * _outputs(case) * k}
    r, c, parts = case["rows"], case["cols"], case["parts"]
    gates = -(-r // case["gate_rows"]) if case["gate_rows"] else 0
    return {"bytes": r * c * size * (parts + 1 + (1 if case["residual"] else 0) + (1 if case["real"] else 0))
            + (r * c if case["codes"] else 0) + gates * c * size + 8 * r * parts + 8 * c, "flops": r * c * (2 * parts + 8)}


# ---------------------------------------------------------------------------
# inputs
# ---------------------------------------------------------------------------

def _generator(seed, stream):
    return torch.Generator(device="cuda").manual_seed(int(seed) * 1000003 + stream)


def _normal(seed, stream, shape, spread=1.0):
    return torch.randn(shape, generator=_generator(seed, stream), device="cuda") * spread


def _codes(seed, stream, shape):
    """Weights and activations in 8 bits: rounded normal numbers."""
    return _normal(seed, stream, shape, 30.0).round().clamp(-127, 127).to(torch.int8)


def _padded(x, pad):
    """x with its last dimension's rows pad elements further apart than they are long."""
    if not pad:
        return x.contiguous()
    buf = torch.zeros((*x.shape[:-1], x.shape[-1] + pad), dtype=x.dtype, device="cuda")
    buf[..., :x.shape[-1]] = x
    return buf[..., :x.shape[-1]]


def _sorted(ids, experts):
    """(starts, order, places) of the experts' rows: flat places of ids in the order of their expert, equal ones as they came."""
    flat = ids.reshape(-1).long()
    order = torch.sort(flat, stable=True).indices
    starts = (flat[None, :] < torch.arange(experts + 1, device="cuda")[:, None]).sum(1)
    places = torch.empty_like(order)
    places[order] = torch.arange(order.numel(), device="cuda")
    return starts.to(torch.int32), order.to(torch.int32), places.to(torch.int32).reshape(ids.shape)


def prepare(case, seed):
    dtype = DTYPES[case["dtype"]]
    s = dict(case)
    if case["kind"] == "route":
        t, e, top = case["tokens"], case["experts"], case["top"]
        # some experts are asked for more than others
        s["logits"] = _padded((_normal(seed, 1, (t, e), 1.5) + _normal(seed, 2, (1, e), 0.7)).to(dtype), case["pad"])
        s["bias_"] = _normal(seed, 3, (e,), 0.1) if case["bias"] else None
        for name, shape, kind in (("ids", (t, top), torch.int32), ("weights", (t, top), torch.float32), ("starts", (e + 1,), torch.int32),
                                  ("order", (t * top,), torch.int32), ("places", (t, top), torch.int32)):
            s[name] = torch.zeros(shape, dtype=kind, device="cuda")
        s["workspace"] = torch.empty(16 << 20, dtype=torch.uint8, device="cuda")
        return s
    if case["kind"] == "experts":
        t, e, top, k, cols, pad = case["tokens"], case["experts"], case["top"], case["k"], _outputs(case), case["pad"]
        score = _normal(seed, 1, (t, e)) + _normal(seed, 2, (1, e), 0.3)
        s["starts"], s["order"], _ = _sorted(torch.topk(score, top, 1).indices, e)
        s["a"] = _padded(_codes(seed, 3, (t if case["gather"] else t * top, k)), pad)
        s["a_scales"] = torch.rand(s["a"].shape[0], generator=_generator(seed, 4), device="cuda") * 0.02 + 0.01
        s["w"] = _padded(_codes(seed, 5, (e, cols, k)), pad)
        s["w_scales"] = (torch.rand((e, cols), generator=_generator(seed, 6), device="cuda") + 0.5) / (30.0 * math.sqrt(k))
        s["bias_"] = _normal(seed, 7, (e, cols), 0.5) if case["bias"] else None
        s["out"] = _padded(torch.zeros((t * top, case["n"]), dtype=dtype, device="cuda"), pad)
        s["most"] = int((s["starts"][1:] - s["starts"][:-1]).max())
        return s
    r, c, parts, pad = case["rows"], case["cols"], case["parts"], case["pad"]
    s["x"] = _padded(_normal(seed, 1, (r * parts, c), 1.5).to(dtype), pad)
    if parts > 1:
        order = torch.randperm(r * parts, generator=_generator(seed, 2), device="cuda")
        s["places"] = order.reshape(r, parts).to(torch.int32)
        w = torch.rand((r, parts), generator=_generator(seed, 3), device="cuda") + 0.05
        s["part_weights"] = w / w.sum(1, keepdim=True)
    else:
        s["places"] = s["part_weights"] = None
    s["post_gain"] = _normal(seed, 4, (c,), 0.2) + 1.0 if case["post"] != "none" else None
    s["post_shift"] = _normal(seed, 5, (c,), 0.2) if case["post"] == "layer" else None
    s["gain"] = _normal(seed, 6, (c,), 0.2) + 1.0 if case["norm"] != "none" else None
    s["shift"] = _normal(seed, 7, (c,), 0.2) if case["norm"] == "layer" else None
    s["gates"] = _padded(_normal(seed, 8, (-(-r // case["gate_rows"]), c), 0.5).to(dtype), pad) if case["gate_rows"] else None
    s["stream"] = _padded(_normal(seed, 9, (r, c), 2.0).to(dtype), pad) if case["residual"] else None
    for name in ("h",) + (("n_out",) if case["real"] else ()) + (("values",) if case["codes"] else ()):
        s[name] = _padded(torch.zeros((r, c), dtype=dtype, device="cuda"), pad)
    s["q"] = torch.zeros((r, (c + 15) // 16 * 16), dtype=torch.int8, device="cuda")[:, :c] if case["codes"] else None
    s["q_scales"] = torch.zeros(r, device="cuda") if case["codes"] else None
    return s


# ---------------------------------------------------------------------------
# plain forms: 32 bits, and 64 where two scores are compared
# ---------------------------------------------------------------------------

def _plain_route(s):
    t, e, top, groups = s["tokens"], s["experts"], s["top"], s["groups"]
    x = s["logits"].double()
    if s["scoring"] == "softmax":
        x = torch.exp(x - x.amax(1, keepdim=True))
        scores = x / x.sum(1, keepdim=True)
    else:
        scores = 1.0 / (1.0 + torch.exp(-x))
    choice = scores + s["bias_"].double() if s["bias"] else scores
    if groups > 1:
        best = torch.sort(choice.reshape(t, groups, -1), dim=2, descending=True).values[..., :s["best"]].sum(2)
        kept = torch.sort(best, dim=1, descending=True, stable=True).indices[:, :s["top_groups"]]
        hidden = torch.ones((t, groups), dtype=torch.bool, device="cuda").scatter_(1, kept, False)
        choice = choice.masked_fill(hidden.repeat_interleave(e // groups, 1), -math.inf)
    ids = torch.sort(choice, dim=1, descending=True, stable=True).indices[:, :top]
    w = torch.gather(scores, 1, ids)
    if s["normalise"]:
        w = w / w.sum(1, keepdim=True)
    starts, order, places = _sorted(ids, e)
    return {"ids": ids.to(torch.int32), "weights": (w * s["scale"]).float(), "starts": starts, "order": order, "places": places}


def _activate(y, act):
    if act == "relu":
        return torch.maximum(y, torch.zeros_like(y))
    if act == "gelu":
        return 0.5 * y * (1.0 + torch.erf(y * math.sqrt(0.5)))
    if act == "gelu_tanh":
        return 0.5 * y * (1.0 + torch.tanh(math.sqrt(2.0 / math.pi) * (y + 0.044715 * y * y * y)))
    if act == "silu":
        return y / (1.0 + torch.exp(-y))
    return y


def _plain_experts(s):
    e, starts, rows = s["experts"], s["starts"].long(), s["order"].numel()
    at = torch.arange(rows, device="cuda")
    of = torch.searchsorted(starts[1:].contiguous(), at, right=True)  # each row's expert
    token = torch.div(s["order"].long(), s["top"], rounding_mode="floor") if s["gather"] else at
    a = s["a"][token].float()
    if rows < e:  # each row with its expert's weights
        sums = torch.bmm(s["w"][of].float(), a[:, :, None])[:, :, 0]
    else:  # each expert with its rows, as many as the most asked for one has
        inside = at - starts[of]
        panel = torch.zeros((e, s["most"], s["k"]), device="cuda")
        panel[of, inside] = a
        sums = torch.bmm(panel, s["w"].float().transpose(1, 2).contiguous())[of, inside]
    y = sums * s["a_scales"][token][:, None] * s["w_scales"][of]
    if s["bias"]:
        y = y + s["bias_"][of]
    if s["gated"]:
        y = _activate(y[:, :s["n"]], s["act"]) * y[:, s["n"]:]
    else:
        y = _activate(y, s["act"])
    return y.to(s["out"].dtype)


def _normed(x, kind, gain, shift):
    if kind == "none":
        return x
    if kind == "layer":
        x = x - x.mean(1, keepdim=True)
    x = x * torch.rsqrt((x * x).mean(1, keepdim=True) + EPS) * gain
    return x + shift if kind == "layer" else x


def _plain_join(s):
    r, c, parts, dtype = s["rows"], s["cols"], s["parts"], s["x"].dtype
    if parts > 1:
        y = (s["x"][s["places"].long()].float() * s["part_weights"][:, :, None]).sum(1)
    else:
        y = s["x"].float()
    y = _normed(y, s["post"], s["post_gain"], s["post_shift"])
    if s["gate_rows"]:
        y = y * s["gates"].float()[torch.div(torch.arange(r, device="cuda"), s["gate_rows"], rounding_mode="floor")]
    y = y * s["scale"]
    if s["residual"]:
        y = y + s["stream"].float()
    h = y.to(dtype)
    n = _normed(h.float(), s["norm"], s["gain"], s["shift"])
    out = {"h": h}
    if s["real"]:
        out["n"] = n.to(dtype)
    if s["codes"]:
        top = n.abs().amax(1, keepdim=True)
        q = torch.round(n * 127.0 / torch.where(top > 0, top, torch.ones_like(top)))
        out["q"] = (q * (top / torch.full_like(top, 127.0))).to(dtype)
    return out


# ---------------------------------------------------------------------------
# this library's calls
# ---------------------------------------------------------------------------

def _own_route(s):
    import paper_2506_11728_amd as M
    M.mipgemm_route(s["tokens"], s["experts"], s["top"], s["logits"], s["logits"].stride(0), getattr(M, s["dtype"].upper()), s["bias_"],
                    M.SIGMOID if s["scoring"] == "sigmoid" else M.SOFTMAX, s["groups"], s["top_groups"], s["best"], int(s["normalise"]),
                    s["scale"], s["ids"], s["weights"], s["starts"], s["order"], s["places"],
                    workspace=s["workspace"], workspace_bytes=s["workspace"].numel())
    return {"ids": s["ids"], "weights": s["weights"], "starts": s["starts"], "order": s["order"], "places": s["places"]}


def _own_experts(s):
    import paper_2506_11728_amd as M
    a, w, out = s["a"], s["w"], s["out"]
    M.mipgemm_s8s8_experts(out.shape[0], s["experts"], s["n"], s["k"], a, a.stride(0), a.shape[0], s["a_scales"], s["starts"],
                           s["order"] if s["gather"] else None, s["top"], w, w.stride(1), w.stride(0), s["w_scales"], s["bias_"],
                           getattr(M, s["act"].upper()), int(s["gated"]), out, out.stride(0), getattr(M, s["dtype"].upper()))
    return out


def _own_join(s):
    import paper_2506_11728_amd as M
    norms = {"none": M.NO_NORM, "rms": M.RMS_NORM, "layer": M.LAYER_NORM}
    x, h, gates, stream, n, q = s["x"], s["h"], s["gates"], s["stream"], s.get("n_out"), s["q"]
    c = s["cols"]
    M.mipgemm_join_rows(s["rows"], c, s["parts"], getattr(M, s["dtype"].upper()), x, x.stride(0), x.shape[0], s["places"],
                        s["part_weights"], norms[s["post"]], s["post_gain"], s["post_shift"], gates,
                        gates.stride(0) if gates is not None else c, s["gate_rows"] or 1, s["scale"], stream,
                        stream.stride(0) if stream is not None else c, h, h.stride(0), norms[s["norm"]], s["gain"], s["shift"], EPS,
                        n, n.stride(0) if n is not None else c, q, q.stride(0) if q is not None else c, s["q_scales"])
    out = {"h": h}
    if s["real"]:
        out["n"] = n
    if s["codes"]:  # what the codes stand for
        out["q"] = torch.mul(q, s["q_scales"][:, None], out=s["values"])
    return out


def run(state):
    kind = state["kind"]
    if own:
        return {"route": _own_route, "experts": _own_experts, "join": _own_join}[kind](state)
    return {"route": _plain_route, "experts": _plain_experts, "join": _plain_join}[kind](state)


# ---------------------------------------------------------------------------
# from the definitions, in 64 bits
# ---------------------------------------------------------------------------

def _exact_route(s):
    x = s["logits"].to(torch.float64)
    score = torch.softmax(x, dim=1) if s["scoring"] == "softmax" else torch.special.expit(x)
    left = score.clone() if s["bias_"] is None else score + s["bias_"].to(torch.float64)
    each = s["experts"] // s["groups"]
    if s["groups"] > 1:
        of_group = torch.stack([torch.topk(left[:, g * each:(g + 1) * each], s["best"], dim=1).values.sum(dim=1) for g in range(s["groups"])], 1)
        open_ = torch.zeros_like(left, dtype=torch.bool)
        for _ in range(s["top_groups"]):
            g = (of_group == of_group.max(dim=1, keepdim=True).values).to(torch.int8).argmax(dim=1)  # the first of the largest
            for i in range(each):
                open_[torch.arange(x.shape[0], device="cuda"), g * each + i] = True
            of_group[torch.arange(x.shape[0], device="cuda"), g] = -math.inf
        left[~open_] = -math.inf
    picked = []
    for _ in range(s["top"]):
        i = (left == left.max(dim=1, keepdim=True).values).to(torch.int8).argmax(dim=1)
        picked.append(i)
        left[torch.arange(x.shape[0], device="cuda"), i] = -math.inf
    ids = torch.stack(picked, 1)
    w = torch.stack([score[torch.arange(x.shape[0], device="cuda"), i] for i in picked], 1)
    if s["normalise"]:
        w = w / w.sum(dim=1, keepdim=True)
    flat = ids.reshape(-1).cpu().tolist()
    rows = [[] for _ in range(s["experts"])]
    for at, i in enumerate(flat):
        rows[i].append(at)
    order = [at for r in rows for at in r]
    places = [0] * len(order)
    for p, at in enumerate(order):
        places[at] = p
    starts = [0]
    for r in rows:
        starts.append(starts[-1] + len(r))
    whole = lambda v: torch.tensor(v, dtype=torch.int32, device="cuda")  # noqa: E731
    return {"ids": ids.to(torch.int32), "weights": w * s["scale"], "starts": whole(starts), "order": whole(order),
            "places": whole(places).reshape(ids.shape)}


def _exact_experts(s):
    f64 = torch.float64
    starts, n = s["starts"].tolist(), s["n"]
    out = torch.empty((s["order"].numel(), n), dtype=f64, device="cuda")
    for e in range(s["experts"]):
        first, last = starts[e], starts[e + 1]
        if last == first:
            continue
        rows = s["order"][first:last].long() // s["top"] if s["gather"] else torch.arange(first, last, device="cuda")
        y = torch.mm(s["a"][rows].to(f64), s["w"][e].to(f64).t().contiguous())
        y = y * s["w_scales"][e].to(f64).unsqueeze(0) * s["a_scales"][rows].to(f64).unsqueeze(1)
        if s["bias_"] is not None:
            y = y + s["bias_"][e].to(f64)
        z = y[:, :n]
        if s["act"] == "relu":
            z = z.clamp_min(0.0)
        elif s["act"] == "gelu":
            z = z * torch.special.ndtr(z)
        elif s["act"] == "gelu_tanh":
            z = z * torch.sigmoid(2.0 * math.sqrt(2.0 / math.pi) * (z + 0.044715 * z.pow(3)))
        elif s["act"] == "silu":
            z = z * torch.sigmoid(z)
        out[first:last] = z * y[:, n:] if s["gated"] else z
    return out


def _exact_join(s):
    f64, parts, dtype = torch.float64, s["parts"], s["x"].dtype

    def norm(v, kind, gain, shift):
        if kind == "rms":
            return v / (v.pow(2).mean(dim=1, keepdim=True) + EPS).sqrt() * gain.to(f64)
        if kind == "layer":
            spread = v.var(dim=1, unbiased=False, keepdim=True)
            return (v - v.mean(dim=1, keepdim=True)) / (spread + EPS).sqrt() * gain.to(f64) + shift.to(f64)
        return v

    y = torch.zeros((s["rows"], s["cols"]), dtype=f64, device="cuda")
    for j in range(parts):
        if s["places"] is None:
            y += s["x"].to(f64)
        else:
            y += s["x"][s["places"][:, j].long()].to(f64) * s["part_weights"][:, j:j + 1].to(f64)
    y = norm(y, s["post"], s["post_gain"], s["post_shift"])
    if s["gates"] is not None:
        y = y * s["gates"].to(f64).repeat_interleave(s["gate_rows"], dim=0)[:s["rows"]]
    h = y * s["scale"]
    if s["stream"] is not None:
        h = h + s["stream"].to(f64)
    n = norm(h.to(dtype).to(f64), s["norm"], s["gain"], s["shift"])  # of the stream as it is stored
    out = {"h": h}
    if s["real"]:
        out["n"] = n
    if s["codes"]:
        step = n.abs().max(dim=1, keepdim=True).values / 127.0
        out["q"] = (n / torch.where(step > 0, step, 1.0)).round() * step
    return out


def exact(case, seed):
    state = prepare(case, seed)
    return {"route": _exact_route, "experts": _exact_experts, "join": _exact_join}[case["kind"]](state)
