"""The operators between the integer products of a quantised transformer layer, as measurable cases.

``linear``     activations brought to 8 bits with a scale for each row (optionally through an RMS norm), the
               8-bit product, and bias, activation and residual in its epilogue;
``rope``       norms of queries and keys for each head and their rotation, keys and values written into a
               cache held in 4 bits, and the written rows read back;
``attention``  queries over that cache, for single tokens, drafted tokens and prompts.

``prepare`` makes what a serving program holds before a call, ``run`` is one pass: the plain form in 32-bit
torch operations, or, where ``own`` is set, the calls into this library.  ``exact`` is the same pass from the
definitions, in 64 bits.

The 4-bit form: a group of 32 channels of one token and head is  x ~ s (n - z), n in 0..15, |z| <= 127 and s a
number of 4 significant bits (the upper byte and a bit of a float16: its code times 128).  A page of the cache
holds, for each head, the keys' codes (token by token, two channels a byte), their (s, z) pairs (group by
group), the values' codes (four tokens interleaved by 4 bytes) and their pairs.
"""
import math

import torch

own = False

DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
GROUP = 32
TOP = 57344.0  # what a group can hold


# ---------------------------------------------------------------------------
# cases
# ---------------------------------------------------------------------------

def _linear(name, m, n, k, dtype="bf16", act="none", norm=False, bias=False, residual=False, quantise=True, pad=0):
    """quantise: the activations arrive as real numbers (else as 8-bit codes with row scales); pad: added
    to every smallest leading dimension."""
    return {"name": name, "kind": "linear", "m": m, "n": n, "k": k, "dtype": dtype, "act": act, "norm": norm,
            "bias": bias, "residual": residual, "quantise": quantise, "pad": pad}


def _rope(name, tokens, heads, kv_heads, d, dtype="bf16", rot=None, interleaved=False, page=64):
    return {"name": name, "kind": "rope", "tokens": tokens, "heads": heads, "kv_heads": kv_heads, "d": d,
            "dtype": dtype, "rot": d if rot is None else rot, "interleaved": interleaved, "page": page}


def _attention(name, requests, max_q, max_kv, heads, kv_heads, d, dtype="bf16", page=64):
    return {"name": name, "kind": "attention", "requests": requests, "max_q": max_q, "max_kv": max_kv,
            "heads": heads, "kv_heads": kv_heads, "d": d, "dtype": dtype, "page": page}


def listed():
    return [
        # one token of one request through an attention output layer: latency
        _linear("linear_1_token", 1, 4096, 4096, residual=True),
        # forty-eight requests decoding together through a down-projection with a long k
        _linear("linear_48_tokens", 48, 4096, 11008, residual=True),
        # the first feed-forward layer of an encoder block on 256 tokens
        _linear("linear_encoder_gelu", 256, 4096, 1024, dtype="f16", act="gelu", bias=True),
        # activations that a statically quantised layer left in 8 bits, nothing a multiple of anything
        _linear("linear_odd_sizes", 1003, 1027, 2051, dtype="f32", act="relu", bias=True, residual=True,
                quantise=False, pad=3),
        # a prompt through an up-projection behind a norm
        _linear("linear_prompt", 4096, 11008, 4096, act="silu", norm=True),
        # one token of each of four requests: latency
        _rope("rope_4_tokens", 4, 32, 8, 128),
        # a ragged batch on wide heads, a part of the channels rotated in neighbouring pairs
        _rope("rope_517_tokens", 517, 16, 4, 256, dtype="f16", rot=64, interleaved=True, page=16),
        # a prompt's queries, keys and values
        _rope("rope_prompt", 8192, 32, 8, 128),
        # one token of one short request on encoder-sized heads: latency
        _attention("attention_1_token", 1, 1, 301, 16, 16, 64, dtype="f16", page=16),
        # thirty-two requests of ragged lengths decoding together
        _attention("attention_32_requests", 32, 1, 8192, 32, 8, 128),
        # one long document: few rows, a long axis
        _attention("attention_long", 1, 1, 131001, 32, 8, 128, page=128),
        # a chunk of a prompt over what came before it and over itself
        _attention("attention_prompt_chunk", 1, 2048, 8192, 32, 8, 128),
    ]


def _size(rng, lo, hi):
    """Log-uniform in lo .. hi; a third of them multiples of 64, a third of 16, a third as drawn."""
    x = int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))
    unit = rng.choice((64, 16, 1))
    if x >= unit:
        x = x // unit * unit
    return max(lo, min(hi, x))


def draw(rng):
    kind = rng.choice(("linear", "linear", "rope", "attention", "attention"))
    if kind == "linear":
        m, n, k = _size(rng, 1, 4096), _size(rng, 64, 11008), _size(rng, 64, 11008)
        while m * n * k > 4096 * 11008 * 4096:
            m = max(1, m // 2)
        case = _linear("", m, n, k, rng.choice(("bf16", "bf16", "f16", "f32")),
                       rng.choice(("none", "relu", "gelu", "gelu_tanh", "silu")),
                       rng.random() < 0.4, rng.random() < 0.5, rng.random() < 0.5, rng.random() < 0.8,
                       rng.choice((0, 0, 16, 5)))
        case["norm"] = case["norm"] and case["quantise"]
    elif kind == "rope":
        d = rng.choice((64, 128, 128, 256))
        kv = rng.choice((1, 2, 4, 8))
        case = _rope("", _size(rng, 1, 8192), kv * rng.choice((1, 2, 4)), kv, d,
                     rng.choice(("bf16", "bf16", "f16")), rng.choice((d, d, d // 2, d // 4)),
                     rng.random() < 0.3, rng.choice((16, 32, 64, 128)))
        while case["tokens"] * (case["heads"] + 2 * kv) * d > 8192 * 48 * 128:
            case["tokens"] //= 2
    else:
        d = rng.choice((64, 128, 128, 256))
        kv = rng.choice((1, 2, 4, 8))
        heads = kv * rng.choice((1, 2, 4, 8))
        requests = _size(rng, 1, 64)
        max_kv = _size(rng, 1, 131072)
        max_q = min(max_kv, rng.choice((1, 1, _size(rng, 2, 16), _size(rng, 17, 2048))))
        while requests > 1 and (requests * max_kv * kv * d > 32 * 8192 * 8 * 128
                                or requests * max_q * max_kv * heads * d > 2048 * 8192 * 32 * 128):
            requests //= 2
        while max_kv > 1 and (max_kv * kv * d > 32 * 8192 * 8 * 128 or max_q * max_kv * heads * d > 2048 * 8192 * 32 * 128):
            max_kv //= 2
            max_q = min(max_q, max_kv)
        case = _attention("", requests, max_q, max_kv, heads, kv, d, rng.choice(("bf16", "bf16", "f16")),
                          rng.choice((16, 32, 64, 128)))
    case.pop("name", None)
    return case


def _lengths(case):
    """(queries, keys) of each request: ragged, the first the longest, the queries among the keys."""
    got = []
    for r in range(case["requests"]):
        part = 1.0 - (r * 0.6180339887) % 1.0
        keys = max(1, int(case["max_kv"] * part))
        got.append((max(1, min(keys, int(round(case["max_q"] * (1.0 - (r * 0.3819660113) % 1.0))))), keys))
    return got


def work(case):
    size = {"f32": 4, "bf16": 2, "f16": 2}[case["dtype"]]
    if case["kind"] == "linear":
        m, n, k = case["m"], case["n"], case["k"]
        return {"bytes": m * k * (size if case["quantise"] else 1) + k * n + m * n * size * (2 if case["residual"] else 1)
                + 4 * n * (2 if case["bias"] else 1), "flops": 2 * m * n * k}
    if case["kind"] == "rope":
        t, h, kv, d = case["tokens"], case["heads"], case["kv_heads"], case["d"]
        # queries twice (in and out), keys and values three times (in, as 4 bits out, read back whole)
        return {"bytes": t * d * (2 * h * size + 2 * kv * (2 * size + 2 * 9 / 16)) + 4 * t * case["rot"],
                "flops": t * (h + kv) * d * 8}
    lengths = _lengths(case)
    rows = sum(q for q, _ in lengths)
    seen = sum(q * (n - q) + q * (q + 1) // 2 for q, n in lengths)
    return {"bytes": sum(n for _, n in lengths) * case["kv_heads"] * case["d"] * 9 / 8
            + 2 * rows * case["heads"] * case["d"] * size,
            "flops": 4 * seen * case["heads"] * case["d"]}


# ---------------------------------------------------------------------------
# the 4-bit form
# ---------------------------------------------------------------------------

def _codes(x):
    """(n, code of s, z) of x, a tensor of float32 with whole groups in its last dimension."""
    g = x.reshape(*x.shape[:-1], -1, GROUP).clamp(-TOP, TOP)
    lo, hi = g.amin(-1), g.amax(-1)
    step = torch.maximum((hi - lo) / torch.full_like(lo, 15.0), torch.maximum(hi, -lo) / torch.full_like(lo, 112.0))
    up = ((step.view(torch.int32) + 0xFFFFF) & ~0xFFFFF).view(torch.float32)  # 4 significant bits
    s = torch.where(step < 2.0 ** -14, torch.ceil(step * 2.0 ** 17) * 2.0 ** -17, up)
    over = torch.where(s > 0, s, torch.ones_like(s))
    z = -torch.round(lo / over)
    n = (torch.round(g / over[..., None]) + z[..., None]).clamp(0, 15)
    code = s.to(torch.float16).view(torch.int16).to(torch.int32) >> 7
    return n.reshape(x.shape), code, z


def _values(n, code, z):
    s = (code << 7).to(torch.int16).view(torch.float16).float()
    g = n.reshape(*n.shape[:-1], -1, GROUP)
    return (s[..., None] * (g - z[..., None])).reshape(n.shape)


def _pages(keys, values, page):
    """The cache with these rows in its slots (slots x heads x d each): bytes."""
    out = []
    for x, interleaved in ((keys, False), (values, True)):
        slots, heads, d = x.shape
        n, code, z = _codes(x)
        n = n.to(torch.uint8).reshape(-1, page, heads, d // 2, 2)
        b = n[..., 0] | (n[..., 1] << 4)                                     # page, token, head, byte
        if interleaved:
            b = b.reshape(-1, page // 4, 4, heads, d // 8, 4).permute(0, 3, 1, 4, 2, 5)
        else:
            b = b.permute(0, 2, 1, 3)
        pairs = torch.stack((code.to(torch.uint8), z.to(torch.int8).view(torch.uint8)), -1)
        pairs = pairs.reshape(-1, page, heads, d // GROUP, 2).permute(0, 2, 3, 1, 4)
        out += [b.reshape(b.shape[0], heads, -1), pairs.reshape(b.shape[0], heads, -1)]
    return torch.cat(out, -1).contiguous()


def _rows(blocks, page, d):
    """Keys and values, float32, of gathered pages (... x pages x heads x bytes): ... x heads x tokens x d."""
    *lead, np_, heads, _ = blocks.shape
    got, at = [], 0
    for interleaved in (False, True):
        b = blocks[..., at:at + page * d // 2]
        at += page * d // 2
        p = blocks[..., at:at + page * d // 16].reshape(*lead, np_, heads, d // GROUP, page, 2)
        at += page * d // 16
        if interleaved:
            b = b.reshape(*lead, np_, heads, page // 4, d // 8, 4, 4).transpose(-3, -2)
        b = b.reshape(*lead, np_, heads, page, d // 2)
        n = torch.stack((b & 15, b >> 4), -1).reshape(*lead, np_, heads, page, d)
        p = p.transpose(-3, -2)
        x = _values(n.float(), p[..., 0].to(torch.int32), p[..., 1].contiguous().view(torch.int8).float())
        got.append(x.transpose(-4, -3).reshape(*lead, heads, np_ * page, d))
    return got


# ---------------------------------------------------------------------------
# inputs
# ---------------------------------------------------------------------------

def _generator(seed, stream):
    return torch.Generator(device="cuda").manual_seed(int(seed) * 1000003 + stream)


def _normal(seed, stream, shape, spread=1.0):
    return torch.randn(shape, generator=_generator(seed, stream), device="cuda") * spread


def _padded(x, pad):
    """x (rows x columns) with rows pad elements further apart than they are long."""
    if not pad:
        return x.contiguous()
    buf = torch.zeros((x.shape[0], x.shape[1] + pad), dtype=x.dtype, device="cuda")
    buf[:, :x.shape[1]] = x
    return buf[:, :x.shape[1]]


def _table(positions, rot):
    angle = torch.arange(positions, device="cuda", dtype=torch.float64)[:, None] * (
        10000.0 ** (-torch.arange(0, rot, 2, device="cuda", dtype=torch.float64) / rot))
    return angle.cos().float().contiguous(), angle.sin().float().contiguous()


def prepare(case, seed):
    dtype = DTYPES[case["dtype"]]
    s = dict(case)
    if case["kind"] == "linear":
        m, n, k, pad = case["m"], case["n"], case["k"], case["pad"]
        if case["quantise"]:
            s["x"] = _padded(_normal(seed, 1, (m, k), 2.0).to(dtype), pad)
        else:
            s["a"] = _padded(_normal(seed, 1, (m, k), 30.0).round().clamp(-127, 127).to(torch.int8), pad)
            s["a_scales"] = torch.rand(m, generator=_generator(seed, 2), device="cuda") * 0.02 + 0.01
        s["gain"] = _normal(seed, 3, (k,), 0.2) + 1.0 if case["norm"] else None
        s["w"] = _padded(_normal(seed, 4, (n, k), 30.0).round().clamp(-127, 127).to(torch.int8), pad)  # n x k
        s["w_scales"] = (torch.rand(n, generator=_generator(seed, 5), device="cuda") + 0.5) / (30.0 * math.sqrt(k))
        s["bias_"] = _normal(seed, 6, (n,), 0.5) if case["bias"] else None
        s["res"] = _padded(_normal(seed, 7, (m, n)).to(dtype), pad) if case["residual"] else None
        s["out"] = _padded(torch.zeros((m, n), dtype=dtype, device="cuda"), pad)
        s["q"] = torch.empty((m, (k + 15) // 16 * 16), dtype=torch.int8, device="cuda")
        s["q_scales"] = torch.empty(m, device="cuda")
        # room for both operands in whole tiles, and for sums of parts of k
        s["workspace"] = torch.empty((m + n + 512) * (k + 128) + (64 << 20), dtype=torch.uint8, device="cuda")
        return s
    heads, kv, d, page = case["heads"], case["kv_heads"], case["d"], case["page"]
    if case["kind"] == "rope":
        tokens, rot = case["tokens"], case["rot"]
        s["qkv"] = _normal(seed, 1, (tokens, (heads + 2 * kv) * d), 1.5).to(dtype)
        s["q_gain"], s["k_gain"] = _normal(seed, 2, (d,), 0.2) + 1.0, _normal(seed, 3, (d,), 0.2) + 1.0
        s["cos"], s["sin"] = _table(16384, rot)
        s["positions"] = torch.randint(0, 16384, (tokens,), generator=_generator(seed, 4), device="cuda", dtype=torch.int32)
        s["pages"] = (tokens + page - 1) // page + 3
        s["slots"] = torch.randperm(s["pages"] * page, generator=_generator(seed, 5), device="cuda")[:tokens].contiguous()
        s["cache"] = torch.zeros(s["pages"] * page * kv * d * 9 // 8, dtype=torch.uint8, device="cuda")
        s["q_out"] = torch.empty((tokens, heads * d), dtype=dtype, device="cuda")
        s["k_back"] = torch.empty((tokens, kv * d), dtype=dtype, device="cuda")
        s["v_back"] = torch.empty((tokens, kv * d), dtype=dtype, device="cuda")
        return s
    lengths = _lengths(case)
    queries, keys = [q for q, _ in lengths], [n for _, n in lengths]
    rows, width = sum(queries), (case["max_kv"] + page - 1) // page
    used = [(n + page - 1) // page for n in keys]
    s["pages"] = sum(used) + 2
    s["rows"], s["width"] = rows, width
    order = torch.randperm(s["pages"], generator=_generator(seed, 1), device="cuda").to(torch.int32)
    s["table"] = torch.zeros((case["requests"], width), dtype=torch.int32, device="cuda")
    at = 0
    for r, u in enumerate(used):
        s["table"][r, :u] = order[at:at + u]
        at += u
    slots = s["pages"] * page
    # keys vary by channel, as they do behind a projection, values less so
    offset = _normal(seed, 4, (1, kv, d), 0.7)
    s["cache"] = _pages(_normal(seed, 2, (slots, kv, d)) + offset, _normal(seed, 3, (slots, kv, d)), page)
    s["q"] = _normal(seed, 5, (rows, heads * d), 1.0).to(dtype)
    s["out"] = torch.empty((rows, heads * d), dtype=dtype, device="cuda")
    starts = torch.tensor([0] + queries, dtype=torch.int32).cumsum(0)
    s["q_starts"] = starts.to(torch.int32).cuda()
    s["kv_lengths"] = torch.tensor(keys, dtype=torch.int32).cuda()
    s["request_of"] = torch.tensor([r for r, q in enumerate(queries) for _ in range(q)]).cuda()
    s["index_in"] = torch.tensor([i for q in queries for i in range(q)]).cuda()
    s["scale"] = 1.0 / math.sqrt(d)
    # the largest partial results that splitting the keys of a call can leave
    s["workspace"] = torch.empty(256 << 20, dtype=torch.uint8, device="cuda")
    return s


# ---------------------------------------------------------------------------
# plain forms: 32 bits
# ---------------------------------------------------------------------------

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


def _plain_linear(s):
    if s["quantise"]:
        x = s["x"].float()
        z = x * s["gain"] if s["norm"] else x
        top = z.abs().amax(1, keepdim=True)
        codes = torch.round(z * 127.0 / torch.where(top > 0, top, torch.ones_like(top)))
        scales = top[:, 0] / torch.full_like(top[:, 0], 127.0)
        if s["norm"]:
            scales = scales * torch.rsqrt((x * x).mean(1) + 1e-6)
    else:
        codes, scales = s["a"].float(), s["a_scales"]
    y = (codes @ s["w"].float().t()) * scales[:, None] * s["w_scales"]
    if s["bias"]:
        y = y + s["bias_"]
    y = _activate(y, s["act"])
    if s["residual"]:
        y = y + s["res"].float()
    return y.to(s["out"].dtype)


def _rotated(x, cos, sin, rot, interleaved):
    if interleaved:
        a, b = x[..., 0:rot:2], x[..., 1:rot:2]
        turned = torch.stack((a * cos - b * sin, b * cos + a * sin), -1).flatten(-2)
    else:
        a, b = x[..., :rot // 2], x[..., rot // 2:rot]
        turned = torch.cat((a * cos - b * sin, b * cos + a * sin), -1)
    return torch.cat((turned, x[..., rot:]), -1)


def _plain_rope(s):
    tokens, heads, kv, d = s["tokens"], s["heads"], s["kv_heads"], s["d"]
    x = s["qkv"].float().reshape(tokens, heads + 2 * kv, d)
    at = s["positions"].long()
    cos, sin = s["cos"][at][:, None], s["sin"][at][:, None]
    gain = torch.cat((s["q_gain"].expand(heads, d), s["k_gain"].expand(kv, d)))
    y = x[:, :heads + kv]
    y = y * torch.rsqrt((y * y).mean(-1, keepdim=True) + 1e-6) * gain
    y = _rotated(y, cos, sin, s["rot"], s["interleaved"])
    dtype = s["qkv"].dtype
    held = _values(*_codes(torch.cat((y[:, heads:], x[:, heads + kv:]), 1)))
    return {"q": y[:, :heads].reshape(tokens, -1).to(dtype), "k": held[:, :kv].reshape(tokens, -1).to(dtype),
            "v": held[:, kv:].reshape(tokens, -1).to(dtype)}


def _plain_attention(s):
    kv, d, page, shared = s["kv_heads"], s["d"], s["page"], s["heads"] // s["kv_heads"]
    keys, values = _rows(s["cache"][s["table"].long()], page, d)  # request, head, token, channel
    n, last = s["kv_lengths"].long(), s["q_starts"][1:].long() - s["q_starts"][:-1].long()
    q = torch.zeros((s["requests"], s["max_q"], kv, shared, d), device="cuda")
    q[s["request_of"], s["index_in"]] = s["q"].float().reshape(-1, kv, shared, d)
    q = q.permute(0, 2, 3, 1, 4).reshape(s["requests"], kv, -1, d)
    p = torch.matmul(q, keys.transpose(-1, -2)).mul_(s["scale"])
    p = p.reshape(s["requests"], kv, shared, s["max_q"], -1)
    token = torch.arange(p.shape[-1], device="cuda")
    sees = token <= (n - last)[:, None, None] + torch.arange(s["max_q"], device="cuda")[None, :, None]
    p.masked_fill_(~sees[:, None, None], -math.inf)
    p.sub_(p.amax(-1, keepdim=True)).exp_()
    p.div_(p.sum(-1, keepdim=True))
    # (what lies behind a request's last key is in no row's sum, whatever its pages hold)
    values = values.masked_fill((token >= n[:, None])[:, None, :, None], 0.0)
    o = torch.matmul(p.reshape(s["requests"], kv, -1, p.shape[-1]), values)
    o = o.reshape(s["requests"], kv, shared, s["max_q"], d).permute(0, 3, 1, 2, 4)
    return o[s["request_of"], s["index_in"]].reshape(-1, s["heads"] * d).to(s["q"].dtype)


# ---------------------------------------------------------------------------
# this library's calls
# ---------------------------------------------------------------------------

def _own_linear(s):
    import paper_2506_11728_amd as M
    m, n, k, out = s["m"], s["n"], s["k"], s["out"]
    dtype = getattr(M, s["dtype"].upper())
    a, a_scales = s.get("a"), s.get("a_scales")
    if s["quantise"]:
        a, a_scales, x = s["q"], s["q_scales"], s["x"]
        M.mipgemm_quantize_rows(m, k, x, x.stride(0), dtype, s["gain"], 1e-6, a, a.stride(0), a_scales)
    res = s["res"]
    M.mipgemm_s8s8_linear(m, n, k, a, a.stride(0), a_scales, s["w"], s["w"].stride(0), M.COL_MAJOR, s["w_scales"],
                          s["bias_"], getattr(M, s["act"].upper()), res, res.stride(0) if res is not None else n,
                          out, out.stride(0), dtype, workspace=s["workspace"], workspace_bytes=s["workspace"].numel())
    return out


def _own_rope(s):
    import paper_2506_11728_amd as M
    heads, kv, d, qkv = s["heads"], s["kv_heads"], s["d"], s["qkv"]
    dtype, ld = getattr(M, s["dtype"].upper()), qkv.stride(0)
    M.mipgemm_qk_norm_rope(s["tokens"], heads, kv, d, dtype, qkv, ld, qkv[:, heads * d:], ld, qkv[:, (heads + kv) * d:], ld,
                           s["q_gain"], s["k_gain"], 1e-6, s["cos"], s["sin"], s["cos"].shape[0], s["rot"],
                           M.ROTATE_PAIRS if s["interleaved"] else M.ROTATE_HALVES, s["positions"],
                           s["q_out"], heads * d, None, kv * d, s["cache"], s["cache"].numel(), s["pages"], s["page"],
                           s["slots"])
    M.mipgemm_kv4_read(s["tokens"], kv, d, dtype, s["cache"], s["cache"].numel(), s["pages"], s["page"], s["slots"],
                       s["k_back"], kv * d, s["v_back"], kv * d)
    return {"q": s["q_out"], "k": s["k_back"], "v": s["v_back"]}


def _own_attention(s):
    import paper_2506_11728_amd as M
    width = s["heads"] * s["d"]
    M.mipgemm_attention_kv4(s["requests"], s["heads"], s["kv_heads"], s["d"], getattr(M, s["dtype"].upper()), s["q"], width,
                            s["rows"], s["q_starts"], s["max_q"], s["kv_lengths"], s["max_kv"], s["cache"],
                            s["cache"].numel(), s["pages"], s["page"], s["table"], s["width"], s["scale"], s["out"], width,
                            workspace=s["workspace"], workspace_bytes=s["workspace"].numel())
    return s["out"]


def run(state):
    kind = state["kind"]
    if own:
        return {"linear": _own_linear, "rope": _own_rope, "attention": _own_attention}[kind](state)
    return {"linear": _plain_linear, "rope": _plain_rope, "attention": _plain_attention}[kind](state)


# ---------------------------------------------------------------------------
# from the definitions, in 64 bits
# ---------------------------------------------------------------------------

def _exact_linear(s):
    f64 = torch.float64
    if s["quantise"]:
        x = s["x"].to(f64)
        z = x if s["gain"] is None else x * s["gain"].to(f64)
        top = z.abs().max(dim=1).values
        codes = (127.0 * z / top.clamp_min(1e-300)[:, None]).round()
        rows = top / 127.0
        if s["gain"] is not None:
            rows = rows / (x.pow(2).mean(dim=1) + 1e-6).sqrt()
    else:
        codes, rows = s["a"].to(f64), s["a_scales"].to(f64)
    y = torch.empty((s["m"], s["n"]), dtype=f64, device="cuda")
    for j in range(0, s["n"], 1024):  # a panel of output columns at a time
        part = s["w"][j:j + 1024].to(f64)
        y[:, j:j + 1024] = torch.mm(codes, part.t().contiguous())
    y = y * rows.unsqueeze(1) * s["w_scales"].to(f64).unsqueeze(0)
    if s["bias_"] is not None:
        y = y + s["bias_"].to(f64)
    if s["act"] == "relu":
        y = y.clamp_min(0.0)
    elif s["act"] == "gelu":
        y = y * torch.special.ndtr(y)
    elif s["act"] == "gelu_tanh":
        y = y * torch.sigmoid(2.0 * math.sqrt(2.0 / math.pi) * (y + 0.044715 * y.pow(3)))
    elif s["act"] == "silu":
        y = y * torch.sigmoid(y)
    if s["res"] is not None:
        y = y + s["res"].to(f64)
    return y


def _exact_held(x):
    """What the cache holds of x (rows x d, float64), group by group."""
    out = torch.empty_like(x)
    for c in range(0, x.shape[1], GROUP):
        g = x[:, c:c + GROUP].clamp(-TOP, TOP)
        low, high = g.min(dim=1).values, g.max(dim=1).values
        step = torch.maximum((high - low) / 15.0, g.abs().max(dim=1).values / 112.0)
        # the next number of 4 significant bits, none of them below 2^-17
        unit = torch.exp2(torch.floor(torch.log2(step.clamp_min(2.0 ** -14))) - 3.0)
        step = torch.ceil(step / unit) * unit
        safe = torch.where(step == 0, 1.0, step).unsqueeze(1)
        first = torch.round(low.unsqueeze(1) / safe)
        out[:, c:c + GROUP] = step.unsqueeze(1) * (torch.round(g / safe) - first).clamp(0, 15).add(first)
    return out


def _exact_rope(s):
    f64, tokens, heads, kv, d, rot = torch.float64, s["tokens"], s["heads"], s["kv_heads"], s["d"], s["rot"]
    at = s["positions"].long()
    turn = torch.complex(s["cos"][at].to(f64), s["sin"][at].to(f64))
    x = s["qkv"].to(f64)
    q, k, v = [], [], []
    for h in range(heads + kv):
        y = x[:, h * d:(h + 1) * d]
        y = y / (y.pow(2).mean(dim=1, keepdim=True) + 1e-6).sqrt() * (s["q_gain"] if h < heads else s["k_gain"]).to(f64)
        if s["interleaved"]:
            first, second = slice(0, rot, 2), slice(1, rot, 2)
        else:
            first, second = slice(0, rot // 2), slice(rot // 2, rot)
        pair = torch.complex(y[:, first].contiguous(), y[:, second].contiguous()) * turn
        y = y.clone()
        y[:, first], y[:, second] = pair.real, pair.imag
        q.append(y) if h < heads else k.append(_exact_held(y))
    for h in range(heads + kv, heads + 2 * kv):
        v.append(_exact_held(x[:, h * d:(h + 1) * d]))
    return {"q": torch.cat(q, 1), "k": torch.cat(k, 1), "v": torch.cat(v, 1)}


def _exact_attention(s):
    f64, kv, d, page = torch.float64, s["kv_heads"], s["d"], s["page"]
    shared, half = s["heads"] // kv, page * d // 2
    starts, lengths = s["q_starts"].tolist(), s["kv_lengths"].tolist()
    out = torch.zeros((s["rows"], s["heads"], d), dtype=f64, device="cuda")
    for r, n in enumerate(lengths):
        blocks = s["cache"][s["table"][r, :(n + page - 1) // page].long()]  # page, head, byte
        count = blocks.shape[0]
        for h in range(kv):
            held = []
            for part in (0, 1):
                b = blocks[:, h, part * (half + half // 8):][:, :half + half // 8]
                words = b[:, :half].reshape(count, page, d // 2)
                if part:
                    words = b[:, :half].reshape(count, page // 4, d // 8, 4, 4).permute(0, 1, 3, 2, 4).reshape(count, page, d // 2)
                x = torch.empty((count, page, d), dtype=f64, device="cuda")
                x[..., 0::2], x[..., 1::2] = (words % 16).to(f64), (words // 16).to(f64)
                pair = b[:, half:].reshape(count, d // GROUP, page, 2).to(f64)
                exponent, mantissa = torch.floor(pair[..., 0] / 8), pair[..., 0] % 8
                step = torch.where(exponent == 0, mantissa * 2.0 ** -17, (8 + mantissa) * torch.exp2(exponent - 18))
                zero = torch.where(pair[..., 1] > 127, pair[..., 1] - 256, pair[..., 1])
                for g in range(d // GROUP):
                    x[..., g * GROUP:(g + 1) * GROUP] -= zero[:, g, :, None]
                    x[..., g * GROUP:(g + 1) * GROUP] *= step[:, g, :, None]
                held.append(x.reshape(count * page, d)[:n])
            first, last = starts[r], starts[r + 1]
            hidden = torch.arange(n, device="cuda") > (n - (last - first) + torch.arange(last - first, device="cuda"))[:, None]
            for j in range(h * shared, (h + 1) * shared):
                q = s["q"][first:last, j * d:(j + 1) * d].to(f64)
                score = torch.mm(q, held[0].t().contiguous()) * s["scale"]
                out[first:last, j] = torch.mm(torch.softmax(score.masked_fill(hidden, -math.inf), dim=1), held[1])
    return out.reshape(s["rows"], -1)


def exact(case, seed):
    state = prepare(case, seed)
    return {"linear": _exact_linear, "rope": _exact_rope, "attention": _exact_attention}[case["kind"]](state)
