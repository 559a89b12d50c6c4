"""Plain forms, in 64 bits, of the operators between the products of a layer: what their tests compare with."""
import numpy as np
import torch

GROUP, TOP = 32, 57344.0
TORCH = {0: torch.float32, 1: torch.bfloat16, 2: torch.float16}
# half the distance of neighbouring numbers, relative to them, and the smallest distance
UNIT = {0: 2.0 ** -24, 1: 2.0 ** -9, 2: 2.0 ** -12}
TINY = {0: 2.0 ** -149, 1: 2.0 ** -133, 2: 2.0 ** -24}


def rounding(y, kind):
    """How far y (float64) may move when it is rounded to the type (twice the half distance)."""
    return 2 * UNIT[kind] * y.abs() + TINY[kind]


def act(y, which):
    if which == 1:
        return y.clamp_min(0)
    if which == 2:
        return y * torch.special.ndtr(y)
    if which == 3:
        return 0.5 * y * (1 + torch.tanh(np.sqrt(2 / np.pi) * (y + 0.044715 * y ** 3)))
    if which == 4:
        return y * torch.sigmoid(y)
    return y


def encode(x):
    """(n, s, z) of x (... x d, float64): groups of 32 channels."""
    g = x.reshape(*x.shape[:-1], -1, GROUP).clamp(-TOP, TOP)
    lo, hi = g.amin(-1), g.amax(-1)
    step = torch.maximum((hi - lo) / 15, torch.maximum(hi, -lo) / 112)
    unit = torch.exp2(torch.floor(torch.log2(step.clamp_min(2.0 ** -14))) - 3)
    s = torch.ceil(step / unit) * unit
    over = torch.where(s == 0, torch.ones_like(s), s)
    z = -torch.round(lo / over)
    n = (torch.round(g / over[..., None]) + z[..., None]).clamp(0, 15)
    return n, s, z


def held(x):
    n, s, z = encode(x)
    out = s[..., None] * (n - z[..., None])
    bad = ~torch.isfinite(x.reshape(n.shape)).all(-1, keepdim=True)
    return torch.where(bad, torch.full_like(out, float("nan")), out).reshape(x.shape)


def cache_bytes(keys, values, page):
    """The bytes of a cache whose slots hold these rows (slots x heads x d, float64), by the layout's text."""
    slots, heads, d = keys.shape
    block = page * d // 8 * 9
    out = np.zeros((slots // page, heads, block), dtype=np.uint8)
    for which, x in enumerate((keys, values)):
        n, s, z = (t.cpu().numpy() for t in encode(x.cpu()))
        n = n.reshape(slots, heads, d).astype(np.uint32)
        half = s.astype(np.float16).view(np.uint16) >> 7
        base = which * page * d // 16 * 9
        pairs = base + page * d // 2
        for slot in range(slots):
            p, t = divmod(slot, page)
            for w in range(d // 8):
                word = sum(n[slot, :, 8 * w + e] << (4 * e) for e in range(8)).astype("<u4")
                at = base + (16 * (t // 4 * (d // 8) + w) + 4 * (t % 4) if which else t * d // 2 + 4 * w)
                out[p, :, at:at + 4] = word.view(np.uint8).reshape(heads, 4)
            for g in range(d // GROUP):
                at = pairs + 2 * (g * page + t)
                out[p, :, at] = half[slot, :, g]
                out[p, :, at + 1] = z[slot, :, g].astype(np.int8).view(np.uint8)
    return out


def attention(q, keys, values, scale):
    """q: n x d, keys and values: t x d, float64, causal with the queries last."""
    n, t = q.shape[0], keys.shape[0]
    sees = torch.arange(t, device=q.device)[None] <= (t - n + torch.arange(n, device=q.device))[:, None]
    score = (q @ keys.T * scale).masked_fill(~sees, -float("inf"))
    p = torch.where(sees, torch.exp(score - score.amax(-1, keepdim=True)), torch.zeros_like(score))
    total = p.sum(-1, keepdim=True)
    return torch.where(total > 0, p @ values / total, torch.zeros_like(q))
