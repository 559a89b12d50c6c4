"""The 4-bit cache: what mipgemm_qk_norm_rope writes, what mipgemm_kv4_read gives back, and attention over it,
against their definitions in 64 bits."""
import numpy as np
import pytest

import layer_reference as R

pytestmark = pytest.mark.gpu

F32, BF16, F16 = 0, 1, 2


@pytest.fixture(scope="module")
def gpu():
    import torch
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_2506_11728_amd as M
    M.load_library()
    return M


def _normed_and_rotated(x, weight, eps, cos, sin, rot, pairs):
    import torch
    y = x.double()
    if weight is not None:
        y = y / torch.sqrt((y * y).mean(-1, keepdim=True) + float(np.float32(eps))) * weight.double()
    if rot == 0:
        return y
    a, b = (slice(0, rot, 2), slice(1, rot, 2)) if pairs else (slice(0, rot // 2), slice(rot // 2, rot))
    c, s = cos.double()[:, None], sin.double()[:, None]
    out = y.clone()
    out[..., a] = y[..., a] * c - y[..., b] * s
    out[..., b] = y[..., b] * c + y[..., a] * s
    return out


def _tables(rows, rot):
    import torch
    angle = torch.arange(rows, dtype=torch.float64)[:, None] * 10000.0 ** (-torch.arange(0, rot, 2, dtype=torch.float64) / max(1, rot))
    return angle.cos().float(), angle.sin().float()


class Heads:
    """Queries, keys and values of `tokens` in one matrix, and a cache with room for them."""

    def __init__(self, M, tokens, hq, hkv, d, kind, page, rot, seed=0, pad=0):
        import torch
        g = torch.Generator().manual_seed(seed)
        width = (hq + 2 * hkv) * d + pad
        x = torch.randn((tokens, width), generator=g) * torch.exp(torch.randn((tokens, 1), generator=g))
        self.x = x.to(R.TORCH[kind])
        self.ld, self.tokens, self.hq, self.hkv, self.d, self.kind, self.page = width, tokens, hq, hkv, d, kind, page
        self.pages = (tokens + page - 1) // page + 2
        self.slots = torch.randperm(self.pages * page, generator=g)[:tokens]
        self.positions = torch.randint(0, 500, (tokens,), generator=g, dtype=torch.int32)
        self.cos, self.sin = _tables(500, rot)
        self.qw, self.kw = (torch.randn(d, generator=g) * 0.3 + 1 for _ in range(2))
        self.rot = rot
        self.bytes = M.mipgemm_kv4_bytes(self.pages, page, hkv, d)
        assert self.bytes == self.pages * page * hkv * d * 9 // 8

    def parts(self):
        q, k, v = self.hq * self.d, self.hkv * self.d, self.hkv * self.d
        x = self.x
        return (x[:, :q].reshape(-1, self.hq, self.d), x[:, q:q + k].reshape(-1, self.hkv, self.d),
                x[:, q + k:q + k + v].reshape(-1, self.hkv, self.d))

    def run(self, M, style, weights=True, eps=1e-5, cache=True, keys=False, in_place=False, slots=None, positions=None):
        import torch
        hq, hkv, d = self.hq, self.hkv, self.d
        x = self.x.cuda()
        # (the tail is for writes past the end)
        self.cache = torch.full((self.bytes + 64,), 0xA5, dtype=torch.uint8, device="cuda")
        qo = x if in_place else torch.full((self.tokens, hq * d + 3), 9.0, dtype=x.dtype, device="cuda")
        ko = torch.full((self.tokens, hkv * d + 1), 9.0, dtype=x.dtype, device="cuda") if keys else None
        slots = (self.slots if slots is None else slots).cuda()
        positions = (self.positions if positions is None else positions).cuda()
        qw, kw = (self.qw.cuda(), self.kw.cuda()) if weights else (None, None)
        cos, sin = self.cos.cuda(), self.sin.cuda()
        M.mipgemm_qk_norm_rope(self.tokens, hq, hkv, d, self.kind, x, self.ld, x[:, hq * d:], self.ld, x[:, (hq + hkv) * d:],
                               self.ld, qw, kw, eps, cos, sin, 500, self.rot, style, positions, qo, qo.stride(0), ko,
                               hkv * d + 1, self.cache if cache else None, self.bytes, self.pages, self.page, slots)
        torch.cuda.synchronize()
        assert (self.cache[self.bytes:] == 0xA5).all()
        if not in_place:
            assert (qo[:, hq * d:] == 9).all()
        return qo[:, :hq * d].cpu().reshape(-1, hq, d), None if ko is None else ko[:, :hkv * d].cpu().reshape(-1, hkv, d)

    def read(self, M, slots=None):
        import torch
        slots = (self.slots if slots is None else slots).cuda()
        n, w = slots.numel(), self.hkv * self.d
        k, v = (torch.full((n, w + 2), 5.0, dtype=R.TORCH[self.kind], device="cuda") for _ in range(2))
        M.mipgemm_kv4_read(n, self.hkv, self.d, self.kind, self.cache, self.bytes, self.pages, self.page, slots, k, w + 2, v, w + 2)
        torch.cuda.synchronize()
        assert (k[:, w:] == 5).all() and (v[:, w:] == 5).all()
        return k[:, :w].cpu().reshape(-1, self.hkv, self.d), v[:, :w].cpu().reshape(-1, self.hkv, self.d)


def _close(got, want, size, kind, steps):
    """steps: float32 roundings on the way, of numbers up to `size`."""
    bound = steps * 2.0 ** -24 * size + R.rounding(want, kind)
    return bool(((got.double() - want).abs() <= bound).all())


CASES = [(1, 1, 1, 64, 16, 64), (5, 4, 2, 64, 32, 32), (33, 8, 8, 64, 16, 22), (7, 8, 2, 128, 64, 128), (130, 32, 8, 128, 16, 64),
         (3, 5, 1, 128, 1024, 2), (9, 4, 4, 256, 32, 256), (65, 16, 2, 256, 128, 100), (300, 3, 3, 128, 64, 0)]


@pytest.mark.parametrize("case", CASES, ids=str)
@pytest.mark.parametrize("kind", [F32, BF16, F16])
@pytest.mark.parametrize("style", [0, 1])
def test_heads_into_the_cache(gpu, case, kind, style):
    tokens, hq, hkv, d, page, rot = case
    t = Heads(gpu, tokens, hq, hkv, d, kind, page, rot, seed=tokens, pad=5)
    for weights in (True, False):
        q, k = t.run(gpu, style, weights=weights, keys=True)
        xq, xk, xv = t.parts()
        at = t.positions.long()
        wq = _normed_and_rotated(xq, t.qw if weights else None, 1e-5, t.cos[at], t.sin[at], rot, style)
        wk = _normed_and_rotated(xk, t.kw if weights else None, 1e-5, t.cos[at], t.sin[at], rot, style)
        # a pair's own size bounds what the rotation adds up
        size = wq.abs().amax(-1, keepdim=True) * 2
        assert _close(q, wq, size, kind, d / 8 + 16)
        assert _close(k, wk, size.amax() * 0, kind, 0)  # keys are worked out in float64
        kb, vb = t.read(gpu)
        hk, hv = R.held(wk), R.held(xv.double())
        assert ((kb.double() - hk).abs() <= R.rounding(hk, kind)).all()
        assert ((vb.double() - hv).abs() <= R.rounding(hv, kind)).all()


@pytest.mark.parametrize("d, page", [(64, 16), (128, 32), (256, 64)])
def test_layout_of_the_cache(gpu, d, page):
    import torch
    t = Heads(gpu, 2 * page, 2, 3, d, F32, page, 0)
    t.pages, t.slots = 2, torch.arange(2 * page)
    t.bytes = gpu.mipgemm_kv4_bytes(2, page, 3, d)
    t.run(gpu, 0, weights=False)
    _, xk, xv = t.parts()
    want = R.cache_bytes(xk.double(), xv.double(), page)
    assert np.array_equal(t.cache[:t.bytes].cpu().numpy(), want.reshape(-1))


def test_groups_that_are_no_ordinary_numbers(gpu):
    import torch
    t = Heads(gpu, 12, 1, 1, 128, F32, 16, 0)
    _, _, v = t.parts()
    v = v[:, 0]
    v[0] = 0
    v[1] = 3.75
    v[2, 5] = float("inf")
    v[3, 40] = float("nan")
    v[4] *= 1e-6
    v[5] *= 1e5
    v[6] += 1000
    v[7] = -1e-9
    v[8, :32] = torch.arange(32) - 15.0    # a range that ends on codes
    v[9] = torch.where(torch.arange(128) % 2 == 0, 60000.0, -60000.0)
    v[10] = torch.linspace(0, 1, 128)
    t.x[:, 256:384] = v
    t.run(gpu, 0, weights=False)
    _, got = t.read(gpu)
    want = R.held(v.double())
    got = got[:, 0].double()
    assert torch.equal(torch.isnan(got), torch.isnan(want))
    assert torch.isnan(got[2, :32]).all() and torch.isfinite(got[2, 32:]).all()
    ok = ~torch.isnan(want)
    assert torch.equal(got[ok], want[ok])
    assert (got[0] == 0).all() and (got[7].abs() <= 2.0 ** -17).all()
    # half a step: the step's rounding up, the zero point's rounding and the cut at 15 leave less than a whole one
    v = v.double().clamp(-R.TOP, R.TOP).reshape(12, 4, 32)
    step = torch.maximum((v.amax(-1) - v.amin(-1)) / 15, v.abs().amax(-1) / 112).clamp_min(2.0 ** -17) * 1.125 + 2.0 ** -17
    off = (got.reshape(12, 4, 32) - v).abs()
    fine = torch.isfinite(off)
    assert (off[fine] <= step[..., None].expand_as(off)[fine]).all()


def test_tokens_without_a_slot_or_a_position(gpu):
    import torch
    t = Heads(gpu, 40, 4, 2, 64, BF16, 16, 64)
    slots, positions = t.slots.clone(), t.positions.clone()
    slots[3], slots[7] = -1, t.pages * t.page
    slots[9] = 1 << 40
    positions[5], positions[6], positions[8] = -1, 500, 2 ** 31 - 1
    q, _ = t.run(gpu, 0, slots=slots, positions=positions)
    lost = torch.zeros(40, dtype=torch.bool)
    lost[[5, 6, 8]] = True
    assert torch.isnan(q[lost]).all() and torch.isfinite(q[~lost]).all()
    kb, vb = t.read(gpu, slots)
    for i in (3, 7, 9):
        assert (kb[i] == 0).all() and (vb[i] == 0).all()
    assert torch.isnan(kb[lost]).all() and torch.isfinite(kb[~lost]).all() and torch.isfinite(vb).all()
    # every byte of the slots that no token has keeps what it held
    touched = torch.zeros(t.pages * t.page, dtype=torch.bool)
    touched[slots[(slots >= 0) & (slots < t.pages * t.page)]] = True
    free = torch.nonzero(~touched).flatten()
    k2, _ = t.read(gpu, free)
    blank = torch.full((1,), 0xA5, dtype=torch.uint8)
    n, code, z = 0xA5 & 15, 0xA5, np.int8(np.uint8(0xA5))
    s = float(np.uint16(code << 7).view(np.float16))
    assert set(np.unique(k2.double().numpy())) <= {float(torch.tensor(s * (a - int(z))).to(torch.bfloat16)) for a in (5, 10)}
    del blank, n


def test_queries_in_place_and_without_keys(gpu):
    t = Heads(gpu, 50, 6, 2, 128, BF16, 16, 128)
    q1, _ = t.run(gpu, 0)
    q2, _ = t.run(gpu, 0, in_place=True)
    assert (q1 == q2).all()
    q3, k3 = t.run(gpu, 0, cache=False, keys=True)
    assert (q1 == q3).all() and k3 is not None
    assert (t.cache == 0xA5).all()


@pytest.mark.parametrize("d", [64, 256])
def test_queries_alone_beside_a_cache(gpu, d):
    """Without key heads nothing goes into a cache that is given, and no slots are asked for."""
    import torch
    t = Heads(gpu, 70, 6, 2, d, BF16, 16, d)
    want, _ = t.run(gpu, 0, cache=False)
    x, qw, cos, sin, at = t.x.cuda(), t.qw.cuda(), t.cos.cuda(), t.sin.cuda(), t.positions.cuda()
    cache = torch.full((256,), 0xA5, dtype=torch.uint8, device="cuda")
    out = torch.full((70, 6 * d), 9.0, dtype=torch.bfloat16, device="cuda")
    gpu.mipgemm_qk_norm_rope(70, 6, 0, d, BF16, x, t.ld, None, 1, None, 1, qw, None, 1e-5, cos, sin, 500, d, 0, at, out, 6 * d,
                             None, 1, cache, 256, t.pages, 16, None)
    torch.cuda.synchronize()
    assert torch.equal(out.cpu().reshape(-1, 6, d), want) and (cache == 0xA5).all()


@pytest.mark.parametrize("kind", [F32, BF16])
@pytest.mark.parametrize("d, rot, style", [(64, 64, 0), (128, 22, 1), (256, 128, 0)])
@pytest.mark.parametrize("eps", [0.0, 1e-30, 1e-5])
def test_heads_of_extreme_size(gpu, kind, d, rot, style, eps):
    """Squares that float32 cannot hold, or holds to few bits, do not reach the result."""
    import torch
    t = Heads(gpu, 12, 3, 9, d, kind, 16, rot, seed=31)
    by = torch.tensor([1e17, 1e18, 1e19, 1e20, 1e30, 2e37, 1e-17, 1e-20, 1e-22, 1e-25, 1e-30, 1e-35], dtype=torch.float64)
    t.x = (torch.randn(t.x.shape, generator=torch.Generator().manual_seed(32), dtype=torch.float64) * by[:, None]).to(R.TORCH[kind])
    at = t.positions.long()
    xq, xk, xv = t.parts()
    for weights in (True, False):
        q, _ = t.run(gpu, style, weights=weights, eps=eps)
        wq = _normed_and_rotated(xq, t.qw if weights else None, eps, t.cos[at], t.sin[at], rot, style)
        wk = _normed_and_rotated(xk, t.kw if weights else None, eps, t.cos[at], t.sin[at], rot, style)
        size = wq.abs().amax(-1, keepdim=True) * 2
        assert _close(q, wq, size, kind, d / 8 + 16), weights
        kb, vb = t.read(gpu)
        hk, hv = R.held(wk), R.held(xv.double())
        assert ((kb.double() - hk).abs() <= R.rounding(hk, kind)).all(), weights
        assert ((vb.double() - hv).abs() <= R.rounding(hv, kind)).all(), weights


@pytest.mark.parametrize("weights", [True, False])
def test_keys_past_float32_before_they_are_cut(gpu, weights):
    """A rotation can add two finite channels up to more than float32 holds: such keys are cut, as all others."""
    import torch
    t = Heads(gpu, 5, 1, 2, 128, F32, 16, 128, seed=33)
    t.x[:] = 3e38 * torch.sign(t.x)
    at = t.positions.long()
    _, xk, _ = t.parts()
    t.kw *= 1.5
    t.run(gpu, 0, weights=weights)
    hk = R.held(_normed_and_rotated(xk, t.kw if weights else None, 1e-5, t.cos[at], t.sin[at], 128, 0))
    kb, _ = t.read(gpu)
    assert torch.isfinite(hk).all() and torch.equal(kb.double(), hk)


@pytest.mark.parametrize("d, rot", [(64, 64), (128, 32), (128, 22), (256, 64), (256, 2)])
@pytest.mark.parametrize("style", [0, 1])
def test_positions_outside_the_tables(gpu, d, rot, style):
    """Queries and keys of such a token are NaN in all their channels, rotated or not; its values are as they were."""
    import torch
    t = Heads(gpu, 40, 3, 2, d, BF16, 16, rot, seed=35)
    positions = t.positions.clone()
    positions[5], positions[6], positions[8] = -1, 500, -2 ** 31
    lost = torch.zeros(40, dtype=torch.bool)
    lost[[5, 6, 8]] = True
    for keys in (False, True):
        q, k = t.run(gpu, style, positions=positions, keys=keys)
        assert torch.isnan(q[lost]).all() and torch.isfinite(q[~lost]).all()
        if keys:
            assert torch.isnan(k[lost]).all() and torch.isfinite(k[~lost]).all()
        kb, vb = t.read(gpu)
        assert torch.isnan(kb[lost]).all() and torch.isfinite(kb[~lost]).all() and torch.isfinite(vb).all()


def _matrix(gpu, tokens, hq, hkv, d, kind, seed):
    """Tokens enough for a workgroup each, made on the device."""
    import torch
    t = Heads(gpu, 1, hq, hkv, d, kind, 64, d, seed=seed)
    g = torch.Generator(device="cuda").manual_seed(seed)
    t.tokens, t.pages = tokens, (tokens + 63) // 64 + 2
    t.x = (torch.randn((tokens, t.ld), generator=g, device="cuda") * torch.exp(torch.randn((tokens, 1), generator=g, device="cuda"))).to(R.TORCH[kind])
    t.slots = torch.randperm(t.pages * 64, generator=g, device="cuda")[:tokens]
    t.positions = torch.randint(0, 500, (tokens,), generator=g, device="cuda", dtype=torch.int32)
    t.bytes = gpu.mipgemm_kv4_bytes(t.pages, 64, hkv, d)
    return t


@pytest.mark.parametrize("kind", [F32, BF16, F16])
@pytest.mark.parametrize("hq, hkv, d, rot, style", [(37, 9, 128, 128, 0), (70, 21, 64, 64, 1), (13, 5, 256, 96, 0), (9, 40, 128, 22, 0)])
def test_heads_of_many_tokens(gpu, kind, hq, hkv, d, rot, style):
    """From 2048 tokens on a wave takes several turns of heads: four and five here, of mixed kinds."""
    import torch
    t = _matrix(gpu, 2100, hq, hkv, d, kind, seed=51)
    t.rot, (t.cos, t.sin) = rot, _tables(500, rot)
    at = t.positions.long()
    xq, xk, xv = t.parts()
    cos, sin = t.cos.cuda()[at], t.sin.cuda()[at]
    for weights in (True, False):
        wq = _normed_and_rotated(xq, t.qw.cuda() if weights else None, 1e-5, cos, sin, rot, style)
        wk = _normed_and_rotated(xk, t.kw.cuda() if weights else None, 1e-5, cos, sin, rot, style)
        hk, hv = R.held(wk), R.held(xv.double())
        for keys in (False, True):
            q, k = t.run(gpu, style, weights=weights, keys=keys)
            assert _close(q.cuda(), wq, wq.abs().amax(-1, keepdim=True) * 2, kind, d / 8 + 16)
            assert k is None or _close(k.cuda(), wk, 0, kind, 0)
            kb, vb = t.read(gpu)
            assert ((kb.cuda().double() - hk).abs() <= R.rounding(hk, kind)).all()
            assert ((vb.cuda().double() - hv).abs() <= R.rounding(hv, kind)).all()


@pytest.mark.parametrize("hkv", [512, 520])
def test_as_many_heads_as_a_wave_has_turns(gpu, hkv):
    """1024 heads of queries and 512 of keys and values are 64 turns of each of four waves; more go to another workgroup."""
    import torch
    hq, d = 1024, 64
    t = _matrix(gpu, 2048, hq, hkv, d, BF16, seed=52)
    at = t.positions.long()
    xq, xk, xv = t.parts()
    wk = _normed_and_rotated(xk, t.kw.cuda(), 1e-5, t.cos.cuda()[at], t.sin.cuda()[at], d, 0)
    hk, hv = R.held(wk), R.held(xv.double())
    q, _ = t.run(gpu, 0)
    wq = _normed_and_rotated(xq, t.qw.cuda(), 1e-5, t.cos.cuda()[at], t.sin.cuda()[at], d, 0)
    assert _close(q.cuda(), wq, wq.abs().amax(-1, keepdim=True) * 2, BF16, d / 8 + 16)
    kb, vb = t.read(gpu)
    assert ((kb.cuda().double() - hk).abs() <= R.rounding(hk, BF16)).all()
    assert ((vb.cuda().double() - hv).abs() <= R.rounding(hv, BF16)).all()


@pytest.mark.parametrize("tokens, hq, hkv, d, style", [(50, 6, 2, 128, 0), (50, 5, 3, 64, 1), (2100, 37, 9, 128, 0), (2100, 13, 5, 256, 1)])
def test_queries_and_keys_in_place(gpu, tokens, hq, hkv, d, style):
    import torch
    t = _matrix(gpu, tokens, hq, hkv, d, BF16, seed=53)
    # (a head whose squares float32 cannot hold goes through the pass in float64, also in place)
    t.x[3, :d] *= 1e20
    t.x[4, hq * d:(hq + 1) * d] *= 1e20
    q, k = t.run(gpu, style, keys=True)
    apart = t.cache.clone()
    x, cache = t.x.clone(), torch.full_like(t.cache, 0xA5)
    keys = x[:, hq * d:]
    gpu.mipgemm_qk_norm_rope(tokens, hq, hkv, d, BF16, x, t.ld, keys, t.ld, x[:, (hq + hkv) * d:], t.ld, t.qw.cuda(), t.kw.cuda(), 1e-5,
                             t.cos.cuda(), t.sin.cuda(), 500, d, style, t.positions, x, t.ld, keys, t.ld, cache, t.bytes, t.pages, 64, t.slots)
    torch.cuda.synchronize()
    assert torch.equal(x[:, :hq * d].cpu().reshape(-1, hq, d), q) and torch.equal(x[:, hq * d:(hq + hkv) * d].cpu().reshape(-1, hkv, d), k)
    assert torch.equal(x[:, (hq + hkv) * d:], t.x[:, (hq + hkv) * d:]) and torch.equal(cache, apart)


# ---- attention ----

class Cached:
    """Requests with ragged lengths over a cache of random rows, the rows in float64 beside it."""

    def __init__(self, lengths, hkv, d, page, seed=0, spread=1.0, extra=3, stale=0xFF):
        import torch
        g = torch.Generator().manual_seed(seed)
        self.lengths, self.hkv, self.d, self.page = lengths, hkv, d, page
        used = [(n + page - 1) // page for n in lengths]
        self.pages = sum(used) + extra
        order = torch.randperm(self.pages, generator=g)
        width = max(used + [1])
        self.table = torch.full((len(lengths), width), -7, dtype=torch.int32)
        keys = torch.randn((self.pages * page, hkv, d), generator=g, dtype=torch.float64) * spread
        values = torch.randn((self.pages * page, hkv, d), generator=g, dtype=torch.float64) + 0.5
        at, live = 0, torch.zeros(self.pages * page, dtype=torch.bool)
        self.rows = []
        for r, u in enumerate(used):
            mine = order[at:at + u]
            at += u
            self.table[r, :u] = mine.to(torch.int32)
            slots = (mine[:, None] * page + torch.arange(page)).flatten()[:lengths[r]]
            live[slots] = True
            self.rows.append(slots)
        self.keys, self.values = R.held(keys).cuda(), R.held(values).cuda()
        cache = R.cache_bytes(keys, values, page) if self.pages * page * hkv * d < 40000 else _cache_bytes(keys.cuda(), values.cuda(), page)
        # what no request holds is no number
        self.cache = torch.from_numpy(cache.reshape(self.pages, hkv, -1)) if isinstance(cache, np.ndarray) else cache
        self.cache = _stale(self.cache, live, page, d, stale).cuda()

    def run(self, M, q, queries, kind, scale, split=True, max_q=None, max_kv=None, stride_pad=0):
        import torch
        rows, heads = q.shape[0], q.shape[1]
        w = heads * self.d
        starts = torch.tensor([0] + list(queries)).cumsum(0).to(torch.int32).cuda()
        lengths = torch.tensor(self.lengths, dtype=torch.int32).cuda()
        out = torch.full((rows + 2, w + 8), 4.0, dtype=R.TORCH[kind], device="cuda")
        qd = torch.zeros((rows, w + 8), dtype=R.TORCH[kind], device="cuda")
        qd[:, :w] = q.reshape(rows, w).to(R.TORCH[kind])
        max_q = max(list(queries) + [1]) if max_q is None else max_q
        max_kv = max(self.lengths + [1]) if max_kv is None else max_kv
        need = M.mipgemm_attention_kv4_workspace_size(len(self.lengths), heads, self.hkv, self.d, max_q, max_kv) if split else 0
        ws = torch.full((need + 64,), 0xFF, dtype=torch.uint8, device="cuda")
        M.mipgemm_attention_kv4(len(self.lengths), heads, self.hkv, self.d, kind, qd, w + 8, rows, starts, max_q, lengths, max_kv,
                                self.cache, self.cache.numel(), self.pages, self.page, self.table.cuda(), self.table.shape[1],
                                scale, out, w + 8, workspace=ws if need else None, workspace_bytes=need)
        torch.cuda.synchronize()
        assert (out[rows:] == 4).all() and (out[:, w:] == 4).all() and (ws[need:] == 0xFF).all()
        return out[:rows, :w].double().reshape(rows, heads, self.d)

    def exact(self, q, queries, scale):
        import torch
        heads, at, out = q.shape[1], 0, []
        for r, n in enumerate(queries):
            got = torch.zeros((n, heads, self.d), dtype=torch.float64, device="cuda")
            for h in range(heads):
                slots = self.rows[r].cuda()
                kv = h // (heads // self.hkv)
                if n and len(slots):
                    got[:, h] = R.attention(q[at:at + n, h].double().cuda(), self.keys[slots, kv], self.values[slots, kv], scale)
            out.append(got)
            at += n
        return torch.cat(out)


def _cache_bytes(keys, values, page):
    """R.cache_bytes with tensor operations, for large caches."""
    import torch
    out = []
    for which, x in enumerate((keys, values)):
        slots, heads, d = x.shape
        n, s, z = R.encode(x)
        n = n.reshape(-1, page, heads, d // 2, 2).to(torch.uint8)
        b = n[..., 0] | (n[..., 1] << 4)
        b = b.reshape(-1, page // 4, 4, heads, d // 8, 4).permute(0, 3, 1, 4, 2, 5) if which else b.permute(0, 2, 1, 3)
        code = (s.to(torch.float16).view(torch.int16).to(torch.int32) >> 7).to(torch.uint8)
        pairs = torch.stack((code, z.to(torch.int8).view(torch.uint8)), -1).reshape(-1, page, heads, d // 32, 2).permute(0, 2, 3, 1, 4)
        out += [b.reshape(b.shape[0], heads, -1), pairs.reshape(b.shape[0], heads, -1)]
    return torch.cat(out, -1)


def _stale(cache, live, page, d, byte):
    """Every byte of the slots that are not live set to `byte`."""
    import torch
    cache = cache.clone()
    pages, heads, _ = cache.shape
    dead = ~live.reshape(pages, page).to(cache.device)
    at = 0
    for which in (0, 1):
        codes = cache[..., at:at + page * d // 2]
        at += page * d // 2
        pairs = cache[..., at:at + page * d // 16]
        at += page * d // 16
        if which:
            codes = codes.reshape(pages, heads, page // 4, d // 8, 4, 4).permute(0, 1, 2, 4, 3, 5).reshape(pages, heads, page, d // 2).clone()
            codes[dead[:, None].expand(pages, heads, page)] = byte
            cache[..., at - page * d // 16 * 9:at - page * d // 16] = codes.reshape(pages, heads, page // 4, 4, d // 8, 4).permute(
                0, 1, 2, 4, 3, 5).reshape(pages, heads, -1)
        else:
            codes = codes.reshape(pages, heads, page, d // 2).clone()
            codes[dead[:, None].expand(pages, heads, page)] = byte
            cache[..., at - page * d // 16 * 9:at - page * d // 16] = codes.reshape(pages, heads, -1)
        pairs = pairs.reshape(pages, heads, d // 32, page, 2).clone()
        pairs[dead[:, None, None].expand(pages, heads, d // 32, page)] = byte
        cache[..., at - page * d // 16:at] = pairs.reshape(pages, heads, -1)
    return cache.contiguous()


def _check(M, lengths, queries, heads, hkv, d, kind, page, seed=0, spread=1.0, scale=None, q=None, splits=(True, False), **more):
    import torch
    c = Cached(lengths, hkv, d, page, seed, spread)
    scale = d ** -0.5 if scale is None else scale
    if q is None:
        q = torch.randn((sum(queries), heads, d), generator=torch.Generator().manual_seed(seed + 1))
    q = q.to(R.TORCH[kind])
    want = c.exact(q, queries, scale)
    # p is rounded to float16 (relative 2^-12 each), scores to float32 (their size times 2^-22 moves p by as
    # much): together no more than this of the largest value a row can average, then the output's own rounding
    size = c.values.abs().amax()
    top = float((q.double().abs().amax() * c.keys.abs().amax() * d * scale).item())
    bound = (2.0 ** -11 + 2.0 ** -20 * (top + 4)) * size + R.rounding(want, kind)
    for split in splits:
        got = c.run(M, q, queries, kind, scale, split=split, **more)
        off = (got - want).abs()
        assert torch.isfinite(got).all()
        assert (off <= bound).all(), (split, float(off.max()), float((off / bound).max()))
        # and over all of them far less
        if want.numel() and float(want.norm()):
            assert float((got - want).norm() / want.norm()) <= 4 * (R.UNIT[kind] + 2.0 ** -12)


@pytest.mark.parametrize("d", [64, 128, 256])
@pytest.mark.parametrize("kind", [BF16, F16])
@pytest.mark.parametrize("page", [16, 128])
def test_single_tokens(gpu, d, kind, page):
    _check(gpu, [1, 15, 16, 17, 31, 33, 127, 129, 640, 2049, 0], [1] * 10 + [0], 8, 2, d, kind, page)


@pytest.mark.parametrize("heads, hkv", [(1, 1), (16, 16), (7, 1), (32, 2), (40, 8), (48, 1)])
def test_head_layouts(gpu, heads, hkv):
    _check(gpu, [700, 90], [1, 1], heads, hkv, 64, BF16, 32)
    _check(gpu, [200, 90], [3, 70], heads, hkv, 128, F16, 32)


@pytest.mark.parametrize("d", [64, 128, 256])
@pytest.mark.parametrize("kind", [BF16, F16])
@pytest.mark.parametrize("queries", [[2, 5, 1], [4, 9, 3], [17, 33, 64], [100, 1, 257]])
def test_several_tokens(gpu, d, kind, queries):
    _check(gpu, [n + e for n, e in zip(queries, (0, 300, 63))], queries, 8, 4, d, kind, 64)


@pytest.mark.parametrize("d", [64, 128, 256])
def test_a_prompt_from_its_start(gpu, d):
    _check(gpu, [1, 130, 513], [1, 130, 513], 4, 2, d, BF16, 16)


def test_rows_that_see_nothing(gpu):
    # more queries than keys: the first of them come before every key
    _check(gpu, [3, 0, 40, 20], [9, 5, 40, 100], 4, 2, 64, BF16, 16)
    _check(gpu, [130, 0], [300, 70], 2, 1, 128, F16, 16)
    _check(gpu, [0], [1], 2, 1, 128, F16, 16)


def test_scores_far_apart(gpu):
    # one key takes nearly all of a row, wherever it stands, and the running maximum moves often
    _check(gpu, [900, 300], [1, 40], 4, 2, 64, BF16, 32, spread=30.0, scale=1.0)
    _check(gpu, [900, 300], [1, 200], 4, 2, 128, F16, 32, spread=0.001)


def test_queries_of_extreme_size(gpu):
    import torch
    q = torch.randn((4, 4, 64), generator=torch.Generator().manual_seed(3))
    q[0] *= 1e30
    q[1] *= 1e-30
    q[2] = 0
    q[3, :, 0] = 1e20
    c = Cached([50, 60, 70, 80], 2, 64, 16)
    q = q.to(torch.bfloat16)
    for split in (True, False):
        got = c.run(gpu, q, [1] * 4, BF16, 0.125, split=split)
        want = c.exact(q, [1] * 4, 0.125)
        # (scores of 1e30: all of the weight on one key, or on keys whose scores are equal)
        assert torch.isfinite(got).all()
        assert float((got - want).abs().max()) <= 2.0 ** -6 * float(want.abs().max())


@pytest.mark.parametrize("d, queries", [(64, 1), (128, 40), (128, 200), (256, 90)])
@pytest.mark.parametrize("kind", [BF16, F16])
def test_scales_at_both_ends(gpu, d, queries, kind):
    """Queries of zeros weigh all keys alike, whatever the scale; so does every query at the smallest."""
    import torch
    c = Cached([300], 2, d, 16, seed=45)
    q = torch.zeros((queries, 4, d))
    want = c.exact(q, [queries], 1.0)
    for scale in (3.4e38, 1e-45, 1e-38):
        got = c.run(gpu, q, [queries], kind, scale)
        assert float((got - want).norm() / want.norm()) <= 2.0 ** -8, scale
    got = c.run(gpu, q + 1, [queries], kind, 1e-45)
    assert float((got - want).norm() / want.norm()) <= 2.0 ** -8


def test_no_number_among_queries_stays_in_its_row(gpu):
    import torch
    c = Cached([300, 90], 2, 128, 16)
    q = torch.randn((60, 4, 128), generator=torch.Generator().manual_seed(4)).to(torch.bfloat16)
    clean = c.run(gpu, q, [40, 20], BF16, 0.1)
    q[7, 1, 5], q[50, 3, 0] = float("nan"), float("inf")
    got = c.run(gpu, q, [40, 20], BF16, 0.1)
    bad = torch.isnan(got).all(-1)
    assert bad[7, 1] and bad[50, 3] and int(bad.sum()) == 2
    assert torch.equal(got[~bad], clean[~bad])


def test_bounds_of_the_host_hold(gpu):
    """Numbers on the device beyond what the host was told are cut, pages that are none are not seen."""
    import torch
    c = Cached([100, 64], 2, 64, 16)
    q = torch.randn((2, 4, 64), generator=torch.Generator().manual_seed(5)).to(torch.bfloat16)
    want = c.exact(q, [1, 1], 0.125)
    lengths, c.lengths = c.lengths, [100, 10 ** 9]
    got = c.run(gpu, q, [1, 1], BF16, 0.125, max_kv=100)      # the second's table names four pages and three that are none
    assert float((got[0] - want[0]).abs().max()) <= 2.0 ** -6 * float(want.abs().max())
    assert float((got[1] - want[1]).abs().max()) <= 2.0 ** -6 * float(want.abs().max())
    c.lengths = [-5, 64]
    got = c.run(gpu, q, [1, 1], BF16, 0.125)
    assert (got[0] == 0).all()
    c.lengths = lengths
    c.table[0, 3] = 10 ** 6                                   # a page number outside the cache: its sixteen keys are not seen
    keep = torch.cat((c.rows[0][:48], c.rows[0][64:]))
    c.rows[0] = keep
    got = c.run(gpu, q, [1, 1], BF16, 0.125)
    want = c.exact(q, [1, 1], 0.125)
    assert float((got - want).abs().max()) <= 2.0 ** -6 * float(want.abs().max())


def test_a_cache_past_32_bits(gpu):
    """Pages whose bytes begin beyond 4 GB."""
    import torch
    page, hkv, d = 128, 8, 256
    pages = (5 << 30) // gpu.mipgemm_kv4_bytes(1, page, hkv, d)
    cache = torch.zeros(gpu.mipgemm_kv4_bytes(pages, page, hkv, d), dtype=torch.uint8, device="cuda")
    tokens = 200
    t = Heads(gpu, tokens, 8, hkv, d, BF16, page, 64)
    slots = torch.arange(tokens) + (pages - 2) * page
    x = t.x.cuda()
    qo = torch.empty((tokens, 8 * d), dtype=torch.bfloat16, device="cuda")
    cos, sin, at, sl = t.cos.cuda(), t.sin.cuda(), t.positions.cuda(), slots.cuda()
    gpu.mipgemm_qk_norm_rope(tokens, 8, hkv, d, BF16, x, t.ld, x[:, 8 * d:], t.ld, x[:, 16 * d:], t.ld, None, None, 0.0, cos, sin,
                             500, 64, 0, at, qo, 8 * d, None, 8 * d, cache, cache.numel(), pages, page, sl)
    k, v = (torch.empty((tokens, hkv * d), dtype=torch.float16, device="cuda") for _ in range(2))
    gpu.mipgemm_kv4_read(tokens, hkv, d, F16, cache, cache.numel(), pages, page, sl, k, hkv * d, v, hkv * d)
    _, _, xv = t.parts()
    assert torch.equal(v.cpu().double().reshape(tokens, hkv, d), R.held(xv.double()))
    table = torch.tensor([[pages - 2, pages - 1]], dtype=torch.int32, device="cuda")
    starts, lengths = torch.tensor([0, tokens], dtype=torch.int32, device="cuda"), torch.tensor([tokens], dtype=torch.int32, device="cuda")
    out = torch.empty_like(qo)
    gpu.mipgemm_attention_kv4(1, 8, hkv, d, BF16, qo, 8 * d, tokens, starts, tokens, lengths, tokens, cache, cache.numel(), pages,
                              page, table, 2, 0.0625, out, 8 * d)
    for h in range(8):
        want = R.attention(qo[:, h * d:(h + 1) * d].double(), k[:, h * d:(h + 1) * d].double(), v[:, h * d:(h + 1) * d].double(), 0.0625)
        got = out[:, h * d:(h + 1) * d].double()
        assert float((got - want).norm() / want.norm()) <= 2.0 ** -7


def test_attention_in_a_graph_over_growing_lengths(gpu):
    import torch
    c = Cached([700, 333], 2, 128, 64)
    q = torch.randn((2, 8, 128), generator=torch.Generator().manual_seed(6)).to(torch.bfloat16)
    qd, table = q.reshape(2, -1).cuda(), c.table.cuda()
    starts, lengths = torch.tensor([0, 1, 2], dtype=torch.int32).cuda(), torch.tensor([1, 1], dtype=torch.int32).cuda()
    need = gpu.mipgemm_attention_kv4_workspace_size(2, 8, 2, 128, 1, 700)
    assert need > 0
    ws, out = torch.empty(need + 16, dtype=torch.uint8, device="cuda"), torch.zeros((2, 1024), dtype=torch.bfloat16, device="cuda")

    def call(to):
        gpu.mipgemm_attention_kv4(2, 8, 2, 128, BF16, qd, 1024, 2, starts, 1, lengths, 700, c.cache, c.cache.numel(), c.pages, 64,
                                  table, c.table.shape[1], 0.09, to, 1024, workspace=ws, workspace_bytes=need + 16)
    call(out)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call(out)
    for n in ((1, 1), (40, 300), (513, 333), (700, 2)):
        lengths.copy_(torch.tensor(n, dtype=torch.int32))
        graph.replay()
        torch.cuda.synchronize()
        eager = torch.zeros_like(out)
        call(eager)
        torch.cuda.synchronize()
        assert torch.equal(out, eager), n
        rows = [r[:m] for r, m in zip(c.rows, n)]
        keep, c.rows = c.rows, rows
        want = c.exact(q, [1, 1], 0.09)
        c.rows = keep
        assert float((eager.double().reshape(2, 8, 128) - want).norm() / want.norm()) <= 2.0 ** -7
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            call(eager.zero_())
        side.synchronize()
        assert torch.equal(out, eager), n


@pytest.mark.parametrize("d", [64, 128, 256])
@pytest.mark.parametrize("queries", [1, 3, 9, 40, 200])
def test_a_value_that_is_no_number_reaches_only_what_sees_it(gpu, d, queries):
    """A group of a value that is NaN makes its 32 channels NaN where the token is seen, and changes nothing elsewhere."""
    import torch
    page, hkv, heads, keys = 32, 2, 8, 333
    c = Cached([keys, 50], hkv, d, page, seed=7)
    q = torch.randn((queries + 1, heads, d), generator=torch.Generator().manual_seed(8)).to(torch.bfloat16)
    clean = c.run(gpu, q, [queries, 1], BF16, d ** -0.5)
    assert torch.isfinite(clean).all()
    block, lost = page * d // 8 * 9, torch.zeros(clean.shape, dtype=torch.bool, device="cuda")
    for token, kv, g in ((keys - 1, 0, 0), (keys - queries // 2 - 1, 1, d // 32 - 1), (keys - queries, 1, 1), (keys - queries - 70, 0, 1)):
        if token < 0:
            continue
        slot = int(c.rows[0][token])
        c.cache.view(-1)[(slot // page * hkv + kv) * block + page * d // 16 * 17 + 2 * (g * page + slot % page)] = 0xFF
        first = max(token - (keys - queries), 0)  # the first query that sees it
        lost[first:queries, kv * (heads // hkv):(kv + 1) * (heads // hkv), 32 * g:32 * g + 32] = True
    for split in (True, False):
        got = c.run(gpu, q, [queries, 1], BF16, d ** -0.5, split=split)
        same = clean if split else got
        assert torch.equal(torch.isnan(got), lost), split
        assert torch.equal(got[~lost], same[~lost])
        want = clean[~lost]
        assert float((got[~lost] - want).norm() / want.norm()) <= 2.0 ** -7


@pytest.mark.parametrize("d", [64, 128, 256])
@pytest.mark.parametrize("page", [16, 32, 64, 256])
@pytest.mark.parametrize("queries", [1, 20, 150])
def test_pages_that_are_none(gpu, d, page, queries):
    """Keys of pages that the table does not name are not seen, whatever the number of rows."""
    import torch
    keys = 5 * page + 7
    queries = min(queries, keys)
    c = Cached([keys], 2, d, page, seed=9)
    q = torch.randn((queries, 8, d), generator=torch.Generator().manual_seed(10)).to(torch.float16)
    full = c.rows[0].clone()
    c.table[0, 1], c.table[0, 4] = -1, 2 ** 30
    got = c.run(gpu, q, [queries], F16, d ** -0.5)
    at = torch.arange(keys)
    there = (at // page != 1) & (at // page != 4)
    for i in range(queries):
        seen = there & (at <= keys - queries + i)
        if i not in (0, 1, queries // 2, queries - 1):
            continue
        slots = full[seen].cuda()
        for h in range(8):
            want = R.attention(q[i:i + 1, h].double().cuda(), c.keys[slots, h // 4], c.values[slots, h // 4], d ** -0.5)
            assert float((got[i, h] - want[0]).norm()) <= 2.0 ** -8 * float(c.values.abs().amax()) * d ** 0.5


def test_a_query_that_is_no_number_among_many(gpu):
    import torch
    c = Cached([500], 1, 128, 64, seed=11)
    q = torch.randn((300, 2, 128), generator=torch.Generator().manual_seed(12)).to(torch.bfloat16)
    clean = c.run(gpu, q, [300], BF16, 0.1)
    q[7, 1, 5], q[250, 0, 0] = float("nan"), float("inf")
    got = c.run(gpu, q, [300], BF16, 0.1)
    bad = torch.isnan(got).all(-1)
    assert bad[7, 1] and bad[250, 0] and int(bad.sum()) == 2
    # (the rows that share a wave with them take their queries unscaled: rounded otherwise, to no fewer bits)
    assert float((got[~bad] - clean[~bad]).norm() / clean[~bad].norm()) <= 2.0 ** -7


@pytest.mark.parametrize("d, queries", [(64, 1), (128, 3), (128, 170), (256, 40)])
def test_lengths_far_beyond_the_table(gpu, d, queries):
    """What a length says beyond the pages that a row of the table can name is not gone through."""
    import torch
    c = Cached([300, 37], 2, d, 16, seed=13)
    q = torch.randn((queries + 1, 8, d), generator=torch.Generator().manual_seed(14)).to(torch.bfloat16)
    c.lengths = [2 ** 31 - 5000, 37]
    width = c.table.shape[1] * 16
    for split in (True, False):
        got = c.run(gpu, q, [queries, 1], BF16, d ** -0.5, split=split, max_kv=2 ** 31 - 5000)
        # every query of the first request sees all of its table; what lies in the last page behind the 300 is no number
        assert torch.isnan(got[:queries]).all()
        want = c.exact(q[queries:], [0, 1], d ** -0.5)
        assert float((got[queries:] - want).norm() / want.norm()) <= 2.0 ** -7
    assert width == 304


@pytest.mark.parametrize("d", [64, 128, 256])
def test_many_rows_in_a_graph(gpu, d):
    import torch
    c = Cached([420, 90], 2, d, 64, seed=15)
    queries, rows = [200, 60], 260
    q = torch.randn((rows, 8, d), generator=torch.Generator().manual_seed(16)).to(torch.bfloat16)
    qd, table = q.reshape(rows, -1).cuda(), c.table.cuda()
    starts, lengths = torch.tensor([0, 200, 260], dtype=torch.int32).cuda(), torch.tensor(c.lengths, dtype=torch.int32).cuda()
    out = torch.zeros((rows, 8 * d), dtype=torch.bfloat16, device="cuda")

    def call(to):
        gpu.mipgemm_attention_kv4(2, 8, 2, d, BF16, qd, 8 * d, rows, starts, 200, lengths, 420, c.cache, c.cache.numel(), c.pages, 64,
                                  table, c.table.shape[1], d ** -0.5, to, 8 * d)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        call(out)
    for n in ((420, 90), (420, 60), (300, 80)):
        lengths.copy_(torch.tensor(n, dtype=torch.int32))
        out.zero_()
        graph.replay()
        torch.cuda.synchronize()
        eager = torch.zeros_like(out)
        call(eager)
        torch.cuda.synchronize()
        assert torch.equal(out, eager), n
        assert torch.isfinite(out).all() and float(out[199].abs().max()) > 0


@pytest.mark.parametrize("d", [64, 128, 256])
@pytest.mark.parametrize("scale", [1.0, 40.0])
def test_scores_far_apart_in_many_rows(gpu, d, scale):
    """Bases that move often, and (scale 40) past what a matrix instruction takes off the scores."""
    import torch
    queries = [150, 200]
    c = Cached([900, 300], 2, d, 32, seed=17, spread=30.0)
    q = torch.randn((350, 4, d), generator=torch.Generator().manual_seed(18)).to(torch.bfloat16)
    whole = float(np.float32(scale) * np.float32(1.4426950408889634))
    # (of more than 128 rows of 64 or 128 channels the queries are rounded to float16 with the scale in them)
    taken = q.double() if d == 256 else (q.float() * whole).half().double() / whole
    want = c.exact(taken, queries, scale)
    # scores in float32, their size times 2^-22 at most, move p by as much where two keys compete; p itself 2^-12
    size, top = c.values.abs().amax(), float((q.double().abs().amax() * c.keys.abs().amax() * d * scale).item())
    bound = (2.0 ** -11 + 2.0 ** -20 * (top + 4)) * size + R.rounding(want, BF16)
    for split in (True, False):
        got = c.run(gpu, q, queries, BF16, scale, split=split)
        assert torch.isfinite(got).all()
        assert ((got - want).abs() <= bound).all(), split
        assert float((got - want).norm() / want.norm()) <= 4 * (R.UNIT[BF16] + 2.0 ** -12)


@pytest.mark.parametrize("d", [64, 128, 256])
def test_queries_of_extreme_size_in_many_rows(gpu, d):
    import torch
    c = Cached([400], 1, d, 64, seed=19)
    q = torch.randn((300, 1, d), generator=torch.Generator().manual_seed(20))
    q[:40] *= 1e30
    q[40:80] *= 1e-30
    q[80:120] = 0
    q[120:160, :, 0] = 1e20
    q = q.to(torch.bfloat16)
    got, want = c.run(gpu, q, [300], BF16, 0.125), c.exact(q, [300], 0.125)
    assert torch.isfinite(got).all()
    assert float((got - want).abs().max()) <= 2.0 ** -6 * float(want.abs().max())


@pytest.mark.parametrize("d, queries", [(64, 1), (128, 40), (128, 200), (256, 90)])
def test_lengths_past_a_table_that_names_no_page(gpu, d, queries):
    """Rows whose length is beyond what the table can name, of which it names nothing: zeros."""
    import torch
    c = Cached([700, 40], 2, d, 16, seed=28)
    q = torch.randn((queries + 1, 4, d), generator=torch.Generator().manual_seed(29)).to(torch.bfloat16)
    c.table[0] = -1
    assert c.table.shape[1] * 16 == 704
    c.lengths[0] = 5000
    for split in (True, False):
        got = c.run(gpu, q, [queries, 1], BF16, 0.1, split=split)
        assert (got[:queries] == 0).all(), split
        want = c.exact(q[queries:], [0, 1], 0.1)
        assert float((got[queries:] - want).norm() / want.norm()) <= 2.0 ** -7


def _positive_keys(lengths, d, page, seed):
    """A cache whose keys are all positive, from about 1 on."""
    import torch
    c = Cached(lengths, 2, d, page, seed=seed)
    g = torch.Generator().manual_seed(seed + 1)
    keys = torch.randn(c.keys.shape, generator=g, dtype=torch.float64).abs().cuda() + 1
    values = torch.randn(c.keys.shape, generator=g, dtype=torch.float64).cuda() + 0.5
    c.keys, c.values = R.held(keys), R.held(values)
    assert float(c.keys.min()) > 0.5
    c.cache = _cache_bytes(keys, values, page)
    return c


@pytest.mark.parametrize("d, queries, keys", [(64, 1, 700), (256, 3, 700), (128, 20, 900), (128, 200, 900), (64, 300, 300), (256, 90, 700)])
@pytest.mark.parametrize("kind", [BF16, F16])
def test_a_query_that_is_no_number_against_keys_of_one_sign(gpu, d, queries, keys, kind):
    """All scores of such a row are minus infinity, or all of them infinity: NaN, unless the row sees no key."""
    import torch
    c = _positive_keys([keys, 1, 2], d, 16, seed=23)
    counts = [queries, 1, 4]  # (the first two of the last request's four come before its two keys)
    q = torch.randn((queries + 5, 4, d), generator=torch.Generator().manual_seed(25)).to(R.TORCH[kind])
    blind = torch.zeros((queries + 5, 4), dtype=torch.bool)
    blind[queries + 1:queries + 3] = True
    clean = {split: c.run(gpu, q, counts, kind, 0.1, split=split) for split in (True, False)}
    lost = torch.zeros_like(blind)
    inf = float("inf")
    for row, head, channel, x in ((0, 0, 3, -inf), (queries - 1, 1, d - 1, inf), (queries // 2, 2, 0, -inf), (queries, 3, 5, -inf),
                                  (queries, 0, 5, inf), (queries + 1, 1, 7, -inf), (queries + 2, 0, 7, inf), (queries + 3, 1, 7, -inf),
                                  (queries + 4, 2, 9, -inf), (queries + 4, 3, 9, inf)):
        q[row, head, channel] = x
        lost[row, head] = True
    if kind == BF16:  # finite, with scores past float32
        q[queries // 3, 3] = -3e38
        lost[queries // 3, 3] = True
    lost &= ~blind
    for split in (True, False):
        got = c.run(gpu, q, counts, kind, 0.1, split=split)
        assert torch.equal(torch.isnan(got).all(-1).cpu(), lost) and torch.equal(torch.isnan(got).any(-1).cpu(), lost), split
        assert (got[blind] == 0).all()
        # (the rows that share a wave with them may take their queries unscaled: rounded otherwise, to no fewer bits)
        fine = ~lost & ~blind
        assert float((got[fine] - clean[split][fine]).norm() / clean[split][fine].norm()) <= 2.0 ** -7


@pytest.mark.parametrize("d, queries", [(64, 1), (128, 40), (128, 200), (256, 90)])
def test_rows_all_of_whose_pages_are_none(gpu, d, queries):
    """Such a row sees no key, whatever its length: zeros, also of a query that is no number."""
    import torch
    c = Cached([700, 40], 2, d, 32, seed=26)
    q = torch.randn((queries + 1, 4, d), generator=torch.Generator().manual_seed(27)).to(torch.bfloat16)
    q[0, 1, 2], q[queries - 1, 2, 3] = float("inf"), float("nan")
    c.table[0] = -1
    c.table[0, 5] = c.pages
    for split in (True, False):
        got = c.run(gpu, q, [queries, 1], BF16, 0.1, split=split)
        assert (got[:queries] == 0).all(), split
        want = c.exact(q[queries:], [0, 1], 0.1)
        assert float((got[queries:] - want).norm() / want.norm()) <= 2.0 ** -7


@pytest.mark.parametrize("d, queries", [(64, 1), (64, 130)])
def test_as_many_keys_as_there_can_be(gpu, d, queries):
    """2^31 - 4097 keys, the most that is not refused: all in one page, but for the last 1023."""
    import torch
    page, keys, scale = 1024, 2 ** 31 - 4097, 0.125
    c = Cached([2 * page], 1, d, page, seed=37, extra=0)
    first, last = c.rows[0][:page].cuda(), c.rows[0][page:].cuda()
    # one head's queries take the last page's keys, the other's those of the page before
    towards = c.keys[last, 0].mean(0) - c.keys[first, 0].mean(0)
    towards = towards / towards.norm()
    spread = torch.randn((queries, 2, d), generator=torch.Generator().manual_seed(38), dtype=torch.float64).cuda()
    spread = spread - (spread @ towards)[..., None] * towards
    g = torch.randn((2 * page, d), generator=torch.Generator().manual_seed(39), dtype=torch.float64).cuda()
    near = torch.zeros((2 * page, 1, d), dtype=torch.float64, device="cuda")
    near[first, 0], near[last, 0] = g[:page] * 0.3, g[page:] * 0.3 + 8 * towards
    values = c.values.clone()
    values[last] -= 3
    c.cache, c.keys, c.values = _cache_bytes(near, values, page), R.held(near), R.held(values)
    q = spread.clone()
    q[:, 0] += 50 * towards      # scores near 50: e^50 against 2^31 keys
    q = q.to(torch.float16)
    width = (keys + page - 1) // page
    table = torch.full((1, width), int(first[0]) // page, dtype=torch.int32, device="cuda")
    table[0, -1] = int(last[0]) // page
    starts, lengths = (torch.tensor(x, dtype=torch.int32, device="cuda") for x in ([0, queries], [keys]))
    need = gpu.mipgemm_attention_kv4_workspace_size(1, 2, 1, d, queries, keys)
    assert need > 0
    ws, out = torch.empty(need, dtype=torch.uint8, device="cuda"), torch.zeros((queries, 2 * d), dtype=torch.float16, device="cuda")
    gpu.mipgemm_attention_kv4(1, 2, 1, d, F16, q, 2 * d, queries, starts, queries, lengths, keys, c.cache, c.cache.numel(), c.pages,
                              page, table, width, scale, out, 2 * d, workspace=ws, workspace_bytes=need)
    out = out.double().reshape(queries, 2, d)
    at, kept = torch.cat((first, last)), torch.arange(page, device="cuda")
    for i in (0, queries // 2, queries - 1):
        here = keys - queries + i + 1 - (width - 1) * page  # keys that the row sees of the last page
        times = torch.cat((torch.full((page,), float(width - 1), dtype=torch.float64, device="cuda"), (kept < here).double()))
        for h in range(2):
            p = torch.softmax(c.keys[at, 0] @ q[i, h].double() * scale + times.log(), 0)
            want = p @ c.values[at, 0]
            # two sums of so many additions in float32, each 2^-24 of them at most, p rounded to float16, scores to float32
            additions = 2 ** 31 // 1024 // 4 // 32 if queries == 1 else 2 ** 31 // 128 // 16
            bound = (2 * additions * 2.0 ** -24 + 2.0 ** -11 + 2.0 ** -20 * 100) * float(c.values.abs().amax()) + R.rounding(want, F16)
            assert ((out[i, h] - want).abs() <= bound).all(), (i, h, float((out[i, h] - want).abs().max()))
        assert float((out[i, 0] - out[i, 1]).norm()) > 1
