"""mipgemm_route against its definition in 64 bits: choices and rows bit for bit, weights within a few roundings."""
import numpy as np
import pytest

import layer_reference as R

pytestmark = pytest.mark.gpu

F32, BF16, F16 = 0, 1, 2
INF = float("inf")


@pytest.fixture(scope="module")
def gpu():
    import torch
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_2506_11728_amd as M
    M.load_library()
    return M


def _reference(x, bias, sigmoid, groups, top_groups, best, top, normalise, scale):
    """(ids, weights) in float64, token by token.  x: tokens x experts float64, bias float64 or None."""
    T, E = x.shape
    ids, weights = np.full((T, top), -1), np.zeros((T, top))
    b = np.zeros(E) if bias is None else bias
    each = E // groups
    for t in range(T):
        l = x[t]
        if np.isnan(l).any() or np.isnan(b).any() or (not sigmoid and l.max() == INF):
            weights[t] = np.nan
            continue
        free = (l > -INF) & (b > -INF)
        with np.errstate(over="ignore"):
            s = 1 / (1 + np.exp(-l)) if sigmoid else (np.exp(l - l.max()) if l.max() > -INF else np.zeros(E))
        whole = 1.0 if sigmoid else s.sum()
        if not sigmoid and whole > 0:
            s = s / whole
        # without a bias the order is that of the logits, also where float64 cannot tell the scores apart
        key = l if bias is None and (groups == 1 or best == 1) else s + b
        key = np.where(free, key, -INF)
        if groups > 1:
            part = -np.sort(-key.reshape(groups, each), 1)[:, :best]
            score = np.where(part[:, 0] > -INF, np.where(part > -INF, part, 0).sum(1), -INF)
            order = np.argsort(-score, kind="stable")[:top_groups]
            kept = np.zeros(groups, bool)
            kept[order] = True
            kept &= score > -INF
            key = np.where(np.repeat(kept, each), key, -INF)
        order = np.argsort(-key, kind="stable")[:top]
        order = order[key[order] > -INF]
        n = len(order)
        ids[t, :n] = order
        if n:
            w = s[order]
            if normalise:
                if sigmoid and l[order].max() > -600:
                    w = w / w.sum()
                else:
                    w = np.exp(l[order] - l[order].max())
                    w = w / w.sum()
            weights[t, :n] = scale * w
    return ids, weights


def _rows(ids, experts):
    flat = ids.reshape(-1)
    order = np.argsort(np.where(flat < 0, experts, flat), kind="stable")[:(flat >= 0).sum()]
    starts = np.searchsorted(flat[order], np.arange(experts + 1))
    places = np.full(flat.shape, -1)
    places[order] = np.arange(len(order))
    return starts, order, places.reshape(ids.shape)


def _route(M, x, kind, top, bias=None, sigmoid=False, groups=1, top_groups=1, best=1, normalise=True, scale=1.0, pad=0, plan=True,
           stream=None):
    """x: tokens x experts (float32 tensor).  Returns numpy ids, weights and, with a plan, starts, order, places."""
    import torch
    T, E = x.shape
    buf = torch.full((T, E + pad), 50.0).to(R.TORCH[kind])
    buf[:, :E] = x.to(R.TORCH[kind])
    d, b = buf.cuda(), None if bias is None else bias.cuda()
    ids = torch.full((T * top + 1,), -7, dtype=torch.int32, device="cuda")
    w = torch.full((T * top + 1,), -7.0, device="cuda")
    starts = torch.full((E + 2,), -7, dtype=torch.int32, device="cuda")
    order, places = torch.full_like(ids, -7), torch.full_like(ids, -7)
    need = M.mipgemm_route_workspace_size(T, E, top)
    ws = torch.full((need + 32,), 0x77, dtype=torch.uint8, device="cuda")
    M.mipgemm_route(T, E, top, d, E + pad, kind, b, int(sigmoid), groups, top_groups, best, int(normalise), scale, ids, w,
                    *((starts, order, places) if plan else (None, None, None)), workspace=ws, workspace_bytes=need, stream=stream)
    torch.cuda.synchronize()
    assert (ws[need:] == 0x77).all() and ids[-1] == -7 and w[-1] == -7 and order[-1] == -7 and places[-1] == -7 and starts[-1] == -7
    out = [t.cpu().numpy() for t in (ids[:-1].reshape(T, top), w[:-1].reshape(T, top))]
    return out + [t.cpu().numpy() for t in (starts[:-1], order[:-1], places[:-1].reshape(T, top))] if plan else out


def _check(M, x, kind, top, bias=None, scale=1.0, **how):
    got = _route(M, x, kind, top, bias=bias, scale=scale, **how)
    how = {k: v for k, v in how.items() if k not in ("pad", "plan", "stream")}
    x64 = x.to(R.TORCH[kind]).double().numpy()
    ref = dict(sigmoid=False, groups=1, top_groups=1, best=1, normalise=True)
    ref.update(how)
    ids, w = _reference(x64, None if bias is None else bias.double().numpy(), ref["sigmoid"], ref["groups"], ref["top_groups"], ref["best"],
                        top, ref["normalise"], scale)
    assert np.array_equal(got[0], ids), np.argwhere(got[0] != ids)[:5]
    lost = np.isnan(w)
    assert np.array_equal(np.isnan(got[1]), lost)
    # an exponential's argument, a difference of float32, is off by 2^-24 of itself and the exponential as much and 2^-23 more; sums
    # of at most 22 additions in a chain, of such exponentials; three roundings after.  Below 2^-120 float32 has fewer bits.
    finite = np.where(np.isfinite(x64), np.abs(x64), 0)
    span = 2 * finite.max(1, keepdims=True) if x64.size else 0
    bound = np.abs(w) * (2 * np.minimum(span, 200) + 60) * 2.0 ** -24 + 2.0 ** -120
    assert (np.abs(got[1] - w)[~lost] <= bound[~lost]).all(), np.nanmax(np.abs(got[1] - w) / bound)
    if len(got) > 2:
        starts, order, places = _rows(ids, x.shape[1])
        assert np.array_equal(got[2], starts) and np.array_equal(got[4], places)
        assert np.array_equal(got[3][:len(order)], order) and (got[3][len(order):] == -7).all()
    return got


def _normal(*shape, seed, spread=1.5):
    import torch
    return torch.randn(shape, generator=torch.Generator().manual_seed(seed)) * spread


@pytest.mark.parametrize("tokens", [1, 2, 31, 32, 33, 64, 65, 300])
@pytest.mark.parametrize("experts,top", [(1, 1), (4, 4), (8, 2), (60, 4), (64, 8), (65, 3), (100, 8), (128, 8), (200, 6), (256, 8), (511, 10),
                                         (512, 32), (1000, 9), (1024, 32)])
def test_routing(gpu, tokens, experts, top):
    kind, n = (tokens + experts) % 3, tokens + experts
    x = _normal(tokens, experts, seed=n)
    bias = _normal(experts, seed=n + 1, spread=0.1)
    _check(gpu, x, kind, top, normalise=n % 2 == 0, pad=n % 3)
    _check(gpu, x, kind, top, bias=bias, sigmoid=True, scale=2.5, normalise=n % 2 == 1)
    _check(gpu, x, F32, top, bias=bias, scale=0.5)
    _check(gpu, x, F32, top, sigmoid=True, normalise=False, pad=5)


@pytest.mark.parametrize("experts,groups,top_groups,top", [(8, 2, 1, 4), (16, 8, 3, 4), (64, 8, 4, 8), (60, 4, 2, 5), (256, 8, 4, 8), (96, 3, 3, 7),
                                                           (128, 64, 10, 12), (1024, 32, 5, 16), (320, 10, 1, 6), (1022, 2, 1, 9)])
@pytest.mark.parametrize("best", [1, 2])
def test_routing_in_groups(gpu, experts, groups, top_groups, top, best):
    for tokens in (1, 40, 200):
        x = _normal(tokens, experts, seed=tokens)
        bias = _normal(experts, seed=5, spread=0.1)
        _check(gpu, x, F32, top, groups=groups, top_groups=top_groups, best=best)
        _check(gpu, x, BF16, top, bias=bias, sigmoid=True, groups=groups, top_groups=top_groups, best=best, scale=2.5)
        _check(gpu, x, F16, top, bias=bias, groups=groups, top_groups=top_groups, best=best, normalise=False)


@pytest.mark.parametrize("experts", [7, 64, 130, 300])
def test_equal_scores_go_to_the_lowest_index(gpu, experts):
    import torch
    x = torch.round(_normal(100, experts, seed=3)) * 0.5
    bias = torch.round(_normal(experts, seed=4)) * 0.25
    top = min(7, experts)
    _check(gpu, x, BF16, top)
    _check(gpu, x, F32, top, bias=bias, sigmoid=True)
    _check(gpu, x, F32, top, bias=bias)
    _check(gpu, torch.zeros(50, experts), F32, top, bias=torch.zeros(experts))
    groups = {7: 7, 64: 8, 130: 10, 300: 20}[experts]
    for best in (1, 2) if experts // groups > 1 else (1,):
        _check(gpu, x, F32, 1, bias=bias, sigmoid=True, groups=groups, top_groups=max(1, groups // 2), best=best)
        _check(gpu, x, F32, 1, groups=groups, top_groups=max(1, groups // 2), best=best)
        _check(gpu, torch.zeros(50, experts), F32, 1, sigmoid=True, groups=groups, top_groups=1, best=best)


@pytest.mark.parametrize("sigmoid", [False, True])
@pytest.mark.parametrize("experts,groups", [(64, 1), (256, 1), (256, 8), (600, 4)])
def test_scores_that_float32_cannot_tell_apart(gpu, sigmoid, experts, groups):
    """A bias that brings all of a token's scores together to within a rounding: the exact ones decide."""
    import torch
    g = torch.Generator().manual_seed(6)
    for tokens, target in ((20, 0.75), (40, 8.0)):
        x = torch.randn((1, experts), generator=g).repeat(tokens, 1)
        x = x + 1e-6 * torch.randn((tokens, experts), generator=g)
        x64 = x[:1].double()
        s = torch.sigmoid(x64) if sigmoid else torch.softmax(x64, 1)
        bias = (target - s[0]).float()
        _check(gpu, x, F32, 8, bias=bias, sigmoid=sigmoid, groups=groups, top_groups=max(1, groups // 2), best=2 if groups > 1 else 1)


def test_masked_experts_and_lost_tokens(gpu):
    import torch
    x = _normal(64, 24, seed=9)
    x[0] = -INF
    x[1, 2:] = -INF
    x[2, ::2] = -INF
    x[3, 5] = float("nan")
    x[4, 23] = INF
    x[5] = -3.4e38
    x[6, :4] = 3.0e38
    x[7, 8:16] = -INF
    x[8, 1:] = -INF
    x[9] = -100.0 + x[9]
    x[10] = 60 + x[10]
    x[11] = -300.0 - 10 * torch.arange(24)
    bias = _normal(24, seed=10, spread=0.2)
    bias[3] = -INF
    for sigmoid in (False, True):
        for normalise in (False, True):
            for b in (None, bias):
                _check(gpu, x, F32, 4, bias=b, sigmoid=sigmoid, normalise=normalise, scale=1.5)
                for best in (1, 2):
                    _check(gpu, x, F32, 4, bias=b, sigmoid=sigmoid, normalise=normalise, groups=3, top_groups=2, best=best)
                    _check(gpu, x[:20], F32, 4, bias=b, sigmoid=sigmoid, normalise=normalise, groups=12, top_groups=2, best=best)
    bias[7] = float("nan")
    ids, w, starts, _, places = _route(gpu, x, F32, 4, bias=bias)
    assert (ids == -1).all() and np.isnan(w).all() and (starts == 0).all() and (places == -1).all()
    # all the same expert, and one that no token takes
    x = torch.zeros(200, 5)
    x[:, 3] = 1
    got = _check(gpu, x, F32, 1)
    assert (got[0] == 3).all() and list(got[2]) == [0, 0, 0, 0, 200, 200]


def test_outputs_that_are_left_out_and_no_tokens(gpu):
    import torch
    x = _normal(100, 40, seed=11)
    whole = _check(gpu, x, F32, 3)
    ids, w = _route(gpu, x, F32, 3, plan=False)
    assert np.array_equal(ids, whole[0]) and np.array_equal(w, whole[1])
    ids, w = torch.empty((100, 3), dtype=torch.int32, device="cuda"), torch.empty((100, 3), device="cuda")
    ws = torch.empty(gpu.mipgemm_route_workspace_size(100, 40, 3), dtype=torch.uint8, device="cuda")
    for with_order in (False, True):
        starts, other = torch.zeros(41, dtype=torch.int32, device="cuda"), torch.zeros(300, dtype=torch.int32, device="cuda")
        gpu.mipgemm_route(100, 40, 3, x.cuda(), 40, F32, None, 0, 1, 1, 1, 1, 1.0, ids, w, starts, other if with_order else None,
                          None if with_order else other, workspace=ws, workspace_bytes=ws.numel())
        assert np.array_equal(starts.cpu().numpy(), whole[2])
        assert np.array_equal(other.cpu().numpy(), whole[3] if with_order else whole[4].reshape(-1))
    starts.fill_(9)
    gpu.mipgemm_route(0, 40, 3, None, 40, F32, None, 0, 1, 1, 1, 1, 1.0, None, None, starts)
    assert (starts == 0).all()


@pytest.mark.parametrize("tokens,experts,top", [(8192, 256, 8), (9001, 100, 5), (70001, 16, 2)])
def test_many_tokens(gpu, tokens, experts, top):
    """Against the definition by sorting: whole matrices at once."""
    import torch
    x = _normal(tokens, experts, seed=12)
    bias = _normal(experts, seed=13, spread=0.1)
    for sigmoid, b in ((False, None), (True, bias)):
        ids, w, starts, order, places = _route(gpu, x, F32, top, bias=b, sigmoid=sigmoid, scale=2.0)
        x64 = x.double()
        s = torch.sigmoid(x64) if sigmoid else torch.softmax(x64, 1)
        want = torch.sort(s + (0 if b is None else b.double()), dim=1, descending=True, stable=True).indices[:, :top]
        assert np.array_equal(ids, want.numpy())
        exact = torch.gather(s, 1, want)
        exact = (2.0 * exact / exact.sum(1, keepdim=True)).numpy()
        assert (np.abs(w - exact) <= exact * 100 * 2.0 ** -24).all()  # (as above: arguments up to 20)
        for got, ref in zip((starts, order, places), _rows(ids, experts)):
            assert np.array_equal(got, ref)


def test_routing_in_a_graph_and_on_another_stream(gpu):
    import torch
    T, E, top = 100, 64, 4
    x = torch.zeros((T, E), device="cuda")
    ws = torch.empty(gpu.mipgemm_route_workspace_size(T, E, top), dtype=torch.uint8, device="cuda")

    def outputs():
        whole = lambda n: torch.zeros(n, dtype=torch.int32, device="cuda")  # noqa: E731
        return [whole(T * top), torch.zeros(T * top, device="cuda"), whole(E + 1), whole(T * top), whole(T * top)]

    def route(o):
        gpu.mipgemm_route(T, E, top, x, E, F32, None, 1, 4, 2, 2, 1, 1.0, *o, workspace=ws, workspace_bytes=ws.numel())
    out = outputs()
    route(out)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        route(out)
    for i in range(4):
        x.copy_(_normal(T, E, seed=20 + i))
        graph.replay()
        torch.cuda.synchronize()
        got = [t.clone() for t in out]
        eager = outputs()
        route(eager)
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, eager)), i
        side, again = torch.cuda.Stream(), outputs()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            route(again)
        side.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, again)), i


@pytest.mark.parametrize("tokens", [5, 70])
@pytest.mark.parametrize("experts", [8, 300, 600])
def test_weights_far_below_the_largest(gpu, tokens, experts):
    """Sigmoid scores that float32 does not hold, whose shares of a sum as small it does."""
    import torch
    x = torch.full((tokens, experts), -200.0)
    x[:, :6] = torch.tensor([-36.0, -39.5, -88.0, -96.5, -103.0, -110.0])
    x = x - 0.05 * torch.arange(tokens)[:, None] % 3
    x[1::5, 0] = 0.3
    x[2::5, 0] = -0.25
    x[3::5, 0] = -41.0
    x[4::5, :2] = -70.0
    for normalise in (True, False):
        _check(gpu, x, F32, 6, sigmoid=True, normalise=normalise)
        _check(gpu, x, F32, 6, sigmoid=True, normalise=normalise, bias=torch.zeros(experts))
        _check(gpu, x, F32, 6, sigmoid=True, normalise=normalise, groups=2, top_groups=2, best=2, scale=2.5)


@pytest.mark.parametrize("tokens", [3, 40])
@pytest.mark.parametrize("kind", [F32, BF16])
def test_offsets_of_tokens_that_pass_31_and_32_bits(gpu, tokens, kind):
    import torch
    experts, top = 70, 5
    x = _normal(tokens, experts, seed=21)
    near = _route(gpu, x, kind, top, sigmoid=True)
    for lead in (2 ** 27 + 1, 2 ** 31 - 1):
        if tokens * lead > 2 ** 34:  # (64 GB of float32)
            continue
        far = torch.as_strided(torch.empty((tokens - 1) * lead + experts, dtype=R.TORCH[kind], device="cuda"), (tokens, experts), (lead, 1))
        far.copy_(x)
        ids, w = torch.zeros((tokens, top), dtype=torch.int32, device="cuda"), torch.zeros((tokens, top), device="cuda")
        gpu.mipgemm_route(tokens, experts, top, far, lead, kind, None, 1, 1, 1, 1, 1, 1.0, ids, w)
        torch.cuda.synchronize()
        assert np.array_equal(ids.cpu().numpy(), near[0]) and np.array_equal(w.cpu().numpy(), near[1]), lead
        del far
