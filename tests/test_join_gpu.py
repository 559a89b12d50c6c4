"""mipgemm_join_rows against its definition in 64 bits."""
import re

import numpy as np
import pytest

import layer_reference as R

pytestmark = pytest.mark.gpu

F32, BF16, F16 = 0, 1, 2
NO, RMS, LAYER = 0, 1, 2
EPS = 1e-6
U = 2.0 ** -24


@pytest.fixture(scope="module")
def gpu():
    import torch
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_2506_11728_amd as M
    M.load_library()
    return M


def _norm(v, wrong, kind, weight, bias, eps):
    """(the norm of v in float64, what the operator's may be off, v being off by `wrong` already)"""
    import torch
    if kind == NO or not v.shape[1]:
        return v, wrong
    cols = v.shape[1]
    mean = v.mean(1, keepdim=True) if kind == LAYER else torch.zeros_like(v[:, :1])
    d = v - mean
    square = (d * d).mean(1, keepdim=True)
    root = torch.sqrt(square + eps)
    r = torch.where(square > 0, 1 / root, torch.zeros_like(root))
    # Differences: three roundings, and the mean's own.  What the mean misses is taken off in a second step, as the mean of the
    # differences from it: that sum of d has, in float32, a depth of at most 16 (a thread's) + 6 (lanes) + 16 (waves) additions, each
    # off by U of a partial sum that is at most the sum of |d|, so the mean that is taken off is off by 38 U mean |d|, whatever d itself is.
    off = wrong + wrong.mean(1, keepdim=True) * (kind == LAYER) + 3 * U * (v.abs() + mean.abs()) * (kind == LAYER)
    off = off + 38 * U * d.abs().mean(1, keepdim=True) * (kind == LAYER)
    # the factor: sums in chains of at most 16 + 6 + 16 additions; a handful of roundings; what the differences are off
    factor = 50 * U + torch.sqrt((off * off).mean(1, keepdim=True)) * r
    y = d * r
    size = y.abs()
    off = off * r + size * factor + 2 * U * size
    if weight is not None:
        y, off, size = y * weight.double(), off * weight.double().abs(), size * weight.double().abs()
    if bias is not None:
        y = y + bias.double()
    return y, off + 2 * U * (size + y.abs())


class Case:
    def __init__(self, rows, cols, parts=1, kind=BF16, post=NO, norm=RMS, gate_rows=0, residual=True, weights=True, biases=False, scale=1.0,
                 pad=0, shuffled=True, seed=0, eps=EPS, spread=1.0, offset=0.0, x_rows=None):
        import torch
        g = torch.Generator().manual_seed(seed)
        rand = lambda *s: torch.randn(s, generator=g)  # noqa: E731
        self.rows, self.cols, self.parts, self.kind, self.post, self.norm, self.scale, self.pad, self.eps = rows, cols, parts, kind, post, norm, scale, pad, eps
        t = R.TORCH[kind]
        self.x_rows = rows * parts if x_rows is None else x_rows
        self.X = (rand(self.x_rows, cols + pad) * spread + offset).to(t)
        self.places = torch.randperm(self.x_rows, generator=g).repeat(1 + rows * parts // max(1, self.x_rows))[:rows * parts].reshape(rows, parts).to(torch.int32) if shuffled else None
        self.w = torch.rand((rows, parts), generator=g) + 0.1 if parts > 1 else None
        self.gate_rows = gate_rows
        self.G = rand(-(-rows // gate_rows), cols + pad).to(t) if gate_rows else None
        self.R_ = (rand(rows, cols + pad) * 2).to(t) if residual else None
        self.pw, self.nw = (rand(cols) * 0.3 + 1, rand(cols) * 0.3 + 1) if weights else (None, None)
        self.pb, self.nb = (rand(cols) * 0.3, rand(cols) * 0.3) if biases else (None, None)

    def call(self, M, h=True, n=True, q=True, in_place=False, stream=None):
        """H, N, Q and scales as they lie, padding and all"""
        import torch
        t, lead = R.TORCH[self.kind], self.cols + self.pad
        make = lambda: torch.full((self.rows, lead), 3.0, dtype=t, device="cuda")  # noqa: E731
        dev = lambda x: None if x is None else x.cuda()  # noqa: E731
        X, G, Rd = dev(self.X), dev(self.G), dev(self.R_)
        H, N = (Rd if in_place else make()) if h else None, make() if n else None
        Q = torch.full((self.rows, lead + 1), 99, dtype=torch.int8, device="cuda") if q else None
        s = torch.full((self.rows + 1,), -5.0, device="cuda") if q else None
        lead = max(1, lead)
        M.mipgemm_join_rows(self.rows, self.cols, self.parts, self.kind, X, lead, self.x_rows, dev(self.places), dev(self.w), self.post,
                            dev(self.pw), dev(self.pb), G, lead, self.gate_rows or 1, self.scale, Rd, lead, H, lead, self.norm, dev(self.nw),
                            dev(self.nb), self.eps, N, lead, Q, lead + 1, s, stream=stream)
        torch.cuda.synchronize()
        if q:
            assert (Q[:, self.cols:] == 99).all() and s[-1] == -5
        if n:
            assert (N[:, self.cols:] == 3).all()
        if h and not in_place:
            assert (H[:, self.cols:] == 3).all()
        if h and in_place:
            assert torch.equal(H[:, self.cols:].cpu(), self.R_[:, self.cols:])
        return H, N, Q, s

    def stream_exact(self):
        import torch
        c = self.cols
        X = torch.cat((self.X[:, :c].double(), torch.zeros((1, c), dtype=torch.float64)))
        at = self.places.long() if self.places is not None else torch.arange(self.rows * self.parts).reshape(self.rows, self.parts)
        at = torch.where((at < 0) | (at >= self.x_rows), self.x_rows, at)
        w = self.w.double() if self.w is not None else torch.ones((self.rows, self.parts), dtype=torch.float64)
        y, size = torch.zeros((self.rows, c), dtype=torch.float64), torch.zeros((self.rows, c), dtype=torch.float64)
        for j in range(self.parts):
            y += X[at[:, j]] * w[:, j:j + 1]
            size += (X[at[:, j]] * w[:, j:j + 1]).abs()
        u, off = _norm(y, self.parts * U * size, self.post, self.pw, self.pb, self.eps)
        by = torch.full_like(u, float(np.float32(self.scale)))
        if self.G is not None:
            by = by * self.G[:, :c].double().repeat_interleave(self.gate_rows, 0)[:self.rows]
        h, off = u * by, (off + 2 * U * u.abs()) * by.abs()
        if self.R_ is not None:
            h = h + self.R_[:, :c].double()
        return h, off + U * h.abs()

    def check(self, M, in_place=False):
        import torch
        H, N, Q, s = self.call(M, in_place=in_place)
        c = self.cols
        want, off = self.stream_exact()
        h = H[:, :c].double().cpu()
        assert ((h - want).abs() <= off + R.rounding(want, self.kind)).all(), float(((h - want).abs() / (off + R.rounding(want, self.kind))).max())
        z, off = _norm(h, torch.zeros_like(h), self.norm, self.nw, self.nb, self.eps)
        n = N[:, :c].double().cpu()
        assert ((n - z).abs() <= off + R.rounding(z, self.kind)).all(), float(((n - z).abs() / (off + R.rounding(z, self.kind))).max())
        if not c:
            assert (s[:-1] == 0).all()
            return
        top, scales = z.abs().amax(1), s[:-1].double().cpu()
        assert ((scales - top / 127).abs() <= (off.amax(1) + 60 * U * top) / 127).all()
        # a code is the nearest: half a step off, and what z is
        back = Q[:, :c].double().cpu() * scales[:, None]
        assert ((back - z).abs() <= 0.5001 * scales[:, None] + 2 * off + 60 * U * z.abs()).all()
        if self.norm == NO or (self.norm == RMS and self.nb is None):
            q, other = torch.empty_like(Q), torch.empty_like(s)
            M.mipgemm_quantize_rows(self.rows, c, H, max(1, c + self.pad), self.kind, (self.nw if self.nw is not None else torch.ones(c)).cuda() if self.norm else None,
                                    self.eps, q, c + self.pad + 1, other)
            torch.cuda.synchronize()
            assert torch.equal(q[:, :c], Q[:, :c])
            assert ((other[:-1].double().cpu() - scales).abs() <= 60 * U * scales).all()


SHAPES = [(1, 1), (3, 7), (5, 64), (2, 511), (9, 513), (4, 1024), (3, 1025), (2, 2048), (3, 2050), (5, 4096), (2, 4100), (3, 8192), (2, 8200), (2, 16384),
          (300, 96)]


@pytest.mark.parametrize("rows,cols", SHAPES)
@pytest.mark.parametrize("kind", [F32, BF16, F16])
@pytest.mark.parametrize("post,norm", [(NO, RMS), (RMS, RMS), (LAYER, LAYER), (NO, LAYER), (RMS, NO), (LAYER, RMS)])
def test_join(gpu, rows, cols, kind, post, norm):
    i = SHAPES.index((rows, cols)) + post + norm
    Case(rows, cols, (1, 2, 8, 3)[i % 4], kind, post, norm, gate_rows=(0, rows, 1, 2)[(i + kind) % 4], residual=i % 5 > 0, biases=i % 2 == 0,
         weights=i % 3 > 0, scale=(1.0, 0.22)[i % 2], pad=(0, 3, 8)[i % 3], shuffled=i % 4 > 0, seed=i).check(gpu)
    Case(rows, cols, (3, 1, 2, 9)[i % 4], kind, post, norm, gate_rows=(1, 0, rows + 5, 2)[(i + kind) % 4], scale=-1.5, pad=(1, 0)[i % 2], seed=i + 1).check(gpu)


@pytest.mark.parametrize("cols", [40, 1000, 3000, 5000, 16000])
def test_in_place_and_results_left_out(gpu, cols):
    import torch
    case = Case(6, cols, 2, BF16, RMS, LAYER, gate_rows=2, pad=4, seed=4)
    case.check(gpu, in_place=True)
    whole = case.call(gpu)
    for h, n, q in ((True, False, False), (False, True, False), (False, False, True), (True, False, True), (False, True, True)):
        got = case.call(gpu, h, n, q)
        for a, b, there in zip(got, whole, (h, n, q, q)):
            assert (a is None) if not there else torch.equal(a, b)


@pytest.mark.parametrize("cols", [70, 1500, 9000])
@pytest.mark.parametrize("parts", [1, 4])
def test_places_that_x_does_not_have(gpu, cols, parts):
    import torch
    case = Case(20, cols, parts, F32, NO, RMS, seed=5)
    case.places[3, 0], case.places[4, -1], case.places[5, 0] = -1, 20 * parts, 2 ** 31 - 1
    case.places[6] = -2 ** 31
    case.check(gpu)
    case = Case(20, cols, parts, BF16, LAYER, RMS, seed=6, residual=False, x_rows=3)
    case.places[7] = -1
    case.check(gpu)
    # no rows at all
    case = Case(4, cols, parts, F32, RMS, RMS, seed=6)
    case.X, case.x_rows = case.X[:0], 0
    case.check(gpu)
    # a weight that is no number shows, whether its row is there or not
    case = Case(4, cols, 2, F32, NO, RMS, seed=7)
    case.places[1, 1], case.w[1, 1], case.w[2, 0] = -1, float("nan"), float("nan")
    H, N, Q, s = case.call(gpu)
    assert torch.isnan(H).all(1).tolist() == [False, True, True, False] and torch.isnan(s[:4]).tolist() == [False, True, True, False]
    assert (Q[1:3, :cols] == 0).all() and torch.isfinite(N[0]).all() and torch.isfinite(N[3]).all()


@pytest.mark.parametrize("kind", [F32, BF16])
@pytest.mark.parametrize("cols", [100, 900, 3000, 12000])
@pytest.mark.parametrize("norm", [RMS, LAYER])
def test_norms_of_rows_of_extreme_size(gpu, kind, cols, norm):
    """Squares that float32 cannot hold, or holds to few bits, and deviations far below the mean."""
    import torch
    by = torch.tensor([1, 1e17, 1e19, 1e30, 1e35, 1e-17, 1e-20, 1e-25, 1e-30, 1e-34], dtype=torch.float64)
    for eps in (0.0, 1e-30, 1e-6):
        case = Case(10, cols, 1, kind, NO, norm, residual=False, shuffled=False, eps=eps, seed=8)
        case.X = (torch.randn((10, cols), generator=torch.Generator().manual_seed(9), dtype=torch.float64) * by[:, None]).to(R.TORCH[kind])
        H, N, Q, s = case.call(gpu, in_place=False)
        assert torch.equal(H.cpu(), case.X)
        z, off = _norm(case.X.double(), torch.zeros((10, cols), dtype=torch.float64), norm, case.nw, None, float(np.float32(eps)))
        n = N.double().cpu()
        assert ((n - z).abs() <= off + R.rounding(z, kind) + 2.0 ** -120).all()
        scales = s[:-1].double().cpu()
        top = z.abs().amax(1)
        assert ((scales - top / 127).abs() <= (off.amax(1) + 60 * U * top) / 127 + 2.0 ** -140).all()
        back = Q[:, :cols].double().cpu() * scales[:, None]
        assert ((back - z).abs() <= 0.5001 * scales[:, None] + 2 * off + 2.0 ** -120).all()
    # the norm behind the sum as well
    case = Case(10, cols, 1, kind, norm, NO, residual=False, shuffled=False, eps=1e-12, seed=8)
    case.X = (torch.randn((10, cols), generator=torch.Generator().manual_seed(9), dtype=torch.float64) * by[:, None]).to(R.TORCH[kind])
    case.check(gpu)


@pytest.mark.parametrize("cols", [64, 1000, 4000, 10000])
@pytest.mark.parametrize("eps", [0.0, 1e-6])
def test_rows_without_a_deviation(gpu, cols, eps):
    import torch
    for norm in (RMS, LAYER):
        case = Case(6, cols, 1, F32, NO, norm, residual=False, shuffled=False, eps=eps, seed=10)
        case.X[0], case.X[1], case.X[2], case.X[3] = 0.0, 7.3, -1e30, 1e-40
        H, N, Q, s = case.call(gpu)
        flat = 4 if norm == LAYER else 1
        assert (N[:flat] == 0).all() and (Q[:flat, :cols] == 0).all() and (s[:flat] == 0).all()
        assert torch.isfinite(N[4:]).all() and (s[4:6] > 0).all()
    # far from zero: what differs is kept
    case = Case(6, cols, 1, F32, NO, LAYER, residual=False, shuffled=False, eps=0.0, seed=11, offset=3e4)
    H, N, Q, s = case.call(gpu)
    d = case.X.double() - case.X.double().mean(1, keepdim=True)
    z = d / torch.sqrt((d * d).mean(1, keepdim=True)) * case.nw.double()
    assert ((N.double().cpu() - z).abs() <= 60 * U * (z.abs() + 1)).all()


@pytest.mark.parametrize("cols", [33, 800, 2500, 7000])
def test_rows_that_are_no_numbers(gpu, cols):
    import torch
    for post, norm in ((NO, RMS), (LAYER, LAYER), (RMS, NO)):
        case = Case(7, cols, 1, F32, post, norm, shuffled=False, residual=False, seed=12)
        clean = case.call(gpu)
        case.X[1, cols // 2], case.X[3, 0], case.X[5, cols - 1] = float("nan"), float("inf"), -float("inf")
        H, N, Q, s = case.call(gpu)
        for r in (1, 3, 5):
            assert not torch.isfinite(N[r]).all() and torch.isnan(s[r]) and (Q[r, :cols] == 0).all()
        for r in (0, 2, 4, 6):  # the others as they were
            assert torch.equal(N[r], clean[1][r]) and torch.equal(Q[r], clean[2][r]) and s[r] == clean[3][r]


def test_no_columns_and_more_than_one_launch(gpu):
    import torch
    for kind in (F32, BF16):
        Case(5, 0, 2, kind, RMS, LAYER).check(gpu)
    rows = 2 ** 21 + 5  # 2^21 rows go into a launch
    X = torch.randn((rows, 2), generator=torch.Generator().manual_seed(13)).cuda()
    H = torch.zeros_like(X)
    gpu.mipgemm_join_rows(rows, 2, 1, F32, X, 2, rows, None, None, 0, None, None, None, 2, 1, 3.0, None, 2, H, 2, 0, None, None, 0.0, None, 2)
    assert torch.equal(H, 3 * X)


def test_join_in_a_graph_and_on_another_stream(gpu):
    import torch
    rows, cols, parts = 70, 640, 4
    g = torch.Generator().manual_seed(14)
    X = torch.zeros((rows * parts, cols), dtype=torch.bfloat16, device="cuda")
    places = torch.zeros((rows, parts), dtype=torch.int32, device="cuda")
    w = torch.ones((rows, parts), device="cuda")
    Rd = torch.randn((rows, cols), generator=g).to(torch.bfloat16).cuda()
    weight = torch.rand(cols, generator=g).cuda()

    def outputs():
        return [torch.zeros((rows, cols), dtype=torch.bfloat16, device="cuda") for _ in range(2)] + \
            [torch.zeros((rows, cols), dtype=torch.int8, device="cuda"), torch.zeros(rows, device="cuda")]

    def call(o):
        gpu.mipgemm_join_rows(rows, cols, parts, BF16, X, cols, rows * parts, places, w, RMS, weight, None, None, cols, 1, 1.0, Rd, cols, o[0], cols,
                              LAYER, weight, weight, EPS, o[1], cols, o[2], cols, o[3])
    out = outputs()
    call(out)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call(out)
    for i in range(4):
        X.copy_(torch.randn((rows * parts, cols), generator=g))
        places.copy_(torch.randperm(rows * parts, generator=g).reshape(rows, parts))
        w.copy_(torch.rand((rows, parts), generator=g))
        graph.replay()
        torch.cuda.synchronize()
        got, eager = [t.clone() for t in out], outputs()
        call(eager)
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, eager)), i
        side, again = torch.cuda.Stream(), outputs()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            call(again)
        side.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, again)), i


# ---- the forms for more rows than two to a compute unit, whose threads keep more of a row ----

MANY = [(513, 513, "1, 4, 2, false"), (520, 520, "1, 4, 2, true"), (600, 1024, "1, 4, 2, true"), (530, 1025, "4, 1, 1, false"),
        (530, 2050, "4, 1, 2, false"), (520, 2056, "4, 1, 2, true"), (600, 4096, "4, 1, 2, true"), (515, 4099, "8, 1, 2, false"),
        (515, 4100, "8, 1, 2, false"), (513, 8184, "8, 1, 2, true"), (514, 8192, "8, 1, 2, true"), (513, 8193, "16, 1, 2, false")]


def _served(kernels_of, gpu, case):
    """The kernel that serves a case of float32, with its template's arguments."""
    names = [re.search(r"join_kernel<([^>]*)>", n) for n in kernels_of(lambda: case.call(gpu))]
    names = [n.group(1) for n in names if n]
    assert len(names) == 1, names
    return names[0]


@pytest.mark.parametrize("rows,cols,form", MANY)
@pytest.mark.parametrize("kind", [F32, BF16, F16])
def test_many_rows(gpu, kernels_of, rows, cols, form, kind):
    i = MANY.index((rows, cols, form)) + kind
    first = Case(rows, cols, (1, 2, 3)[i % 3], kind, RMS, RMS, gate_rows=(200, 0, rows, 1)[i % 4], scale=0.22, pad=(0, 3, 8)[i % 3], seed=i)
    if kind == F32:
        assert _served(kernels_of, gpu, first) == "float, " + form
    first.check(gpu, in_place=i % 2 == 0)
    Case(rows, cols, (2, 1)[i % 2], kind, LAYER, LAYER, gate_rows=(0, 7)[i % 2], biases=True, pad=(5, 0)[i % 2], residual=i % 3 > 0, seed=i + 1).check(gpu)
    Case(rows, cols, 1, kind, NO, (RMS, LAYER, NO)[i % 3], weights=i % 2 == 0, shuffled=i % 4 > 0, seed=i + 2).check(gpu, in_place=True)


@pytest.mark.parametrize("cols", [520, 1001, 2056, 4096, 4100, 8192])
def test_many_rows_that_are_no_numbers_and_of_extreme_size(gpu, cols):
    import torch
    rows = 520
    by = torch.tensor([1, 1e17, 1e19, 1e30, 1e35, 1e-17, 1e-20, 1e-25, 1e-30, 1e-34], dtype=torch.float64).repeat(52)
    for kind, post, norm in ((F32, NO, RMS), (BF16, NO, LAYER), (F32, LAYER, NO)):
        case = Case(rows, cols, 1, kind, post, norm, residual=False, shuffled=False, eps=1e-12, seed=15)
        case.X = (torch.randn((rows, cols), generator=torch.Generator().manual_seed(16), dtype=torch.float64) * by[:, None]).to(R.TORCH[kind])
        case.check(gpu)
        clean = case.call(gpu)
        case.X[1, cols // 2], case.X[300, 0], case.X[519, cols - 1] = float("nan"), float("inf"), -float("inf")
        H, N, Q, s = case.call(gpu)
        others = torch.ones(rows, dtype=torch.bool)
        others[[1, 300, 519]] = False
        for r in (1, 300, 519):
            assert not torch.isfinite(N[r]).all() and torch.isnan(s[r]) and (Q[r, :cols] == 0).all()
        for a, b in zip((H, N, Q, s[:-1]), clean):
            assert torch.equal(a.cpu()[others], b.cpu()[:rows][others])


@pytest.mark.parametrize("parts", [63, 64, 65, 130, 1024])
@pytest.mark.parametrize("rows,cols", [(3, 100), (2, 1500), (1, 4096)])
def test_many_parts(gpu, parts, rows, cols):
    """More parts than a wave has lanes, with places and weights, without either, and without both."""
    import torch
    for shuffled in (True, False):
        for weights in (True, False):
            case = Case(rows, cols, parts, BF16 if weights else F32, NO, RMS, shuffled=shuffled, pad=3, seed=parts)
            if not weights:
                case.w = None
            case.check(gpu)
            if shuffled:
                case.places[0, 0], case.places[-1, parts - 1], case.places[0, min(64, parts - 1)] = -1, -3, rows * parts
                case.check(gpu)
                if weights:
                    case.w[-1, parts - 1] = float("nan")
                    assert torch.isnan(case.call(gpu)[0][-1, :cols]).all()


@pytest.mark.parametrize("kind", [F32, BF16])
@pytest.mark.parametrize("cols", [96, 1500, 4096])
@pytest.mark.parametrize("rows", [8, 520])
def test_scales_of_rows_next_to_the_smallest_numbers(gpu, kind, cols, rows):
    """A 127th of a row's largest has few bits left below 2^-126; what the norm makes of it has all of them."""
    import torch
    by = torch.tensor([1e-36, 1e-37, 1e-38, 1e-39, 1e-40, 1e-41, 1e-42, 1e-43], dtype=torch.float64).repeat(rows // 8)
    case = Case(rows, cols, 1, kind, NO, RMS, residual=False, shuffled=False, weights=False, eps=0.0, seed=17)
    case.X = (torch.randn((rows, cols), generator=torch.Generator().manual_seed(18), dtype=torch.float64) * by[:, None]).to(R.TORCH[kind])
    H, N, Q, s = case.call(gpu)
    assert torch.equal(H.cpu(), case.X)
    x = case.X.double()
    z = (x / torch.sqrt((x * x).mean(1, keepdim=True))).nan_to_num(0.0)  # (rows that bfloat16 has only zeros for stay zeros)
    assert ((N.double().cpu() - z).abs() <= 60 * U * z.abs() + R.rounding(z, kind)).all()
    # the factor and the product are in float64: one rounding to float32 is left (U), and there is room for two more
    assert ((s[:-1].double().cpu() - z.abs().amax(1) / 127).abs() <= 3 * U * z.abs().amax(1) / 127).all()
    q, other = torch.empty_like(Q), torch.empty_like(s)
    gpu.mipgemm_quantize_rows(rows, cols, H, cols, kind, torch.ones(cols, device="cuda"), 0.0, q, cols + 1, other)
    torch.cuda.synchronize()
    assert torch.equal(q[:, :cols], Q[:, :cols])
    assert ((other[:-1].double() - s[:-1].double()).abs() <= 60 * U * s[:-1]).all()


@pytest.mark.parametrize("cols", [100, 4096])
def test_offsets_of_rows_that_pass_31_and_32_bits(gpu, cols):
    """Three rows 2^30 and 2^31 - 1 elements apart, in every operand at once, against the same rows side by side."""
    import torch
    rows = 3
    case = Case(rows, cols, 2, BF16, RMS, RMS, gate_rows=1, seed=19)
    near = case.call(gpu)
    weights = [x.cuda() for x in (case.pw, case.nw, case.w)]
    for lead in (2 ** 30, 2 ** 31 - 1):
        far = lambda x, n, kind=torch.bfloat16: torch.as_strided(torch.empty((n - 1) * lead + cols, dtype=kind, device="cuda"), (n, cols), (lead, 1)).copy_(x)  # noqa: E731
        X, G, Rd = far(case.X, rows * 2), far(case.G, rows), far(case.R_, rows)
        H, N, Q = far(torch.zeros(rows, cols), rows), far(torch.zeros(rows, cols), rows), far(torch.zeros(rows, cols), rows, torch.int8)
        s = torch.zeros(rows, device="cuda")
        gpu.mipgemm_join_rows(rows, cols, 2, BF16, X, lead, rows * 2, case.places.cuda(), weights[2], RMS, weights[0], None, G, lead, 1, 1.0, Rd, lead, H, lead,
                              RMS, weights[1], None, EPS, N, lead, Q, lead, s)
        torch.cuda.synchronize()
        for got, want in zip((H, N, Q, s), near):
            assert torch.equal(got, want[:rows, :cols] if want.dim() > 1 else want[:rows]), lead
        del X, G, Rd, H, N, Q
