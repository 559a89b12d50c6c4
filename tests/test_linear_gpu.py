"""mipgemm_quantize_rows and mipgemm_s8s8_linear against their definitions in 64 bits."""
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


def _rows(rows, cols, kind, seed):
    import torch
    g = torch.Generator().manual_seed(seed)
    x = torch.randn((rows, cols), generator=g) * torch.exp(3 * torch.randn((rows, 1), generator=g))
    return x.to(R.TORCH[kind])


def _quantize(M, x, pad, weight, eps):
    import torch
    rows, cols = x.shape
    buf = torch.full((rows, cols + pad), 7.0, dtype=x.dtype)
    buf[:, :cols] = x
    q = torch.full((rows, cols + pad + 1), 99, dtype=torch.int8, device="cuda")
    s = torch.full((rows,), -5.0, device="cuda")
    kind = {v: k for k, v in R.TORCH.items()}[x.dtype]
    d = buf.cuda()
    w = None if weight is None else weight.cuda()
    M.mipgemm_quantize_rows(rows, cols, d, cols + pad, kind, w, eps, q, cols + pad + 1, s)
    torch.cuda.synchronize()
    assert (q[:, cols:] == 99).all()
    return q[:, :cols].cpu().numpy(), s.cpu().numpy()


def _codes(z):
    """rint of the correctly rounded quotient of float32(127 z) and the row's largest."""
    z = z.astype(np.float32)
    a = np.abs(z).max(1, keepdims=True) if z.shape[1] else np.zeros((z.shape[0], 1), np.float32)
    with np.errstate(all="ignore"):
        q = np.rint((z * np.float32(127)) / np.where(a > 0, a, np.float32(1)))
    return np.where(np.isfinite(a), q, 0).astype(np.int8), a[:, 0]


@pytest.mark.parametrize("kind", [F32, BF16, F16])
@pytest.mark.parametrize("shape", [(1, 1), (3, 7), (5, 64), (2, 1023), (9, 1025), (4, 4096), (2, 4099), (3, 11008),
                                   (2, 16385), (1, 40001), (1000, 33)])
@pytest.mark.parametrize("norm", [False, True])
def test_rows_in_8_bits(gpu, kind, shape, norm):
    import torch
    x = _rows(*shape, kind, 1)
    w = torch.randn(shape[1], generator=torch.Generator().manual_seed(2)) + 1 if norm else None
    q, s = _quantize(gpu, x, 3, w, 1e-6)
    z = x.float().numpy() * (w.numpy() if norm else np.float32(1))
    want, a = _codes(z)
    assert np.array_equal(q, want)
    exact = a.astype(np.float64) / 127
    if norm:
        exact = exact / np.sqrt((x.double().numpy() ** 2).mean(1) + 1e-6)
    # the squares: a chain of at most cols / 64 + 16 float32 additions; a handful of roundings after
    bound = ((shape[1] / 64 + 16) * norm + 8) * 2.0 ** -24
    fine = np.isfinite(a)  # (a few float16 rows hold an infinity)
    assert (np.abs(s - exact)[fine] <= (bound * exact)[fine]).all()
    assert np.isnan(s[~fine]).all() and (q[~fine] == 0).all()


@pytest.mark.parametrize("cols", [5, 100, 3000, 20000])
@pytest.mark.parametrize("norm", [False, True])
def test_rows_that_are_no_ordinary_numbers(gpu, cols, norm):
    import torch
    x = torch.randn((8, cols), generator=torch.Generator().manual_seed(3))
    x[0] = 0
    x[1, cols // 2] = float("inf")
    x[2, 0] = float("nan")
    x[3, -1] = -float("inf")
    x[4] *= 1e-42
    x[5] *= 1e37
    x[6] = -2.5
    w = torch.ones(cols) if norm else None
    q, s = _quantize(gpu, x, 0, w, 1e-6)
    assert (q[0] == 0).all() and s[0] == 0
    for r in (1, 2, 3):
        assert (q[r] == 0).all() and np.isnan(s[r])
    for r in (4, 5, 6, 7):
        z = x[r].double().numpy()
        t = 127 * z / np.abs(z).max()
        # (float32 subnormals hold the tiny row to few digits: the codes are of what is held)
        assert np.abs(q[r] - t).max() <= 0.5 + 1e-4, r
        if not norm:
            assert abs(s[r] - np.abs(z).max() / 127) <= 2.0 ** -23 * s[r] + 2.0 ** -149
    assert (q[6] == -127).all()


@pytest.mark.parametrize("kind", [F32, BF16])
@pytest.mark.parametrize("shape", [(14, 100), (14, 3000), (14, 5000), (600, 5000), (14, 20000)])
@pytest.mark.parametrize("eps", [0.0, 1e-30, 1e-6])
def test_norms_of_rows_of_extreme_size(gpu, kind, shape, eps):
    """Squares that float32 cannot hold, or holds to few bits, do not reach the scales."""
    import torch
    rows, cols = shape
    by = torch.tensor([1, 1e17, 1e18, 1e19, 1e20, 1e30, 2e37, 1e-17, 1e-20, 1e-22, 1e-25, 1e-30, 1e-35, 0], dtype=torch.float64)
    x = torch.randn((rows, cols), generator=torch.Generator().manual_seed(41), dtype=torch.float64)
    x = (x * by[torch.arange(rows) % 14, None]).to(R.TORCH[kind])
    w = torch.rand(cols, generator=torch.Generator().manual_seed(42)) + 0.5
    q, s = _quantize(gpu, x, 1, w, eps)
    z = x.float().numpy() * w.numpy()
    a = np.abs(z).max(1)
    # (a power of two for each row: 127 times the largest would leave float32)
    want, _ = _codes(z * np.exp2(-np.floor(np.log2(np.where(a > 0, a, 1), dtype=np.float64)))[:, None])
    assert np.array_equal(q, want)
    mean = (x.double().numpy() ** 2).mean(1) + float(np.float32(eps))
    exact = np.where(a > 0, a.astype(np.float64) / 127 / np.sqrt(np.where(a > 0, mean, 1)), 0)
    # the squares: a chain of at most cols / 64 + 16 float32 additions; a handful of roundings after, of numbers that may be subnormal
    assert (np.abs(s - exact) <= (cols / 64 + 24) * 2.0 ** -24 * exact + 2.0 ** -149).all()
    assert (s[13::14] == 0).all()


@pytest.mark.parametrize("kind", [F32, BF16, F16])
@pytest.mark.parametrize("shape", [(513, 4097), (600, 11008), (515, 12301), (520, 16384)])
@pytest.mark.parametrize("norm", [False, True])
def test_many_rows_of_more_than_4096_columns(gpu, kind, shape, norm):
    import torch
    rows, cols = shape
    x = (torch.randn(shape, generator=torch.Generator().manual_seed(43)) * 3).to(R.TORCH[kind])
    x[7], x[9, cols - 1], x[11, 0] = 0, float("inf"), float("nan")
    w = torch.randn(cols, generator=torch.Generator().manual_seed(44)) + 1 if norm else None
    q, s = _quantize(gpu, x, 5, w, 1e-6)
    z = x.float().numpy() * (w.numpy() if norm else np.float32(1))
    lost = np.isin(np.arange(rows), (9, 11))
    assert np.isnan(s[lost]).all() and (q[lost] == 0).all() and s[7] == 0 and (q[7] == 0).all()
    want, a = _codes(z[~lost])
    assert np.array_equal(q[~lost], want)
    exact = a.astype(np.float64) / 127
    if norm:
        exact = exact / np.sqrt((x.double().numpy()[~lost] ** 2).mean(1) + 1e-6)
    # the squares: a chain of at most cols / 256 + 16 float32 additions; a handful of roundings after
    bound = ((cols / 256 + 16) * norm + 8) * 2.0 ** -24
    assert (np.abs(s[~lost] - exact) <= bound * exact).all()


def test_rows_of_more_than_one_launch(gpu):
    """2^21 rows go into a launch, whose grid then holds them with the most threads a row can have."""
    import torch
    rows = 2 ** 21 + 5
    x = torch.randn((rows, 3), generator=torch.Generator().manual_seed(5))
    q, s = _quantize(gpu, x, 1, None, 0.0)
    want, a = _codes(x.numpy())
    assert np.array_equal(q, want) and np.array_equal(s, a / np.float32(127))


def test_no_columns_and_no_rows(gpu):
    import torch
    s = torch.full((3,), 4.0, device="cuda")
    w = torch.ones(1, device="cuda")
    gpu.mipgemm_quantize_rows(3, 0, None, 1, F32, w, 1e-6, None, 1, s)
    assert (s == 0).all()
    gpu.mipgemm_quantize_rows(0, 5, None, 5, F32, None, 0.0, None, 5, None)


def _linear_case(m, n, k, order, kind, pad, seed, scales=True, bias=True, residual=True):
    import torch
    g = torch.Generator().manual_seed(seed)
    A = torch.randint(-128, 128, (m, k + pad), generator=g, dtype=torch.int8)
    B = torch.randint(-128, 128, ((n, k + pad) if order else (k, n + pad)), generator=g, dtype=torch.int8)
    a = torch.rand(m, generator=g) * 0.02 + 0.001 if scales else None
    b = torch.rand(n, generator=g) * 0.02 / max(1, k) ** 0.5 if scales else None
    c = torch.randn(n, generator=g) if bias else None
    r = torch.randn((m, n + pad), generator=g).to(R.TORCH[kind]) if residual else None
    return A, B, a, b, c, r


def _linear_exact(m, n, k, order, A, B, a, b, c, r, which):
    """(the result, a bound on the size of what is added up on the way), float64"""
    import torch
    A64, B64 = A[:, :k].double(), (B[:, :k].double().T if order else B[:k, :n].double())
    S = A64 @ B64  # exact: below 2^53
    S = torch.remainder(S + 2.0 ** 31, 2.0 ** 32) - 2.0 ** 31
    y = S * (a.double()[:, None] if a is not None else 1) * (b.double() if b is not None else 1)
    size = y.abs()
    if c is not None:
        y = y + c.double()
        size = size + c.double().abs()
    y = R.act(y, which)
    if r is not None:
        y = y + r[:, :n].double()
        size = size + r[:, :n].double().abs()
    return y, size


def _check_linear(M, m, n, k, order, kind, which, pad=0, seed=0, workspace=True, in_place=False, **parts):
    import torch
    A, B, a, b, c, r = _linear_case(m, n, k, order, kind, pad, seed, **parts)
    want, size = _linear_exact(m, n, k, order, A, B, a, b, c, r, which)
    dev = [None if t is None else t.cuda() for t in (A, B, a, b, c, r)]
    dA, dB, da, db, dc, dr = dev
    C = dr if in_place else torch.full((m, n + pad), 3.0, dtype=R.TORCH[kind], device="cuda")
    behind = C[:, n:].clone()
    need = M.mipgemm_workspace_size_f32(m, n, k, 0, order, 0) + (m + n + 512) * (k + 128) if workspace else 0
    ws = torch.full((need + 64,), 0x77, dtype=torch.uint8, device="cuda") if workspace else None
    M.mipgemm_s8s8_linear(m, n, k, dA, max(1, k + pad), da, dB, max(1, (k if order else n) + pad), order, db, dc, which, dr, n + pad,
                          C, n + pad, kind, workspace=ws, workspace_bytes=need)
    torch.cuda.synchronize()
    got = C[:, :n].double().cpu()
    # five float32 roundings and an activation within 2e-7 of its argument's size, of slope below 1.13
    bound = 2.0 ** -21 * size + 1e-6 * size * (which >= 2) + R.rounding(want, kind)
    off = (got - want).abs()
    if kind == F16:  # what is past the type's range (within its bound on either side) is an infinity of its sign
        past = (got == torch.copysign(torch.full_like(got, float("inf")), want)) & (want.abs() + bound >= 65520)
        off = torch.where(past, torch.zeros_like(off), off)
    assert (off <= bound).all(), (m, n, k, order, kind, which, float((off / bound).max()))
    assert torch.equal(C[:, n:], behind)
    if ws is not None:
        assert (ws[need:] == 0x77).all()


SHAPES = [(1, 1, 1), (1, 4096, 512), (3, 17, 5), (16, 48, 64), (33, 100, 200), (64, 256, 192), (100, 130, 257), (130, 257, 384),
          (128, 128, 128), (256, 256, 256), (257, 300, 1024), (300, 520, 128), (512, 512, 2048), (1000, 96, 640)]


@pytest.mark.parametrize("order", [0, 1])
@pytest.mark.parametrize("shape", SHAPES, ids=str)
@pytest.mark.parametrize("kind", [F32, BF16, F16])
def test_linear(gpu, shape, order, kind):
    which = (SHAPES.index(shape) + kind + order) % 5
    _check_linear(gpu, *shape, order, kind, which, pad=0)
    _check_linear(gpu, *shape, order, kind, (which + 1) % 5, pad=16, workspace=False)
    _check_linear(gpu, *shape, order, kind, (which + 2) % 5, pad=5)
    _check_linear(gpu, *shape, order, kind, (which + 3) % 5, pad=3, workspace=False)


VARIANTS = ["simple", "dma256k128", "dma128k128", "dma128k128split", "slab16", "slab32", "slab64", "wave32", "wave32x64",
            "tile256", "tile128", "tile64", "tile64x256", "tile256x64", "tile64x128", "tile128x64",
            "dma256", "dma128", "dma64", "dma64x256", "dma256x64", "dma64x128", "dma128x64"]


@pytest.mark.parametrize("variant", VARIANTS)
@pytest.mark.parametrize("order", [0, 1])
def test_linear_of_every_kernel(gpu, variant, order):
    for i, (m, n, k) in enumerate([(256, 512, 256), (48, 256, 1024), (300, 272, 384), (512, 512, 1024)]):
        for which in (i, i + 1):
            with gpu.tuning(MIPGEMM_VARIANT=variant):
                _check_linear(gpu, m, n, k, order, (i + which) % 3, which % 5, seed=i)


@pytest.mark.parametrize("variant", ["dma128", "dma64", "dma64x256", "dma128x64"])
@pytest.mark.parametrize("splits", [2, 5])
def test_linear_with_ranges_of_k(gpu, variant, splits):
    with gpu.tuning(MIPGEMM_VARIANT=variant, MIPGEMM_SPLITK=str(splits)):
        for which in range(5):
            _check_linear(gpu, 100, 200, 1280, 1, which % 3, which)
            _check_linear(gpu, 130, 208, 640, 0, which % 3, which, workspace=False)


@pytest.mark.parametrize("shape", [(256, 768, 1024), (700, 384, 512), (768, 768, 1280)])
def test_linear_on_tiles_with_a_side_of_192(gpu, shape):
    for which in range(5):
        _check_linear(gpu, *shape, 1, which % 3, which)
        _check_linear(gpu, *shape, 0, which % 3, which)


@pytest.mark.parametrize("shape", [(5, 48, 64), (129, 200, 256), (512, 640, 1024), (61, 77, 91)])
@pytest.mark.parametrize("kind", [F32, BF16, F16])
def test_linear_with_parts_left_out_and_in_place(gpu, shape, kind):
    _check_linear(gpu, *shape, 1, kind, 0, scales=False, bias=False, residual=False)
    _check_linear(gpu, *shape, 1, kind, 4, bias=False)
    _check_linear(gpu, *shape, 1, kind, 1, residual=False)
    _check_linear(gpu, *shape, 1, kind, 2, pad=4, in_place=True)


def test_linear_of_an_empty_sum_and_of_nothing(gpu):
    for kind in (F32, BF16, F16):
        _check_linear(gpu, 7, 9, 0, 1, kind, 4, workspace=False)
        _check_linear(gpu, 300, 300, 0, 0, kind, 2, workspace=False)
    import torch
    X = torch.zeros(25, dtype=torch.int8, device="cuda")
    gpu.mipgemm_s8s8_linear(0, 5, 5, None, 5, None, X, 5, 1, None, None, 0, None, 0, None, 5, F32)
    gpu.mipgemm_s8s8_linear(5, 0, 5, X, 5, None, None, 5, 1, None, None, 0, None, 0, None, 5, F32)


def test_linear_sums_wrap_as_the_products_do(gpu):
    import torch
    m, n, k = 16, 64, 140032  # 140032 * 2^14 is past 2^31
    A = torch.full((m, k), -128, dtype=torch.int8, device="cuda")
    C = torch.zeros((m, n), device="cuda")
    B = torch.full((n, k), -128, dtype=torch.int8, device="cuda")
    gpu.mipgemm_s8s8_linear(m, n, k, A, k, None, B, k, 1, None, None, 0, None, n, C, n, F32)
    assert (C == float(np.float32(k * 16384 - 2 ** 32))).all()


def test_linear_is_the_same_bits_with_and_without_workspace(gpu):
    import torch
    m, n, k = 200, 300, 1024
    A, B, a, b, c, r = (t.cuda() for t in _linear_case(m, n, k, 1, BF16, 0, 4))
    outs = []
    for size in (0, 1 << 24):
        ws = torch.empty(size, dtype=torch.uint8, device="cuda") if size else None
        C = torch.zeros((m, n), dtype=torch.bfloat16, device="cuda")
        gpu.mipgemm_s8s8_linear(m, n, k, A, k, a, B, k, 1, b, c, 4, r, n, C, n, BF16, workspace=ws, workspace_bytes=size)
        outs.append(C)
    assert torch.equal(*outs)


def test_a_layer_in_a_graph_and_on_another_stream(gpu):
    """quantise, multiply: captured once, replayed over changing activations, against eager calls."""
    import torch
    m, n, k = 48, 512, 2048
    g = torch.Generator().manual_seed(8)
    W = torch.randint(-127, 128, (n, k), generator=g, dtype=torch.int8).cuda()
    b = (torch.rand(n, generator=g) * 0.001).cuda()
    X = torch.zeros((m, k), dtype=torch.bfloat16, device="cuda")
    Q, s = torch.empty((m, k), dtype=torch.int8, device="cuda"), torch.empty(m, device="cuda")
    ws = torch.empty(1 << 24, dtype=torch.uint8, device="cuda")

    def layer(C):
        gpu.mipgemm_quantize_rows(m, k, X, k, BF16, None, 0.0, Q, k, s)
        gpu.mipgemm_s8s8_linear(m, n, k, Q, k, s, W, k, 1, b, None, 4, None, n, C, n, BF16, workspace=ws, workspace_bytes=1 << 24)
    out = torch.zeros((m, n), dtype=torch.bfloat16, device="cuda")
    layer(out)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        layer(out)
    for i in range(4):
        X.copy_(torch.randn((m, k), generator=g).to(torch.bfloat16))
        graph.replay()
        torch.cuda.synchronize()
        got = out.clone()
        eager = torch.zeros_like(out)
        layer(eager)
        torch.cuda.synchronize()
        assert torch.equal(got, eager), i
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            layer(eager.zero_())
        side.synchronize()
        assert torch.equal(got, eager), i
