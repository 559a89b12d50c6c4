"""mipgemm_s8s8_experts against its definition in 64 bits."""
import re

import numpy as np
import pytest

import layer_reference as R

pytestmark = pytest.mark.gpu

F32, BF16, F16 = 0, 1, 2
NONE, RELU, GELU, GELU_TANH, SILU = 0, 1, 2, 3, 4


@pytest.fixture(scope="module")
def gpu():
    import torch
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_2506_11728_amd as M
    M.load_library()
    return M


def _counts(experts, rows, seed, skew):
    """Rows of each expert: some have none, one may have most."""
    g = np.random.RandomState(seed)
    p = g.dirichlet(np.full(experts, skew))
    return g.multinomial(rows, p)


class Case:
    def __init__(self, counts, n, k, top=2, gated=False, gather=True, pad=0, kind=BF16, act=NONE, scales=True, bias=True, seed=0, behind=3,
                 shift=0):
        """behind: rows of the bound that no expert has; shift: bytes that the operands start away from 16-byte alignment."""
        import torch
        g = torch.Generator().manual_seed(seed)
        self.counts, self.n, self.k, self.top, self.gated, self.kind, self.act, self.behind = counts, n, k, top, gated, kind, act, behind
        self.experts, self.used = len(counts), int(sum(counts))
        self.rows, self.outputs = self.used + behind, n * (1 + gated)
        self.a_rows = max(1, -(-self.rows // top)) if gather else max(1, self.rows)
        self.A = torch.randint(-128, 128, (self.a_rows, k + pad), generator=g, dtype=torch.int8)
        self.B = torch.randint(-128, 128, (self.experts, self.outputs, k + pad), generator=g, dtype=torch.int8)
        self.order = torch.randperm(self.a_rows * top, generator=g)[:self.rows].to(torch.int32) if gather else None
        self.starts = torch.tensor([0] + list(counts)).cumsum(0).to(torch.int32)
        self.a = torch.rand(self.a_rows, generator=g) * 0.02 + 0.001 if scales else None
        self.b = torch.rand((self.experts, self.outputs), generator=g) * 0.03 / max(1, k) ** 0.5 if scales else None
        self.bias = torch.randn((self.experts, self.outputs), generator=g) if bias else None
        self.pad, self.shift = pad, shift

    def on_gpu(self, x):
        """x as it lies in a larger buffer, `shift` elements from its start."""
        import torch
        if x is None:
            return None
        buf = torch.empty(x.numel() + 64, dtype=x.dtype, device="cuda")
        part = buf[self.shift:self.shift + x.numel()].view(x.shape)
        part.copy_(x)
        return part

    def call(self, M, C=None, stream=None, bound=0):
        import torch
        lead = self.k + self.pad
        if C is None:
            C = torch.full((self.rows + bound, self.n + self.pad), 3.0, dtype=R.TORCH[self.kind], device="cuda")
        dev = [self.on_gpu(x) for x in (self.A, self.B)] + [None if x is None else x.cuda() for x in (self.a, self.starts, self.order, self.b, self.bias)]
        A, B, a, starts, order, b, bias = dev
        M.mipgemm_s8s8_experts(self.rows, self.experts, self.n, self.k, A, max(1, lead), self.a_rows, a, starts, order, self.top, B,
                               max(1, lead), self.outputs * max(1, lead), b, bias, self.act, int(self.gated), C, self.n + self.pad, self.kind,
                               stream=stream)
        torch.cuda.synchronize()
        return C

    def exact(self):
        """(the result of the used rows, a bound on what it may be off)"""
        import torch
        out, bound = torch.zeros((self.used, self.n), dtype=torch.float64), torch.zeros((self.used, self.n), dtype=torch.float64)
        A, B = self.A[:, :self.k].double(), self.B[:, :, :self.k]
        for e in range(self.experts):
            at = torch.arange(int(self.starts[e]), int(self.starts[e + 1]))
            if not len(at):
                continue
            i = torch.div(self.order[at].long(), self.top, rounding_mode="floor") if self.order is not None else at
            there = (i >= 0) & (i < self.a_rows) if self.order is None else (self.order[at] >= 0) & (i < self.a_rows)
            i = torch.where(there, i, 0)
            S = A[i] @ B[e].double().T * there[:, None]
            S = torch.remainder(S + 2.0 ** 31, 2.0 ** 32) - 2.0 ** 31
            y = S * (self.a.double()[i][:, None] if self.a is not None else 1) * (self.b[e].double() if self.b is not None else 1)
            size = y.abs()
            if self.bias is not None:
                y, size = y + self.bias[e].double(), size + self.bias[e].double().abs()
            z, zsize = y[:, :self.n], size[:, :self.n]
            act = R.act(z, self.act)
            # three float32 roundings of the sum, and an activation within 2e-7 of its argument's size, of slope below 1.13
            off = 2.0 ** -21 * zsize + 1e-6 * zsize * (self.act >= GELU)
            if self.gated:
                up, usize = y[:, self.n:], size[:, self.n:]
                off = off * up.abs() + (act.abs() + off) * 2.0 ** -21 * usize + 2.0 ** -23 * (act * up).abs()
                act = act * up
            out[at], bound[at] = act, off + R.rounding(act, self.kind)
        return out, bound

    def check(self, M, **how):
        import torch
        got = self.call(M, **how).cpu()
        want, bound = self.exact()
        off = (got[:self.used, :self.n].double() - want).abs()
        if self.kind == F16:  # past the type's range an infinity
            past = (got[:self.used, :self.n].double() == torch.copysign(torch.full_like(want, float("inf")), want)) & (want.abs() + bound >= 65520)
            off = torch.where(past, torch.zeros_like(off), off)
        assert (off <= bound).all(), (self.experts, self.n, self.k, float((off / bound).nan_to_num(1e9).max()))
        assert (got[self.used:] == 3).all() and (got[:, self.n:] == 3).all()  # rows behind the last, and between the rows
        return got


SHAPES = [(1, 1), (16, 64), (17, 5), (64, 128), (48, 256), (128, 512), (129, 130), (200, 192), (256, 1024), (320, 77), (512, 640), (33, 4096)]


@pytest.mark.parametrize("n,k", SHAPES)
@pytest.mark.parametrize("experts,rows,skew", [(1, 1, 1.0), (4, 3, 1.0), (8, 60, 0.5), (8, 500, 0.3), (40, 130, 2.0), (3, 700, 0.5)])
def test_experts(gpu, n, k, experts, rows, skew):
    i = SHAPES.index((n, k)) + rows
    counts = _counts(experts, rows, i, skew)
    for j, (pad, gated, gather) in enumerate([(0, False, True), (0, True, False), (16, True, True), (5, i % 2 == 0, i % 3 == 0)]):
        Case(counts, n, k, top=1 + (i + j) % 3, gated=gated, gather=gather, pad=pad, kind=(i + j) % 3, act=(i + j) % 5, seed=i).check(gpu)


@pytest.mark.parametrize("rows", [1, 2, 15, 16, 17, 31, 32, 33, 63, 64, 65, 127, 128, 129, 255, 256, 257])
def test_rows_of_an_expert_at_the_tiles_edges(gpu, rows):
    for kind, gated in ((BF16, True), (F32, False)):
        Case([0, rows, 1, 0, rows, 0], 272, 384, gated=gated, kind=kind, act=SILU, seed=rows).check(gpu)
        Case([rows] * 5, 96, 256, gated=gated, kind=kind, act=GELU, seed=rows, gather=False).check(gpu)


@pytest.mark.parametrize("k", [1, 15, 16, 17, 63, 64, 65, 127, 128, 129, 191, 192, 256, 320, 500, 2048])
def test_lengths_of_the_sum(gpu, k):
    for pad in (0, (-k) % 16, 3):
        Case([3, 20, 0, 100], 80, k, kind=F32, pad=pad, seed=k, act=RELU).check(gpu)
        Case([3, 2, 0, 1], 80, k, kind=F32, pad=pad, seed=k, gated=True, act=GELU_TANH).check(gpu)


@pytest.mark.parametrize("n", [1, 2, 3, 4, 5, 15, 16, 17, 31, 32, 33, 63, 65, 127, 128, 130, 255, 258])
def test_columns(gpu, n):
    for counts in ([2, 0, 5], [90, 40, 300]):
        Case(counts, n, 192, kind=F16, seed=n, gated=True, act=SILU).check(gpu)
        Case(counts, n, 192, kind=BF16, seed=n, pad=16).check(gpu)
        Case(counts, n, 192, kind=F32, seed=n).check(gpu)


@pytest.mark.parametrize("shift", [1, 4, 8, 16])
def test_operands_at_other_addresses(gpu, shift):
    for counts in ([2, 0, 5], [90, 40, 300]):
        Case(counts, 144, 256, kind=BF16, seed=shift, gated=True, act=SILU, shift=shift).check(gpu)
        Case(counts, 144, 256, kind=F32, seed=shift, shift=shift).check(gpu)


@pytest.mark.parametrize("counts", [[3, 0, 2], [200, 90, 0, 400]])
def test_parts_left_out(gpu, counts):
    for kind in (F32, BF16, F16):
        Case(counts, 160, 256, kind=kind, scales=False, bias=False).check(gpu)
        Case(counts, 160, 256, kind=kind, bias=False, gated=True, act=SILU).check(gpu)
        Case(counts, 160, 0, kind=kind, act=SILU, gated=True).check(gpu)


def test_many_experts(gpu):
    for experts in (63, 64, 65, 1000, 1024):
        Case(_counts(experts, 900, experts, 0.2), 48, 128, gated=True, act=SILU, seed=1).check(gpu)
        Case(_counts(experts, experts // 2, experts, 5.0), 64, 64, kind=F32, seed=2).check(gpu)
        Case([0] * (experts - 1) + [5], 64, 64, kind=F32, seed=3).check(gpu)


@pytest.mark.parametrize("counts", [[30, 0, 2, 9], [300, 200, 0, 129]])
def test_rows_that_a_does_not_have(gpu, counts):
    """An index outside A, as a damaged order would hold, reads zeros."""
    for kind in (F32, BF16):
        c = Case(counts, 96, 192, kind=kind, act=SILU, gated=True, top=3)
        c.order[1], c.order[5], c.order[20], c.order[40] = -1, c.a_rows * 3, 2 ** 31 - 1, -2 ** 31
        c.check(gpu)
        c = Case(counts, 96, 192, kind=kind, top=1, scales=False)
        c.order[0], c.order[7], c.order[30] = -5, c.a_rows, 2 ** 30
        c.check(gpu)


@pytest.mark.parametrize("n,k,pad", [(64, 128, 0), (256, 256, 0), (60, 100, 3)])
def test_starts_beyond_the_bound_and_out_of_order(gpu, n, k, pad):
    """Rows beyond the bound are cut; starts that fall name no rows outside it."""
    import torch
    c = Case([40, 30, 50], n, k, kind=F32, behind=0, gather=False, pad=pad)
    whole = c.call(gpu).clone()
    c.starts = torch.tensor([0, 40, 70, 5000], dtype=torch.int32)
    assert torch.equal(c.call(gpu, bound=2)[:120], whole)
    assert (c.call(gpu, bound=2)[120:] == 3).all()
    for starts in ([-9, 40, 70, 120], [0, 100, 20, 120], [130, 120, 60, 0], [2 ** 31 - 1, -2 ** 31, 2 ** 31 - 1, -2 ** 31]):
        c.starts = torch.tensor(starts, dtype=torch.int32)
        assert (c.call(gpu, bound=2)[120:] == 3).all()
        if starts[0] == -9:
            assert torch.equal(c.call(gpu), whole)


def test_sums_wrap_as_the_products_do(gpu):
    import torch
    k = 140032  # 140032 * 2^14 is past 2^31
    for rows in (2, 70, 300):
        A = torch.full((rows, k), -128, dtype=torch.int8, device="cuda")
        B = torch.full((1, 32, k), -128, dtype=torch.int8, device="cuda")
        C = torch.zeros((rows, 32), device="cuda")
        starts = torch.tensor([0, rows], dtype=torch.int32, device="cuda")
        gpu.mipgemm_s8s8_experts(rows, 1, 32, k, A, k, rows, None, starts, None, 1, B, k, 32 * k, None, None, 0, 0, C, 32, F32)
        assert (C == float(np.float32(k * 16384 - 2 ** 32))).all()


@pytest.mark.parametrize("rows", [3, 300])
def test_offsets_that_pass_31_and_32_bits(gpu, rows):
    import torch
    g = torch.Generator().manual_seed(4)
    k, n = 128, 4096
    small = torch.randint(-127, 128, (rows, k), generator=g, dtype=torch.int8)
    weights = torch.randint(-127, 128, (2, n, k), generator=g, dtype=torch.int8)
    want = torch.cat([small[:rows // 3].double() @ weights[0].double().T, small[rows // 3:].double() @ weights[1].double().T])
    starts = torch.tensor([0, rows // 3, rows], dtype=torch.int32, device="cuda")
    for lda, ldb, strideB in ((1 << 14, k, n * k), (1 << 15, k, n * k), (k, 800000, 800000 * n), (k, 1 << 20, n << 20), (k, k, 5 * (1 << 30))):
        a_rows = 200000 if lda > k else rows  # 3.3 or 6.6 GB
        A = torch.empty((a_rows, lda), dtype=torch.int8, device="cuda")
        at = torch.arange(a_rows - rows, a_rows)
        A[at.cuda(), :k] = small.cuda()
        B = torch.empty(strideB + (n - 1) * ldb + k, dtype=torch.int8, device="cuda")
        for e in range(2):
            torch.as_strided(B, (n, k), (ldb, 1), e * strideB).copy_(weights[e])
        C = torch.zeros((rows, n), device="cuda")
        gpu.mipgemm_s8s8_experts(rows, 2, n, k, A, lda, a_rows, None, starts, at.to(torch.int32).cuda(), 1, B, ldb, strideB, None, None, 0, 0, C, n, F32)
        assert torch.equal(C.double().cpu(), want), (lda, ldb, strideB)
        del A, B


def test_scales_that_are_no_numbers_stay_in_their_rows_and_columns(gpu):
    import torch
    for counts in ([3, 4], [150, 200]):
        c = Case(counts, 64, 128, kind=F32, bias=False, gather=False)
        c.a[1], c.b[1, 7] = float("nan"), float("inf")
        got = c.call(gpu).cpu()
        bad = torch.zeros((c.used, c.n), dtype=torch.bool)
        bad[1] = True
        bad[counts[0]:, 7] = True
        assert torch.equal(~torch.isfinite(got[:c.used, :64]), bad)


def test_experts_in_a_graph_and_on_another_stream(gpu):
    """Captured once, replayed over other routings and activations, against eager calls."""
    import torch
    experts, n, k, tokens, top = 6, 128, 256, 90, 2
    g = torch.Generator().manual_seed(3)
    B = torch.randint(-127, 128, (experts, 2 * n, k), generator=g, dtype=torch.int8).cuda()
    b = (torch.rand((experts, 2 * n), generator=g) * 0.01).cuda()
    A = torch.zeros((tokens, k), dtype=torch.int8, device="cuda")
    a = torch.ones(tokens, device="cuda")
    starts = torch.zeros(experts + 1, dtype=torch.int32, device="cuda")
    order = torch.zeros(tokens * top, dtype=torch.int32, device="cuda")

    def call(C):
        gpu.mipgemm_s8s8_experts(tokens * top, experts, n, k, A, k, tokens, a, starts, order, top, B, k, 2 * n * k, b, None, SILU, 1, C, n, BF16)
    out = torch.zeros((tokens * top, n), dtype=torch.bfloat16, device="cuda")
    call(out)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call(out)
    for i in range(4):
        A.copy_(torch.randint(-127, 128, (tokens, k), generator=g, dtype=torch.int8))
        starts.copy_(torch.tensor([0] + list(_counts(experts, tokens * top - 20 * i, i, 0.6))).cumsum(0))
        order.copy_(torch.randperm(tokens * top, generator=g))
        out.zero_()
        graph.replay()
        torch.cuda.synchronize()
        got, eager = out.clone(), torch.zeros_like(out)
        call(eager)
        torch.cuda.synchronize()
        assert torch.equal(got, eager), i
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            call(eager.zero_())
        side.synchronize()
        assert torch.equal(got, eager), i


# ---- the kernels for many rows, by name: sizes that the kernel of 16 rows to a workgroup leaves to them ----

def _served(kernels_of, gpu, case):
    """The kernel that serves a case, with its template's arguments."""
    names = [re.search(r"experts_\w*kernel<[^>]*>", n) for n in kernels_of(lambda: case.call(gpu))]
    names = [n.group(0) for n in names if n]
    assert len(names) == 1, names
    return names[0]


RAGGED = [129, 1, 0, 257]                 # experts whose rows end inside tiles of 128
FEW = [40, 13, 64, 0, 1, 65, 20, 33]      # 13 to 64 rows to an expert on average
LONG = [700, 70]                          # at least 384, over a k of 4096 and more


@pytest.mark.parametrize("k", [16, 112, 128, 144, 256, 272, 400])
@pytest.mark.parametrize("gated", [False, True])
def test_tiles_of_many_rows(gpu, kernels_of, k, gated):
    """One block of k, several, and what is left of it; columns that end inside a tile, at its end and one behind it."""
    for i, n in enumerate((1250, 1280, 1217) if gated else (2501, 2560, 2433)):
        for pad in (0, 16):
            j = i + k // 16 + pad // 16
            case = Case(RAGGED, n, k, top=1 + j % 3, gated=gated, gather=j % 2 == 0, pad=pad, kind=j % 3, act=j % 5, bias=j % 4 > 0, seed=j)
            if i == 0:
                assert _served(kernels_of, gpu, case) == "experts_tile_kernel<128, 128, %d>" % gated
            case.check(gpu)


@pytest.mark.parametrize("act", [NONE, RELU, GELU, GELU_TANH, SILU])
@pytest.mark.parametrize("gated", [False, True])
def test_tiles_in_every_type_and_activation(gpu, act, gated):
    for kind in (F32, BF16, F16):
        Case([128, 300, 2, 31], 1251 if gated else 2500, 208, gated=gated, kind=kind, act=act, seed=act, gather=kind != F16).check(gpu)
        Case([128, 300, 2, 31], 1251 if gated else 2500, 208, gated=gated, kind=kind, act=act, seed=act, scales=False, bias=kind == F32, behind=0).check(gpu)


@pytest.mark.parametrize("k", [4096, 4112, 4208])
@pytest.mark.parametrize("gated", [False, True])
def test_large_tiles_under_a_long_sum(gpu, kernels_of, k, gated):
    for i, (counts, n) in enumerate([(LONG, 700), ([384, 0, 769], 640), ([385], 1281)] if gated else [(LONG, 1345), ([384, 0, 769], 1280), ([385], 2561)]):
        j = i + k // 16 + gated
        case = Case(counts, n, k, top=1 + j % 2, gated=gated, gather=j % 2 == 0, pad=16 * (i % 2), kind=j % 3, act=(NONE, SILU, GELU)[j % 3],
                    bias=i > 0, seed=j)
        assert _served(kernels_of, gpu, case) == "experts_tile_kernel<192, 256, %d>" % gated
        case.check(gpu)


@pytest.mark.parametrize("counts,blocks", [(FEW, 1), (RAGGED, 2)])
@pytest.mark.parametrize("k", [1, 15, 17, 63, 65, 100, 130, 200])
@pytest.mark.parametrize("gated", [False, True])
def test_unaligned_rows_of_many(gpu, kernels_of, counts, blocks, k, gated):
    for i, n in enumerate((1601, 1664) if gated else (3101, 3200)):
        for pad in (0, 3):
            j = i + k + pad
            case = Case(counts, n, k, top=1 + j % 3, gated=gated, gather=j % 2 == 0, pad=pad, kind=j % 3, act=(j // 2) % 5, bias=j % 4 > 0, seed=j)
            if i == 0 and pad == 0:
                assert _served(kernels_of, gpu, case) == "experts_kernel<%d, %d>" % (gated, blocks)
            case.check(gpu)


@pytest.mark.parametrize("counts,blocks", [(FEW, 1), (RAGGED, 2)])
@pytest.mark.parametrize("shift,pad", [(1, 0), (8, 0), (4, 16), (0, 8)])
def test_unaligned_places_of_many_rows(gpu, kernels_of, counts, blocks, shift, pad):
    for gated in (False, True):
        case = Case(counts, 1601 if gated else 3101, 192, gated=gated, kind=BF16 if gated else F32, act=SILU, pad=pad, shift=shift, seed=shift + pad)
        assert _served(kernels_of, gpu, case) == "experts_kernel<%d, %d>" % (gated, blocks)
        case.check(gpu)


# what each kernel for many rows is called with: rows of the experts, columns, k, padding
MANY = [(RAGGED, 2501, 272, 0), (LONG, 1345, 4112, 0), (FEW, 3101, 130, 0), (RAGGED, 2501, 200, 3)]


@pytest.mark.parametrize("counts,n,k,pad", MANY)
def test_rows_that_a_does_not_have_among_many(gpu, counts, n, k, pad):
    for gated in (False, True):
        c = Case(counts, n, k, top=3, pad=pad, gated=gated, kind=F32 if gated else BF16, act=SILU)
        c.order[1], c.order[5], c.order[20], c.order[40], c.order[131] = -1, c.a_rows * 3, 2 ** 31 - 1, -2 ** 31, -7
        c.check(gpu)


@pytest.mark.parametrize("counts,n,k,pad", MANY)
def test_starts_of_many_rows_beyond_the_bound_and_out_of_order(gpu, counts, n, k, pad):
    import torch
    c = Case(counts, n, k, kind=F32, behind=0, gather=False, pad=pad)
    whole, used = c.call(gpu).clone(), c.used
    fine = c.starts.clone()
    c.starts = fine.clone()
    c.starts[-1] = 2 ** 31 - 1
    assert torch.equal(c.call(gpu, bound=2)[:used], whole)
    for at, to in ((0, -9), (0, 100), (1, 2 ** 31 - 1), (1, -2 ** 31), (-1, 50)):
        c.starts = fine.clone()
        c.starts[at] = to
        got = c.call(gpu, bound=2)
        assert (got[used:] == 3).all()
        if to == -9:
            assert torch.equal(got[:used], whole)


@pytest.mark.parametrize("counts,n,k,pad", MANY)
def test_scales_of_many_rows_that_are_no_numbers(gpu, counts, n, k, pad):
    import torch
    c = Case(counts, n, k, kind=F32, bias=False, gather=False, pad=pad)
    last = max(e for e, rows in enumerate(counts) if rows)
    c.a[1], c.b[last, 7], c.b[last, n - 1] = float("nan"), float("inf"), float("nan")
    got = c.call(gpu).cpu()
    bad = torch.zeros((c.used, n), dtype=torch.bool)
    bad[1] = True
    bad[c.used - counts[last]:, 7] = bad[c.used - counts[last]:, n - 1] = True
    assert torch.equal(~torch.isfinite(got[:c.used, :n]), bad)


@pytest.mark.parametrize("rows,n,pad", [(300, 3500, 0), (400, 2600, 0), (300, 3500, 1), (50, 16400, 1)])
def test_sums_of_many_rows_wrap_as_the_products_do(gpu, rows, n, pad):
    import torch
    k = 140032  # 140032 * 2^14 is past 2^31
    A = torch.full((rows, k + pad), -128, dtype=torch.int8, device="cuda")
    B = torch.full((1, n, k + pad), -128, dtype=torch.int8, device="cuda")
    C = torch.zeros((rows, n), device="cuda")
    starts = torch.tensor([0, rows], dtype=torch.int32, device="cuda")
    gpu.mipgemm_s8s8_experts(rows, 1, n, k, A, k + pad, rows, None, starts, None, 1, B, k + pad, n * (k + pad), None, None, 0, 0, C, n, F32)
    assert (C == float(np.float32(k * 16384 - 2 ** 32))).all()


@pytest.mark.parametrize("counts,n,k,pad", MANY)
def test_many_rows_in_a_graph(gpu, counts, n, k, pad):
    """Captured once, replayed over other rows of the experts and other codes, against eager calls."""
    import torch
    c = Case(counts, n, k, top=1, kind=BF16, act=RELU, pad=pad)
    g = torch.Generator().manual_seed(3)
    lead, rows = k + pad, c.rows
    A, B = c.A.cuda(), c.B.cuda()
    a, b, bias, starts, order = (x.cuda() for x in (c.a, c.b, c.bias, c.starts, c.order))
    out = torch.zeros((rows, n), dtype=torch.bfloat16, device="cuda")

    def call(C):
        gpu.mipgemm_s8s8_experts(rows, c.experts, n, k, A, lead, c.a_rows, a, starts, order, 1, B, lead, n * lead, b, bias, RELU, 0, C, n, BF16)
    call(out)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call(out)
    for i in range(4):
        A.copy_(torch.randint(-127, 128, A.shape, generator=g, dtype=torch.int8))
        starts.copy_(torch.tensor([0] + list(_counts(c.experts, rows - 30 * i, i, 0.6))).cumsum(0))
        order.copy_(torch.randperm(c.a_rows, generator=g)[:rows])
        out.zero_()
        graph.replay()
        torch.cuda.synchronize()
        got, eager = out.clone(), torch.zeros_like(out)
        call(eager)
        torch.cuda.synchronize()
        assert torch.equal(got, eager), i
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            call(eager.zero_())
        side.synchronize()
        assert torch.equal(got, eager), i
