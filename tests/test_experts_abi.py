"""Refusals of the operators of a mixture of experts: every invalid argument is reported by its number, before anything is
enqueued (none of these calls needs a GPU), and empty calls succeed."""
import math
import os
import re

import pytest


@pytest.fixture(scope="module")
def M():
    import paper_2506_11728_amd as M
    if not os.path.exists(M.library_path()):
        from paper_2506_11728_amd.build import build_library
        build_library()
    M.load_library()
    return M


X = 4096  # stands for an address: no call below gets as far as using it
BIG = 2 ** 31
NEED = 32 + 70  # 3 blocks of tokens x 8 experts, up to a multiple of 16, and a rank to each row

ROUTE = dict(tokens=70, experts=8, top=1, logits=X, ldl=8, type=0, bias=X, scoring=0, groups=2, top_groups=1, group_best=2, normalise=1,
             scale=1.0, ids=X, weights=X, starts=X, order=X, places=X, workspace=X, workspace_bytes=1 << 20)
EXPERTS = dict(rows=6, experts=3, n=5, k=7, A=X, lda=7, a_rows=2, a_scales=X, starts=X, order=X, top=3, B=X, ldb=8, strideB=40, b_scales=X,
               bias=X, activation=0, gated=0, C=X, ldc=5, c_type=1)
JOIN = dict(rows=4, cols=8, parts=2, type=1, X=X, ldx=8, x_rows=8, places=None, weights=X, post_norm=1, post_weight=X, post_bias=X, gate=X,
            ldg=8, gate_rows=1, scale=1.0, R=X, ldr=8, H=X + 1024, ldh=8, norm=2, norm_weight=X, norm_bias=X, eps=1e-6, N=X, ldn=8, Q=X, ldq=8,
            scales=X)
ENTRIES = {"mipgemm_route": ROUTE, "mipgemm_s8s8_experts": EXPERTS, "mipgemm_join_rows": JOIN}

WRONG = [
    ("mipgemm_route", 1, dict(tokens=-1)), ("mipgemm_route", 1, dict(tokens=2 ** 26 + 1)),
    ("mipgemm_route", 1, dict(tokens=2 ** 26, experts=64, ldl=64, top=32, groups=1)), ("mipgemm_route", 2, dict(experts=0)),
    ("mipgemm_route", 2, dict(experts=1025, ldl=2000)), ("mipgemm_route", 3, dict(top=0)), ("mipgemm_route", 3, dict(top=9)),
    ("mipgemm_route", 3, dict(top=5)), ("mipgemm_route", 3, dict(experts=64, ldl=64, top=33, groups=1)),
    ("mipgemm_route", 4, dict(logits=None)), ("mipgemm_route", 5, dict(ldl=7)), ("mipgemm_route", 5, dict(ldl=BIG)),
    ("mipgemm_route", 6, dict(type=3)), ("mipgemm_route", 6, dict(type=-1)), ("mipgemm_route", 8, dict(scoring=2)),
    ("mipgemm_route", 9, dict(groups=0)), ("mipgemm_route", 9, dict(groups=3)), ("mipgemm_route", 9, dict(groups=128, experts=128, ldl=128)),
    ("mipgemm_route", 10, dict(top_groups=0)), ("mipgemm_route", 10, dict(top_groups=3)), ("mipgemm_route", 11, dict(group_best=0)),
    ("mipgemm_route", 11, dict(group_best=3)), ("mipgemm_route", 11, dict(groups=8)), ("mipgemm_route", 13, dict(scale=math.inf)),
    ("mipgemm_route", 13, dict(scale=math.nan)), ("mipgemm_route", 14, dict(ids=None)), ("mipgemm_route", 15, dict(weights=None)),
    ("mipgemm_route", 19, dict(workspace=None)), ("mipgemm_route", 19, dict(workspace=X + 8)),
    ("mipgemm_route", 20, dict(workspace_bytes=NEED - 1)),
    ("mipgemm_route", 20, dict(workspace=None, workspace_bytes=0)),
    ("mipgemm_s8s8_experts", 1, dict(rows=-1)), ("mipgemm_s8s8_experts", 1, dict(rows=BIG)), ("mipgemm_s8s8_experts", 2, dict(experts=0)),
    ("mipgemm_s8s8_experts", 2, dict(experts=1025)), ("mipgemm_s8s8_experts", 3, dict(n=-1)), ("mipgemm_s8s8_experts", 3, dict(n=BIG)),
    ("mipgemm_s8s8_experts", 3, dict(n=2 ** 30, gated=1)), ("mipgemm_s8s8_experts", 4, dict(k=-1)), ("mipgemm_s8s8_experts", 5, dict(A=None)),
    ("mipgemm_s8s8_experts", 6, dict(lda=6)), ("mipgemm_s8s8_experts", 7, dict(a_rows=0)),
    ("mipgemm_s8s8_experts", 7, dict(a_rows=5, order=None)), ("mipgemm_s8s8_experts", 9, dict(starts=None)),
    ("mipgemm_s8s8_experts", 11, dict(top=0)), ("mipgemm_s8s8_experts", 12, dict(B=None)), ("mipgemm_s8s8_experts", 13, dict(ldb=6)),
    ("mipgemm_s8s8_experts", 14, dict(strideB=39)), ("mipgemm_s8s8_experts", 14, dict(strideB=79, gated=1)),
    ("mipgemm_s8s8_experts", 14, dict(strideB=2 ** 52 + 1)), ("mipgemm_s8s8_experts", 17, dict(activation=5)),
    ("mipgemm_s8s8_experts", 17, dict(activation=-1)), ("mipgemm_s8s8_experts", 19, dict(C=None)), ("mipgemm_s8s8_experts", 20, dict(ldc=4)),
    ("mipgemm_s8s8_experts", 21, dict(c_type=3)),
    ("mipgemm_join_rows", 1, dict(rows=-1)), ("mipgemm_join_rows", 1, dict(rows=BIG)), ("mipgemm_join_rows", 2, dict(cols=-1)),
    ("mipgemm_join_rows", 2, dict(cols=16385)), ("mipgemm_join_rows", 3, dict(parts=0)), ("mipgemm_join_rows", 3, dict(parts=1025)),
    ("mipgemm_join_rows", 4, dict(type=3)), ("mipgemm_join_rows", 5, dict(X=None)), ("mipgemm_join_rows", 6, dict(ldx=7)),
    ("mipgemm_join_rows", 7, dict(x_rows=7)), ("mipgemm_join_rows", 7, dict(x_rows=-1, places=X)), ("mipgemm_join_rows", 7, dict(x_rows=BIG)),
    ("mipgemm_join_rows", 10, dict(post_norm=3)), ("mipgemm_join_rows", 10, dict(post_norm=-1)), ("mipgemm_join_rows", 14, dict(ldg=7)),
    ("mipgemm_join_rows", 15, dict(gate_rows=0)), ("mipgemm_join_rows", 16, dict(scale=math.inf)), ("mipgemm_join_rows", 16, dict(scale=math.nan)),
    ("mipgemm_join_rows", 18, dict(ldr=7)), ("mipgemm_join_rows", 20, dict(ldh=7)), ("mipgemm_join_rows", 20, dict(H=X, ldh=9)),
    ("mipgemm_join_rows", 21, dict(norm=3)), ("mipgemm_join_rows", 24, dict(eps=-1.0)), ("mipgemm_join_rows", 24, dict(eps=math.nan)),
    ("mipgemm_join_rows", 24, dict(eps=math.inf)), ("mipgemm_join_rows", 26, dict(ldn=7)), ("mipgemm_join_rows", 27, dict(Q=None)),
    ("mipgemm_join_rows", 28, dict(ldq=7)), ("mipgemm_join_rows", 29, dict(scales=None)),
]


@pytest.mark.parametrize("native", [True, False])
def test_refusals(M, native, monkeypatch):
    from paper_2506_11728_amd import binding
    if not native:
        monkeypatch.setattr(binding, "_native", None)  # the arguments' conversion through ctypes
    for name, number, change in WRONG:
        got = getattr(M, name)(**{**ENTRIES[name], **change}, stream=0, check=False)
        assert got == -number, (name, change, got)
        assert str(number) in M.mipgemm_strerror(got)
        with pytest.raises(M.MipGemmError) as refused:
            getattr(M, name)(**{**ENTRIES[name], **change}, stream=0)
        assert refused.value.code == -number


def test_empty_calls_enqueue_nothing(M):
    for name, change in [
            ("mipgemm_route", dict(tokens=0, logits=None, ids=None, weights=None, starts=None, order=None, places=None, workspace=None,
                                   workspace_bytes=0)),
            ("mipgemm_s8s8_experts", dict(rows=0, a_rows=0, A=None, B=None, C=None, starts=None)),
            ("mipgemm_s8s8_experts", dict(n=0, A=None, B=None, C=None, starts=None)),
            ("mipgemm_join_rows", dict(rows=0, x_rows=0, X=None, R=None, H=None, N=None, Q=None, scales=None)),
            ("mipgemm_join_rows", dict(H=None, N=None, Q=None, scales=None))]:
        assert getattr(M, name)(**{**ENTRIES[name], **change}, stream=0) == 0, (name, change)


def test_workspace_sizes(M):
    assert M.mipgemm_route_workspace_size(32, 256, 8) == 0
    assert M.mipgemm_route_workspace_size(70, 8, 1) == NEED
    for bad in ((-1, 8, 2), (2 ** 26 + 1, 8, 1), (100, 0, 1), (100, 1025, 1), (100, 8, 9), (100, 8, 0), (2 ** 26, 64, 32)):
        assert M.mipgemm_route_workspace_size(*bad) == 0


def test_header_constants_match_the_binding(M):
    header = open(os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "include", "mipgemm.h")).read()
    consts = dict(re.findall(r"#define\s+MIPGEMM_(\w+)\s+(\d+)\b", header))
    for name in ("SOFTMAX", "SIGMOID", "NO_NORM", "RMS_NORM", "LAYER_NORM"):
        assert int(consts[name]) == getattr(M, name)
