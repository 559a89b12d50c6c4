"""Refusals of the operators between the products of a layer: every invalid argument is reported by its number,
before anything is enqueued (none of these calls needs a GPU), and empty calls succeed."""
import math

import pytest


@pytest.fixture(scope="module")
def M():
    import os

    import paper_2506_11728_amd as M
    if not os.path.exists(M.library_path()):
        from paper_2506_11728_amd.build import build_library
        build_library()
    M.load_library()
    return M


X = 4096  # stands for an address: no call below gets as far as using it

QUANTIZE = dict(rows=4, cols=8, X=X, ldx=8, x_type=1, norm_weight=X, eps=1e-6, Q=X, ldq=8, scales=X)
LINEAR = dict(m=4, n=5, k=6, A=X, lda=6, a_scales=X, B=X, ldb=6, orderB=1, b_scales=X, bias=X, activation=0, R=X, ldr=5,
              C=X, ldc=5, c_type=1, workspace=None, workspace_bytes=0)
ROPE = dict(tokens=4, q_heads=4, kv_heads=2, head_dim=64, type=1, Q=X, ldq=256, K=X, ldk=128, V=X, ldv=128, q_weight=X,
            k_weight=X, eps=1e-6, cosine=X, sine=X, table_rows=10, rot_dim=64, style=0, positions=X, Qo=X, ldqo=256, Ko=X,
            ldko=128, cache=X, cache_bytes=2 * 32 * 2 * 72, pages=2, page_tokens=32, slots=X)
READ = dict(tokens=4, kv_heads=2, head_dim=64, type=1, cache=X, cache_bytes=2 * 32 * 2 * 72, pages=2, page_tokens=32, slots=X,
            K=X, ldk=128, V=X, ldv=128)
ATTENTION = dict(requests=2, q_heads=4, kv_heads=2, head_dim=64, type=1, Q=X, ldq=256, q_rows=2, q_starts=X, max_q=1, kv_lengths=X,
                 max_kv=64, cache=X, cache_bytes=2 * 32 * 2 * 72, pages=2, page_tokens=32, block_table=X, table_stride=2, scale=0.1,
                 O=X, ldo=256, workspace=None, workspace_bytes=0)
ENTRIES = {"mipgemm_quantize_rows": QUANTIZE, "mipgemm_s8s8_linear": LINEAR, "mipgemm_qk_norm_rope": ROPE,
           "mipgemm_kv4_read": READ, "mipgemm_attention_kv4": ATTENTION}
BIG = 2 ** 31

WRONG = [
    ("mipgemm_quantize_rows", 1, dict(rows=-1)), ("mipgemm_quantize_rows", 1, dict(rows=BIG)),
    ("mipgemm_quantize_rows", 2, dict(cols=-1)), ("mipgemm_quantize_rows", 3, dict(X=None)),
    ("mipgemm_quantize_rows", 4, dict(ldx=7)), ("mipgemm_quantize_rows", 5, dict(x_type=3)),
    ("mipgemm_quantize_rows", 5, dict(x_type=-1)), ("mipgemm_quantize_rows", 7, dict(eps=-1.0)),
    ("mipgemm_quantize_rows", 7, dict(eps=math.inf)), ("mipgemm_quantize_rows", 7, dict(eps=math.nan)),
    ("mipgemm_quantize_rows", 8, dict(Q=None)), ("mipgemm_quantize_rows", 9, dict(ldq=7)),
    ("mipgemm_quantize_rows", 10, dict(scales=None)),
    ("mipgemm_s8s8_linear", 1, dict(m=-1)), ("mipgemm_s8s8_linear", 2, dict(n=BIG)), ("mipgemm_s8s8_linear", 3, dict(k=-3)),
    ("mipgemm_s8s8_linear", 4, dict(A=None)), ("mipgemm_s8s8_linear", 5, dict(lda=5)), ("mipgemm_s8s8_linear", 7, dict(B=None)),
    ("mipgemm_s8s8_linear", 8, dict(ldb=5)), ("mipgemm_s8s8_linear", 8, dict(orderB=0, ldb=4)),
    ("mipgemm_s8s8_linear", 9, dict(orderB=2)), ("mipgemm_s8s8_linear", 12, dict(activation=5)),
    ("mipgemm_s8s8_linear", 12, dict(activation=-1)), ("mipgemm_s8s8_linear", 14, dict(ldr=4)),
    ("mipgemm_s8s8_linear", 15, dict(C=None)), ("mipgemm_s8s8_linear", 16, dict(ldc=4)), ("mipgemm_s8s8_linear", 17, dict(c_type=7)),
    ("mipgemm_s8s8_linear", 18, dict(workspace_bytes=64)), ("mipgemm_s8s8_linear", 5, dict(lda=1, activation=9, ldc=1)),
    ("mipgemm_qk_norm_rope", 1, dict(tokens=-1)), ("mipgemm_qk_norm_rope", 2, dict(q_heads=1025)),
    ("mipgemm_qk_norm_rope", 3, dict(kv_heads=-1)), ("mipgemm_qk_norm_rope", 4, dict(head_dim=96)),
    ("mipgemm_qk_norm_rope", 5, dict(type=3)), ("mipgemm_qk_norm_rope", 6, dict(Q=None)), ("mipgemm_qk_norm_rope", 7, dict(ldq=255)),
    ("mipgemm_qk_norm_rope", 8, dict(K=None)), ("mipgemm_qk_norm_rope", 9, dict(ldk=127)), ("mipgemm_qk_norm_rope", 10, dict(V=None)),
    ("mipgemm_qk_norm_rope", 11, dict(ldv=127)), ("mipgemm_qk_norm_rope", 14, dict(eps=-1e-9)),
    ("mipgemm_qk_norm_rope", 15, dict(cosine=None)), ("mipgemm_qk_norm_rope", 16, dict(sine=None)),
    ("mipgemm_qk_norm_rope", 17, dict(table_rows=-1)), ("mipgemm_qk_norm_rope", 18, dict(rot_dim=66)),
    ("mipgemm_qk_norm_rope", 18, dict(rot_dim=31)), ("mipgemm_qk_norm_rope", 19, dict(style=2)),
    ("mipgemm_qk_norm_rope", 20, dict(positions=None)), ("mipgemm_qk_norm_rope", 21, dict(Qo=None)),
    ("mipgemm_qk_norm_rope", 22, dict(ldqo=255)), ("mipgemm_qk_norm_rope", 24, dict(ldko=127)),
    ("mipgemm_qk_norm_rope", 25, dict(cache=X + 8)), ("mipgemm_qk_norm_rope", 26, dict(cache_bytes=2 * 32 * 2 * 72 - 1)),
    ("mipgemm_qk_norm_rope", 27, dict(pages=-1)), ("mipgemm_qk_norm_rope", 28, dict(page_tokens=24)),
    ("mipgemm_qk_norm_rope", 28, dict(page_tokens=8)), ("mipgemm_qk_norm_rope", 28, dict(page_tokens=2048)),
    ("mipgemm_qk_norm_rope", 29, dict(slots=None)),
    ("mipgemm_kv4_read", 1, dict(tokens=-1)), ("mipgemm_kv4_read", 2, dict(kv_heads=-2)), ("mipgemm_kv4_read", 3, dict(head_dim=80)),
    ("mipgemm_kv4_read", 4, dict(type=9)), ("mipgemm_kv4_read", 5, dict(cache=None)), ("mipgemm_kv4_read", 5, dict(cache=X + 1)),
    ("mipgemm_kv4_read", 6, dict(cache_bytes=0)), ("mipgemm_kv4_read", 7, dict(pages=-1)), ("mipgemm_kv4_read", 8, dict(page_tokens=0)),
    ("mipgemm_kv4_read", 9, dict(slots=None)), ("mipgemm_kv4_read", 11, dict(ldk=1)), ("mipgemm_kv4_read", 13, dict(ldv=1)),
    ("mipgemm_attention_kv4", 1, dict(requests=-1)), ("mipgemm_attention_kv4", 2, dict(q_heads=0)),
    ("mipgemm_attention_kv4", 3, dict(kv_heads=3)), ("mipgemm_attention_kv4", 3, dict(kv_heads=0)),
    ("mipgemm_attention_kv4", 4, dict(head_dim=32)), ("mipgemm_attention_kv4", 5, dict(type=0)),
    ("mipgemm_attention_kv4", 6, dict(Q=None)), ("mipgemm_attention_kv4", 7, dict(ldq=255)),
    ("mipgemm_attention_kv4", 8, dict(q_rows=-1)), ("mipgemm_attention_kv4", 9, dict(q_starts=None)),
    ("mipgemm_attention_kv4", 10, dict(max_q=-1)), ("mipgemm_attention_kv4", 10, dict(max_q=BIG - 1)),
    ("mipgemm_attention_kv4", 11, dict(kv_lengths=None)), ("mipgemm_attention_kv4", 12, dict(max_kv=-1)),
    ("mipgemm_attention_kv4", 12, dict(max_kv=BIG - 1)), ("mipgemm_attention_kv4", 13, dict(cache=None)),
    ("mipgemm_attention_kv4", 13, dict(cache=X + 4)), ("mipgemm_attention_kv4", 14, dict(cache_bytes=100)),
    ("mipgemm_attention_kv4", 15, dict(pages=-1)), ("mipgemm_attention_kv4", 16, dict(page_tokens=20)),
    ("mipgemm_attention_kv4", 17, dict(block_table=None)), ("mipgemm_attention_kv4", 18, dict(table_stride=-1)),
    ("mipgemm_attention_kv4", 19, dict(scale=0.0)), ("mipgemm_attention_kv4", 19, dict(scale=-1.0)),
    ("mipgemm_attention_kv4", 19, dict(scale=math.nan)), ("mipgemm_attention_kv4", 20, dict(O=None)),
    ("mipgemm_attention_kv4", 21, dict(ldo=255)), ("mipgemm_attention_kv4", 22, dict(workspace_bytes=1)),
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


@pytest.mark.parametrize("q_heads", [1, 2, 64, 1000, 1024])
def test_bounds_whose_products_wrap(M, q_heads):
    """A bound on the queries of a request that passes 64 bits, or comes back into range, times the heads is refused."""
    more = dict(q_heads=q_heads, kv_heads=q_heads, ldq=64 * q_heads, ldo=64 * q_heads, cache_bytes=2 ** 40)
    most = 2 ** 63 - 1
    for max_q in (most, 2 ** 62, 2 ** 55, 2 ** 54, 2 ** 53, min(2 ** 64 // q_heads + 1, most), 2 ** 31, (2 ** 31 - 4097) // q_heads + 1):
        assert M.mipgemm_attention_kv4(**{**ATTENTION, **more, "max_q": max_q}, stream=0, check=False) == -10, max_q
        assert M.mipgemm_attention_kv4_workspace_size(2, q_heads, q_heads, 64, min(max_q + 4096, most), 64) == 0


def test_empty_calls_enqueue_nothing(M):
    for name, change in [
            ("mipgemm_quantize_rows", dict(rows=0, X=None, Q=None, scales=None)),
            ("mipgemm_s8s8_linear", dict(m=0, A=None, C=None, R=None)), ("mipgemm_s8s8_linear", dict(n=0, B=None, C=None, R=None)),
            ("mipgemm_qk_norm_rope", dict(tokens=0, Q=None, K=None, V=None, positions=None, Qo=None, slots=None)),
            ("mipgemm_kv4_read", dict(tokens=0, slots=None)), ("mipgemm_kv4_read", dict(K=None, V=None)),
            ("mipgemm_attention_kv4", dict(requests=0, Q=None, q_starts=None, kv_lengths=None, block_table=None, O=None)),
            ("mipgemm_attention_kv4", dict(q_rows=0, Q=None, O=None)), ("mipgemm_attention_kv4", dict(max_q=0))]:
        assert getattr(M, name)(**{**ENTRIES[name], **change}, stream=0) == 0, (name, change)


def test_sizes(M):
    assert M.mipgemm_kv4_bytes(3, 64, 8, 128) == 3 * 64 * 8 * 128 * 9 // 8
    for bad in ((-1, 64, 8, 128), (3, 65, 8, 128), (3, 64, 8, 100), (3, 64, 5000, 128)):
        assert M.mipgemm_kv4_bytes(*bad) == 0
    assert M.mipgemm_attention_kv4_workspace_size(1, 8, 8, 64, 1, 16) == 0          # one range of keys
    assert M.mipgemm_attention_kv4_workspace_size(1, 32, 8, 128, 1, 100000) > 32 * 132 * 4
    for bad in ((0, 8, 8, 64, 1, 100000), (1, 8, 3, 64, 1, 100000), (1, 8, 8, 65, 1, 100000), (1, 8, 8, 64, -1, 100000)):
        assert M.mipgemm_attention_kv4_workspace_size(*bad) == 0


def test_header_constants_of_the_operators_match_the_binding(M):
    import os
    import re
    header = open(os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "include", "mipgemm.h")).read()
    consts = dict(re.findall(r"#define\s+MIPGEMM_(\w+)\s+(\d+)\b", header))
    for name in ("F32", "BF16", "F16", "NONE", "RELU", "GELU", "GELU_TANH", "SILU", "ROTATE_HALVES", "ROTATE_PAIRS"):
        assert int(consts[name]) == getattr(M, name)
