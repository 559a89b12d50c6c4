// C-ABI entry points of the operators between the integer products of a layer: argument checks.
// Host only.
#include "api_internal.h"
#include "layer_internal.h"
#include "real.h"

extern "C" {

int mipgemm_quantize_rows(int64_t rows, int64_t cols, const void *X, int64_t ldx, int x_type, const float *norm_weight,
                          float eps, int8_t *Q, int64_t ldq, float *scales, void *stream) {
  if (rows < 0 || rows > MIPGEMM_MAX_DIM) return -1;
  if (cols < 0 || cols > MIPGEMM_MAX_DIM) return -2;
  if (!X && rows > 0 && cols > 0) return -3;
  if (ldx < (cols > 1 ? cols : 1) || ldx > MIPGEMM_MAX_DIM) return -4;
  if (!mip::real_type_ok(x_type)) return -5;
  if (!(eps >= 0.0f) || eps - eps != 0.0f) return -7;
  if (!Q && rows > 0 && cols > 0) return -8;
  if (ldq < (cols > 1 ? cols : 1) || ldq > MIPGEMM_MAX_DIM) return -9;
  if (!scales && rows > 0) return -10;
  if (rows == 0) return 0;
  if (cols == 0) norm_weight = nullptr;  // nothing to take a mean of: scales of zero
  return static_cast<int>(mip::launch_quantize(rows, cols, X, ldx, x_type, norm_weight, eps, Q, ldq, scales,
                                               static_cast<hipStream_t>(stream)));
}

int mipgemm_s8s8_linear(int64_t m, int64_t n, int64_t k, const int8_t *A, int64_t lda, const float *a_scales,
                        const int8_t *B, int64_t ldb, int orderB, const float *b_scales, const float *bias,
                        int activation, const void *R, int64_t ldr, void *C, int64_t ldc, int c_type,
                        void *workspace, size_t workspace_bytes, void *stream) {
  mip::Problem checked;
  int rc = mip::validate_and_normalise(0, 0, m, n, k, A, lda, MIPGEMM_ROW_MAJOR, B, ldb, orderB, C, ldc,
                                       MIPGEMM_ROW_MAJOR, MIPGEMM_OVERWRITE, workspace, workspace_bytes, &checked);
  // (B stands at 7 here as there; what follows it does not)
  if (rc <= -1 && rc >= -9) return rc;
  if (activation < mip::ACT_NONE || activation > mip::ACT_SILU) return -12;
  if (R && (ldr < (n > 1 ? n : 1) || ldr > MIPGEMM_MAX_DIM)) return -14;
  if (rc == -10) return -15;
  if (rc == -11) return -16;
  if (!mip::real_type_ok(c_type)) return -17;
  if (rc == -14) return -18;
  const mip::LinearArgs linear{C, R, ldc, ldr, a_scales, b_scales, bias, activation, c_type};
  return mip::run_gemm(0, 0, 3, 1.0f, m, n, k, A, lda, MIPGEMM_ROW_MAJOR, B, ldb, orderB, C, ldc, MIPGEMM_ROW_MAJOR,
                       MIPGEMM_OVERWRITE, workspace, workspace_bytes, stream, mip::Batch(), nullptr, &linear);
}


// ---- the 4-bit cache ----

static bool head_dim_ok(int64_t d) { return d == 64 || d == 128 || d == 256; }
static bool page_ok(int64_t page) { return page >= 16 && page <= 1024 && (page & (page - 1)) == 0; }
static int log2_of(int64_t page) {
  int n = 0;
  while (((int64_t)1 << n) < page) ++n;
  return n;
}
constexpr int64_t MOST_HEADS = 1024;

size_t mipgemm_kv4_bytes(int64_t pages, int64_t page_tokens, int64_t kv_heads, int64_t head_dim) {
  if (pages < 0 || pages > MIPGEMM_MAX_DIM || !page_ok(page_tokens) || kv_heads < 0 || kv_heads > MOST_HEADS || !head_dim_ok(head_dim))
    return 0;
  return (size_t)pages * (size_t)kv_heads * (size_t)(page_tokens * head_dim / 8 * 9);
}

int mipgemm_qk_norm_rope(int64_t tokens, int64_t q_heads, int64_t kv_heads, int64_t head_dim, int type, const void *Q,
                         int64_t ldq, const void *K, int64_t ldk, const void *V, int64_t ldv, const float *q_weight,
                         const float *k_weight, float eps, const float *cosine, const float *sine, int64_t table_rows,
                         int64_t rot_dim, int style, const int32_t *positions, void *Qo, int64_t ldqo, void *Ko, int64_t ldko,
                         void *cache, size_t cache_bytes, int64_t pages, int64_t page_tokens, const int64_t *slots, void *stream) {
  const bool q = tokens > 0 && q_heads > 0, kv = tokens > 0 && kv_heads > 0;
  const bool keys = kv && (Ko || cache), turned = tokens > 0 && rot_dim > 0 && (q || keys);
  if (tokens < 0 || tokens > MIPGEMM_MAX_DIM) return -1;
  if (q_heads < 0 || q_heads > MOST_HEADS) return -2;
  if (kv_heads < 0 || kv_heads > MOST_HEADS) return -3;
  if (!head_dim_ok(head_dim)) return -4;
  if (!mip::real_type_ok(type)) return -5;
  if (!Q && q) return -6;
  if (ldq < q_heads * head_dim || ldq > MIPGEMM_MAX_DIM) return -7;
  if (!K && keys) return -8;
  if (K && (ldk < kv_heads * head_dim || ldk > MIPGEMM_MAX_DIM)) return -9;
  if (!V && kv && cache) return -10;
  if (V && (ldv < kv_heads * head_dim || ldv > MIPGEMM_MAX_DIM)) return -11;
  if (!(eps >= 0.0f) || eps - eps != 0.0f) return -14;
  if (!cosine && turned) return -15;
  if (!sine && turned) return -16;
  if (table_rows < 0 || table_rows > MIPGEMM_MAX_DIM) return -17;
  if (rot_dim < 0 || rot_dim > head_dim || rot_dim % 2) return -18;
  if (style != mip::ROTATE_STYLE_HALVES && style != mip::ROTATE_STYLE_PAIRS) return -19;
  if (!positions && turned) return -20;
  if (!Qo && q) return -21;
  if (ldqo < q_heads * head_dim || ldqo > MIPGEMM_MAX_DIM) return -22;
  if (Ko && (ldko < kv_heads * head_dim || ldko > MIPGEMM_MAX_DIM)) return -24;
  if (cache && reinterpret_cast<uintptr_t>(cache) % 16) return -25;
  if (cache) {
    if (pages < 0 || pages > MIPGEMM_MAX_DIM) return -27;
    if (!page_ok(page_tokens)) return -28;
    if (cache_bytes < mipgemm_kv4_bytes(pages, page_tokens, kv_heads, head_dim)) return -26;
    if (!slots && kv) return -29;
  }
  if (tokens == 0) return 0;
  mip::RopeArgs P;
  P.Q = Q; P.K = K; P.V = V; P.Qo = Qo; P.Ko = Ko;
  P.ldq = ldq; P.ldk = ldk; P.ldv = ldv; P.ldqo = ldqo; P.ldko = ldko;
  P.q_weight = q_weight; P.k_weight = k_weight; P.cosine = cosine; P.sine = sine;
  P.positions = positions;
  P.slots = slots;
  P.cache = kv_heads > 0 ? static_cast<uint8_t *>(cache) : nullptr;  // (without heads nothing goes there, and slots may be null)
  P.pages = pages; P.table_rows = cosine && rot_dim > 0 ? table_rows : 0; P.token0 = 0;
  P.log_page = cache ? log2_of(page_tokens) : 4;
  P.q_heads = (int)q_heads; P.kv_heads = (int)kv_heads; P.rot = (int)rot_dim; P.style = style; P.blocks = 0;
  P.eps = eps;
  return static_cast<int>(mip::launch_rope(P, tokens, (int)head_dim, type, static_cast<hipStream_t>(stream)));
}

int mipgemm_kv4_read(int64_t tokens, int64_t kv_heads, int64_t head_dim, int type, const void *cache, size_t cache_bytes,
                     int64_t pages, int64_t page_tokens, const int64_t *slots, void *K, int64_t ldk, void *V, int64_t ldv,
                     void *stream) {
  const bool any = tokens > 0 && kv_heads > 0;
  if (tokens < 0 || tokens > MIPGEMM_MAX_DIM) return -1;
  if (kv_heads < 0 || kv_heads > MOST_HEADS) return -2;
  if (!head_dim_ok(head_dim)) return -3;
  if (!mip::real_type_ok(type)) return -4;
  if ((!cache && any && pages > 0) || reinterpret_cast<uintptr_t>(cache) % 16) return -5;
  if (pages < 0 || pages > MIPGEMM_MAX_DIM) return -7;
  if (!page_ok(page_tokens)) return -8;
  if (cache_bytes < mipgemm_kv4_bytes(pages, page_tokens, kv_heads, head_dim)) return -6;
  if (!slots && any) return -9;
  if (K && (ldk < kv_heads * head_dim || ldk > MIPGEMM_MAX_DIM)) return -11;
  if (V && (ldv < kv_heads * head_dim || ldv > MIPGEMM_MAX_DIM)) return -13;
  if (!any || (!K && !V)) return 0;
  const mip::Kv4ReadArgs P{static_cast<const uint8_t *>(cache), slots, K, V, ldk, ldv, pages, 0, log2_of(page_tokens), (int)kv_heads, 0};
  return static_cast<int>(mip::launch_kv4_read(P, tokens, (int)head_dim, type, static_cast<hipStream_t>(stream)));
}

size_t mipgemm_attention_kv4_workspace_size(int64_t requests, int64_t q_heads, int64_t kv_heads, int64_t head_dim,
                                            int64_t max_q, int64_t max_kv) {
  if (requests < 1 || requests > MIPGEMM_MAX_DIM || kv_heads < 1 || kv_heads > MOST_HEADS || q_heads < 1 || q_heads > MOST_HEADS ||
      q_heads % kv_heads || !head_dim_ok(head_dim) || max_q < 1 || max_q > MIPGEMM_MAX_DIM || max_kv < 1 || max_kv > MIPGEMM_MAX_DIM ||
      max_q * q_heads > MIPGEMM_MAX_DIM)
    return 0;
  return mip::attention_scratch(requests, kv_heads, q_heads / kv_heads, (int)head_dim, max_q, max_kv);
}

int mipgemm_attention_kv4(int64_t requests, int64_t q_heads, int64_t kv_heads, int64_t head_dim, int type, const void *Q,
                          int64_t ldq, int64_t q_rows, const int32_t *q_starts, int64_t max_q, const int32_t *kv_lengths,
                          int64_t max_kv, const void *cache, size_t cache_bytes, int64_t pages, int64_t page_tokens,
                          const int32_t *block_table, int64_t table_stride, float scale, void *O, int64_t ldo, void *workspace,
                          size_t workspace_bytes, void *stream) {
  const bool any = requests > 0 && q_rows > 0 && max_q > 0;
  if (requests < 0 || requests > MIPGEMM_MAX_DIM) return -1;
  if (q_heads < 1 || q_heads > MOST_HEADS) return -2;
  if (kv_heads < 1 || kv_heads > MOST_HEADS || q_heads % kv_heads) return -3;
  if (!head_dim_ok(head_dim)) return -4;
  if (type != mip::REAL_BF16 && type != mip::REAL_F16) return -5;
  if (!Q && any) return -6;
  if (ldq < q_heads * head_dim || ldq > MIPGEMM_MAX_DIM) return -7;
  if (q_rows < 0 || q_rows > MIPGEMM_MAX_DIM) return -8;
  if (!q_starts && any) return -9;
  if (max_q < 0 || max_q > (MIPGEMM_MAX_DIM - 4096) / q_heads) return -10;  // (a product could wrap)
  if (!kv_lengths && any) return -11;
  if (max_kv < 0 || max_kv > MIPGEMM_MAX_DIM - 4096) return -12;
  if ((!cache && any && pages > 0) || reinterpret_cast<uintptr_t>(cache) % 16) return -13;
  if (pages < 0 || pages > MIPGEMM_MAX_DIM) return -15;
  if (!page_ok(page_tokens)) return -16;
  if (cache_bytes < mipgemm_kv4_bytes(pages, page_tokens, kv_heads, head_dim)) return -14;
  if (table_stride < 0 || table_stride > MIPGEMM_MAX_DIM) return -18;
  if (!block_table && any && table_stride > 0) return -17;
  if (!(scale > 0.0f) || scale - scale != 0.0f) return -19;
  if (!O && any) return -20;
  if (ldo < q_heads * head_dim || ldo > MIPGEMM_MAX_DIM) return -21;
  if (workspace_bytes > 0 && !workspace) return -22;
  if (!any) return 0;
  mip::AttentionArgs P;
  P.Q = Q; P.O = O;
  P.cache = static_cast<const uint8_t *>(cache);
  P.q_starts = q_starts; P.kv_lengths = kv_lengths; P.block_table = block_table;
  P.partials = nullptr;
  P.ldq = ldq; P.ldo = ldo; P.q_rows = q_rows; P.table_stride = table_stride;
  P.pages = (int)pages; P.log_page = log2_of(page_tokens); P.kv_heads = (int)kv_heads; P.shared = (int)(q_heads / kv_heads);
  P.max_q = (int)max_q;
  if (pages == 0 || table_stride == 0) {  // no page can be named: no key is seen, and the table is not used
    P.max_kv = 0;
    P.block_table = q_starts;
    P.table_stride = 1;
  } else {
    P.max_kv = (int)max_kv;
  }
  const int64_t named = P.table_stride << P.log_page;
  P.named_kv = named < P.max_kv ? (int)named : P.max_kv;
  P.ranges = 1; P.span = 0; P.first = 0;
  P.scale = scale < 2.3e38f ? scale : 2.3e38f;  // (the kernels multiply it by log2 e: not to infinity, which makes NaN of zero)
  return static_cast<int>(mip::launch_attention(P, (int)requests, (int)head_dim, type, workspace, workspace_bytes,
                                                static_cast<hipStream_t>(stream)));
}

}  // extern "C"
