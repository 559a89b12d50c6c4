// C-ABI entry points of a mixture of experts: argument checks.  Host only.
#include "api_internal.h"
#include "layer_internal.h"
#include "real.h"

extern "C" {

size_t mipgemm_route_workspace_size(int64_t tokens, int64_t experts, int64_t top) {
  if (tokens < 0 || tokens > (int64_t)1 << 26 || experts < 1 || experts > mip::MOST_EXPERTS || top < 1 || top > mip::MOST_CHOSEN ||
      top > experts || tokens * top > MIPGEMM_MAX_DIM)
    return 0;
  return mip::route_scratch(tokens, experts, top);
}

int mipgemm_route(int64_t tokens, int64_t experts, int64_t top, const void *logits, int64_t ldl, int type, const float *bias,
                  int scoring, int64_t groups, int64_t top_groups, int64_t group_best, int normalise, float scale, int32_t *ids,
                  float *weights, int32_t *starts, int32_t *order, int32_t *places, void *workspace, size_t workspace_bytes,
                  void *stream) {
  if (tokens < 0 || tokens > (int64_t)1 << 26) return -1;
  if (experts < 1 || experts > mip::MOST_EXPERTS) return -2;
  if (top < 1 || top > mip::MOST_CHOSEN || top > experts) return -3;
  if (tokens * top > MIPGEMM_MAX_DIM) return -1;
  if (!logits && tokens > 0) return -4;
  if (ldl < experts || ldl > MIPGEMM_MAX_DIM) return -5;
  if (!mip::real_type_ok(type)) return -6;
  if (scoring != MIPGEMM_SOFTMAX && scoring != MIPGEMM_SIGMOID) return -8;
  if (groups < 1 || groups > mip::MOST_GROUPS || experts % groups) return -9;
  if (top_groups < 1 || top_groups > groups) return -10;
  if (group_best < 1 || group_best > 2 || group_best > experts / groups) return -11;
  if (top > top_groups * (experts / groups)) return -3;
  if (scale - scale != 0.0f) return -13;
  if (!ids && tokens > 0) return -14;
  if (!weights && tokens > 0) return -15;
  if (workspace_bytes > 0 && !workspace) return -19;
  if (starts && reinterpret_cast<uintptr_t>(workspace) % 16) return -19;
  if (starts && workspace_bytes < mip::route_scratch(tokens, experts, top)) return -20;
  if (tokens == 0 && !starts) return 0;
  mip::RouteArgs P;
  P.logits = logits; P.bias = bias;
  P.ids = ids; P.weights = weights;
  P.starts = starts; P.order = order; P.places = places;
  P.counts = P.ranks = nullptr;
  P.ldl = ldl; P.tokens = tokens;
  P.experts = (int)experts; P.top = (int)top; P.groups = (int)groups; P.top_groups = (int)top_groups; P.best = (int)group_best;
  P.normalise = normalise != 0; P.sigmoid = scoring == MIPGEMM_SIGMOID;
  P.each = mip::divisor(experts / groups, mip::MOST_EXPERTS);
  P.span = 16;
  P.scale = scale;
  return static_cast<int>(mip::launch_route(P, type, workspace, static_cast<hipStream_t>(stream)));
}

int mipgemm_s8s8_experts(int64_t rows, int64_t experts, int64_t n, int64_t k, const int8_t *A, int64_t lda, int64_t a_rows,
                         const float *a_scales, const int32_t *starts, const int32_t *order, int64_t top, const int8_t *B,
                         int64_t ldb, int64_t strideB, const float *b_scales, const float *bias, int activation, int gated,
                         void *C, int64_t ldc, int c_type, void *stream) {
  const bool any = rows > 0 && n > 0;
  if (rows < 0 || rows > MIPGEMM_MAX_DIM) return -1;
  if (experts < 1 || experts > mip::MOST_EXPERTS) return -2;
  if (n < 0 || n > (gated ? MIPGEMM_MAX_DIM / 2 : MIPGEMM_MAX_DIM)) return -3;
  if (k < 0 || k > MIPGEMM_MAX_DIM) return -4;
  if (!A && any && k > 0) return -5;
  if (lda < (k > 1 ? k : 1) || lda > MIPGEMM_MAX_DIM) return -6;
  if (a_rows < (any ? (order ? 1 : rows) : 0) || a_rows > MIPGEMM_MAX_DIM) return -7;
  if (!starts && any) return -9;
  if (top < 1 || top > MIPGEMM_MAX_DIM) return -11;
  if (!B && any && k > 0) return -12;
  if (ldb < (k > 1 ? k : 1) || ldb > MIPGEMM_MAX_DIM) return -13;
  const int64_t outputs = gated ? 2 * n : n;
  if (experts > 1 && (strideB < outputs * ldb || strideB > (int64_t)1 << 52)) return -14;
  if (activation < mip::ACT_NONE || activation > mip::ACT_SILU) return -17;
  if (!C && any) return -19;
  if (ldc < (n > 1 ? n : 1) || ldc > MIPGEMM_MAX_DIM) return -20;
  if (!mip::real_type_ok(c_type)) return -21;
  if (!any) return 0;
  mip::ExpertsArgs P;
  P.A = reinterpret_cast<const uint8_t *>(A); P.B = reinterpret_cast<const uint8_t *>(B);
  P.a_scales = a_scales; P.b_scales = b_scales; P.bias = bias;
  P.starts = starts; P.order = order; P.C = C;
  P.lda = lda; P.ldb = ldb; P.strideB = experts > 1 ? strideB : 0; P.ldc = ldc;
  P.a_rows = a_rows; P.rows = rows; P.n = n; P.k = k;
  P.experts = (int)experts; P.act = activation; P.gated = gated != 0; P.type = c_type;
  P.top = mip::divisor(top, MIPGEMM_MAX_DIM);
  return static_cast<int>(mip::launch_experts(P, static_cast<hipStream_t>(stream)));
}

static bool norm_ok(int norm) { return norm >= mip::ROW_NORM_NONE && norm <= mip::ROW_NORM_LAYER; }

int mipgemm_join_rows(int64_t rows, int64_t cols, int64_t parts, int type, const void *X, int64_t ldx, int64_t x_rows,
                      const int32_t *places, const float *weights, int post_norm, const float *post_weight,
                      const float *post_bias, const void *gate, int64_t ldg, int64_t gate_rows, float scale, const void *R,
                      int64_t ldr, void *H, int64_t ldh, int norm, const float *norm_weight, const float *norm_bias, float eps,
                      void *N, int64_t ldn, int8_t *Q, int64_t ldq, float *scales, void *stream) {
  const int64_t least = cols > 1 ? cols : 1;
  if (rows < 0 || rows > MIPGEMM_MAX_DIM) return -1;
  if (cols < 0 || cols > 16384) return -2;
  if (parts < 1 || parts > 1024) return -3;
  if (!mip::real_type_ok(type)) return -4;
  if (x_rows < (places ? 0 : rows * parts) || x_rows > MIPGEMM_MAX_DIM) return -7;
  if (!X && rows > 0 && cols > 0 && x_rows > 0) return -5;
  if (ldx < least || ldx > MIPGEMM_MAX_DIM) return -6;
  if (!norm_ok(post_norm)) return -10;
  if (gate && (ldg < least || ldg > MIPGEMM_MAX_DIM)) return -14;
  if (gate && (gate_rows < 1 || gate_rows > MIPGEMM_MAX_DIM)) return -15;
  if (scale - scale != 0.0f) return -16;
  if (R && (ldr < least || ldr > MIPGEMM_MAX_DIM)) return -18;
  if (H && (ldh < least || ldh > MIPGEMM_MAX_DIM)) return -20;
  if (H && H == R && ldh != ldr && rows > 1) return -20;
  if (!norm_ok(norm)) return -21;
  if (!(eps >= 0.0f) || eps - eps != 0.0f) return -24;
  if (N && (ldn < least || ldn > MIPGEMM_MAX_DIM)) return -26;
  if (!Q && scales) return -27;
  if (Q && (ldq < least || ldq > MIPGEMM_MAX_DIM)) return -28;
  if (Q && !scales && rows > 0) return -29;
  if (rows == 0 || (!H && !N && !Q)) return 0;
  mip::JoinArgs P;
  P.X = X; P.gate = gate; P.R = R; P.H = H; P.N = N; P.Q = Q; P.scales = scales;
  P.places = places; P.weights = weights;
  P.post_weight = post_norm ? post_weight : nullptr; P.post_bias = post_norm ? post_bias : nullptr;
  P.norm_weight = norm ? norm_weight : nullptr; P.norm_bias = norm ? norm_bias : nullptr;
  P.rows = rows; P.row0 = 0; P.ldx = ldx; P.x_rows = x_rows; P.ldg = ldg; P.gate_rows = gate ? gate_rows : 1;
  P.ldr = ldr; P.ldh = ldh; P.ldn = ldn; P.ldq = ldq;
  P.cols = (int)cols; P.parts = (int)parts; P.post_norm = post_norm; P.norm = norm;
  P.scale = scale; P.eps = eps;
  return static_cast<int>(mip::launch_join(P, type, static_cast<hipStream_t>(stream)));
}

}  // extern "C"
