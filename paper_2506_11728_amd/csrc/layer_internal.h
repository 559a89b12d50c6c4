// The operators between the integer products of a layer: launchers.  Not installed.
#pragma once
#include "mip_internal.h"

namespace mip {

hipError_t launch_quantize(int64_t rows, int64_t cols, const void *X, int64_t ldx, int type, const float *weight, float eps,
                           int8_t *Q, int64_t ldq, float *scales, hipStream_t s);

enum RotateStyle { ROTATE_STYLE_HALVES = 0, ROTATE_STYLE_PAIRS = 1 };

struct RopeArgs {
  const void *Q, *K, *V;
  void *Qo, *Ko;  // Ko null: the keys go to the cache alone
  int64_t ldq, ldk, ldv, ldqo, ldko;
  const float *q_weight, *k_weight, *cosine, *sine;  // weights null: no norm
  const int32_t *positions;
  const int64_t *slots;
  uint8_t *cache;  // null: none
  int64_t pages, table_rows, token0;
  int log_page, q_heads, kv_heads, rot, style, blocks;
  float eps;
};
// (token0 and blocks are the launchers' own)
hipError_t launch_rope(const RopeArgs &P, int64_t tokens, int head_dim, int type, hipStream_t s);

struct Kv4ReadArgs {
  const uint8_t *cache;
  const int64_t *slots;
  void *K, *V;  // either null: not read
  int64_t ldk, ldv, pages, token0;
  int log_page, kv_heads, blocks;
};
hipError_t launch_kv4_read(const Kv4ReadArgs &P, int64_t tokens, int head_dim, int type, hipStream_t s);

struct AttentionArgs {
  const void *Q;
  void *O;
  const uint8_t *cache;
  const int32_t *q_starts, *kv_lengths, *block_table;
  float *partials;  // of split keys; null: one range
  int64_t ldq, ldo, q_rows, table_stride;
  int pages, log_page, kv_heads, shared, max_q, max_kv, ranges, span, first;
  int named_kv;  // tokens that a row of the table can name pages for: there is nothing to be seen behind them
  float scale;
};
typedef void (*AttentionKernel)(AttentionArgs);
// The kernel for 256 rows of 64 or 128 channels to a workgroup of 512 threads (8 KB of dynamic LDS to 16 channels).
AttentionKernel attention_wide(int head_dim, int type, int log_page);
// ranges, span, first and partials are the launcher's own; ws: scratch memory, or null.
hipError_t launch_attention(AttentionArgs P, int requests, int head_dim, int type, void *ws, size_t ws_bytes, hipStream_t s);
size_t attention_scratch(int64_t requests, int64_t kv_heads, int64_t shared, int head_dim, int64_t max_q, int64_t max_kv);

}  // namespace mip
