// Write-back of the experts' products from blocks of v_mfma_i32_16x16x64_i8.
#pragma once
#include "epilogue16.h"
#include "experts.h"

namespace mip {

// What is written of a wave's sub-tile, sixteen rows at a time through the wave's patch (store_linear16, with pairs of columns
// where there is a gate and scales by expert).  `scales`: of the sub-tile's rows, in LDS.
template <int FM, int FN, int GATED, int KIND>
__device__ __forceinline__ void store_experts_as(const v4i (&acc)[FM][FN], const ExpertsArgs &X, int e, int64_t row0, int64_t rows,
                                                 int64_t col0, int lane, int32_t *patch, const float *scales) {
  constexpr int PITCH = Patch16<FN>::PITCH;
  constexpr int LANES_PER_ROW = GATED ? 2 * FN : 4 * FN, ROWS = 64 / LANES_PER_ROW, PASSES = 16 / ROWS;
  static_assert(64 % LANES_PER_ROW == 0, "every lane has a piece");
  const int r0 = lane / LANES_PER_ROW, q = lane % LANES_PER_ROW;
  const int c0 = 4 * q;                                       // the piece's first column in C
  const int at = GATED ? 32 * (q / 4) + 4 * (q % 4) : c0;     // and in the patch; its other half is 16 words on
  const int64_t outputs = GATED ? 2 * X.n : X.n, col = col0 + c0, count = X.n - col;
  LinearArgs L{X.C, nullptr, X.ldc, 0, nullptr, X.b_scales ? X.b_scales + e * outputs : nullptr, X.bias ? X.bias + e * outputs : nullptr, X.act, X.type};
  const LinearColumns gate = linear_columns(L, col, count);
  const LinearColumns up = GATED ? linear_columns(L, X.n + col, count) : gate;
  const Activate<KIND> act = Activate<KIND>::of(X.act);
#pragma unroll
  for (int i = 0; i < FM; ++i) {
    if (i * 16 >= rows) break;  // wave-uniform
#pragma unroll
    for (int j = 0; j < FN; ++j)
      *reinterpret_cast<v4i *>(patch + (lane & 15) * PITCH + 16 * j + 4 * (lane >> 4)) = acc[i][j];
    // same wave wrote and reads: LDS operations of a wave complete in order
#pragma unroll
    for (int t = 0; t < PASSES; ++t) {
      const int r = i * 16 + t * ROWS + r0;
      const int32_t *sums = patch + (t * ROWS + r0) * PITCH + at;
      const v4i s = *reinterpret_cast<const v4i *>(sums);
      const float scale = scales[r];
      v4f y;
#pragma unroll
      for (int k = 0; k < 4; ++k) y[k] = act(linear_value(s[k], scale, gate.scale[k], gate.bias[k]));
      if (GATED) {
        const v4i u = *reinterpret_cast<const v4i *>(sums + 16);
#pragma unroll
        for (int k = 0; k < 4; ++k) y[k] *= linear_value(u[k], scale, up.scale[k], up.bias[k]);
      }
      if (r >= rows || count <= 0) continue;
      if (count >= 4) {
        store_real4<false>(X.C, (row0 + r) * X.ldc + col, X.type, y);
      } else {
#pragma unroll
        for (int k = 0; k < 3; ++k)
          if (k < count) store_real(X.C, (row0 + r) * X.ldc + col + k, X.type, y[k]);
      }
    }
    asm volatile("" ::: "memory");  // (the next rows' sums go where these were)
  }
}

template <int FM, int FN, int GATED>
__device__ __forceinline__ void store_experts(const v4i (&acc)[FM][FN], const ExpertsArgs &X, int e, int64_t row0, int64_t rows, int64_t col0,
                                              int lane, int32_t *patch, const float *scales) {
  switch (activation_kind(X.act)) {  // wave-uniform
    case 0: store_experts_as<FM, FN, GATED, 0>(acc, X, e, row0, rows, col0, lane, patch, scales); break;
    case 1: store_experts_as<FM, FN, GATED, 1>(acc, X, e, row0, rows, col0, lane, patch, scales); break;
    default: store_experts_as<FM, FN, GATED, 2>(acc, X, e, row0, rows, col0, lane, patch, scales); break;
  }
}

}  // namespace mip
