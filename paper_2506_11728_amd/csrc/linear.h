// Write-back of a linear layer on 8-bit operands: from the int32 sums S of the product to
//     C(i, j) = act( float(S(i, j)) * row_scale(i) * col_scale(j) + bias(j) ) + R(i, j)
// in float32, rounded once to the type of C.  Shared by the MFMA kernels, whose LINEAR forms
// (UNS == LINEAR_OUT) differ from the others in nothing else: the sums are complete before anything
// is converted, in integers, and what the write-back adds to a product is the traffic of R and of
// C, which in 16 bits is half that of int32 sums.  4096 x 11008 x 4096 in bfloat16: 164 us, 170 with SiLU, 192 with GELU (its
// polynomial, with the matrix unit idle), 168 with a residual (213 when what was fetched ahead was converted as it came, and
// so waited for); int32 results 179.
#pragma once
#include "epilogue16.h"
#include "mip_internal.h"
#include "real.h"

namespace mip {

constexpr int LINEAR_OUT = 5;  // the kernels' UNS parameter: both operands signed, this write-back

// The activations fall into three kinds, by how much code they are; the write-back loops are
// instantiated once per kind and entered through a wave-uniform switch.
//   0: max(y, floor), floor 0 or -infinity
//   1: y / (1 + exp(-y (c1 + c3 y^2))): SiLU, and GELU's tanh form, since (1 + tanh u) / 2 = 1 / (1 + exp(-2 u))
//   2: y * erfc(-y / sqrt 2) / 2: GELU
// The argument of the exponential is one rounded product (of two, GELU's), |t| 2^-24 off at most, and so is the exponential,
// relatively: where y is far below zero and the result as small, 20 2^-24 of it at y = -20.  In 16 bits that does not show, in float32
// it is the last few bits of a tail of 1e-8; a second product for what the first one's rounding loses would be five
// instructions more in a write-back that nothing overlaps.
template <int KIND>
struct Activate {
  float c1, c3;  // kind 0: the floor in c1
  __device__ static __forceinline__ Activate of(int act) {
    if (KIND == 0) return {act == ACT_RELU ? 0.0f : -__builtin_inff(), 0.0f};
    const float c = 1.5957691216057308f;  // 2 sqrt(2 / pi)
    if (act == ACT_GELU_TANH) return {c, c * 0.044715f};
    return {1.0f, 0.0f};
  }
  __device__ __forceinline__ float operator()(float y) const {
    if (KIND == 0) return y < c1 ? c1 : y;  // (a NaN stays one)
    if (KIND == 1) {
      const float t = y * (c1 + c3 * y * y);
      // (at the far negative end exp overflows to infinity and the quotient is -0)
      return y * __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(-1.4426950408889634f * t));
    }
    // erfc(z) for z >= 0 within 1.2e-7 of its value: t exp(-z^2 + P(t)), t = 1 / (1 + z / 2), the
    // Chebyshev fit of Press et al., Numerical Recipes, section 6.2
    const float z = fabsf(y) * 0.70710678118654752f;
    const float t = __builtin_amdgcn_rcpf(1.0f + 0.5f * z);
    float p = 0.17087277f;
    p = p * t - 0.82215223f;
    p = p * t + 1.48851587f;
    p = p * t - 1.13520398f;
    p = p * t + 0.27886807f;
    p = p * t - 0.18628806f;
    p = p * t + 0.09678418f;
    p = p * t + 0.37409196f;
    p = p * t + 1.00002368f;
    p = p * t - 1.26551223f;
    const float half = 0.5f * t * __builtin_amdgcn_exp2f(1.4426950408889634f * (p - z * z));  // erfc(z) / 2
    return y * (y < 0.0f ? half : 1.0f - half);
  }
};
__device__ __forceinline__ int activation_kind(int act) { return act == ACT_GELU ? 2 : (act >= ACT_GELU_TANH ? 1 : 0); }

// The same roundings in every kernel: a result does not depend on which of them serves a call.
__device__ __forceinline__ float linear_value(int sum, float row_scale, float col_scale, float bias) {
  return __builtin_fmaf(__fmul_rn((float)sum, row_scale), col_scale, bias);
}

// Scales and biases of a lane's four columns, `count` of which exist.
struct LinearColumns {
  v4f scale, bias;
};
__device__ __forceinline__ LinearColumns linear_columns(const LinearArgs &L, int64_t col, int64_t count) {
  LinearColumns c{{1.0f, 1.0f, 1.0f, 1.0f}, {0.0f, 0.0f, 0.0f, 0.0f}};
  if (count >= 4) {
    if (L.col_scale) c.scale = load_real4(L.col_scale, col, REAL_F32);
    if (L.bias) c.bias = load_real4(L.bias, col, REAL_F32);
    return c;
  }
#pragma unroll
  for (int e = 0; e < 3; ++e) {
    if (e < count && L.col_scale) c.scale[e] = L.col_scale[col + e];
    if (e < count && L.bias) c.bias[e] = L.bias[col + e];
  }
  return c;
}

// Four numbers of R as they lie in memory (in a 16-bit type: in the first two words), and what they are: a number that is
// worked on is waited for, so what is fetched ahead stays as it came.
__device__ __forceinline__ v4w linear_residual(const LinearArgs &L, int64_t row, int64_t col, int64_t count) {
  const int64_t at = row * L.ldr + col;
  v4w r = {0, 0, 0, 0};
  if (L.type == REAL_F32) {
    const uint32_t *from = static_cast<const uint32_t *>(L.R) + at;
    if (count >= 4) return *reinterpret_cast<const v4w *>(from);
#pragma unroll
    for (int e = 0; e < 3; ++e)
      if (e < count) r[e] = from[e];
    return r;
  }
  const uint16_t *from = static_cast<const uint16_t *>(L.R) + at;
  if (count >= 4) {
    const v2w w = *reinterpret_cast<const v2w *>(from);
    return v4w{w[0], w[1], 0, 0};
  }
#pragma unroll
  for (int e = 0; e < 3; ++e)
    if (e < count) r[e / 2] |= (uint32_t)from[e] << (e % 2 * 16);
  return r;
}
__device__ __forceinline__ v4f linear_numbers(v4w r, int type) {
  if (type == REAL_F32) return __builtin_bit_cast(v4f, r);
  const v2w w = {r[0], r[1]};
  return type == REAL_BF16 ? __builtin_convertvector(__builtin_bit_cast(v4b, w), v4f)
                           : __builtin_convertvector(__builtin_bit_cast(v4h, w), v4f);
}

// STREAM: whole cache lines of a large C, which would push the operands of other workgroups out of L2 (as in the
// other write-backs).
template <int KIND, bool STREAM = false>
__device__ __forceinline__ void linear_quad(const LinearArgs &L, const Activate<KIND> act, const LinearColumns &c,
                                            int64_t row, int64_t col, int64_t count, v4i sum, float row_scale, v4w residual) {
  v4f y;
#pragma unroll
  for (int e = 0; e < 4; ++e) y[e] = act(linear_value(sum[e], row_scale, c.scale[e], c.bias[e]));
  if (L.R) y += linear_numbers(residual, L.type);
  if (count >= 4) {
    store_real4<STREAM>(L.C, row * L.ldc + col, L.type, y);
  } else {
#pragma unroll
    for (int e = 0; e < 3; ++e)
      if (e < count) store_real(L.C, row * L.ldc + col + e, L.type, y[e]);
  }
}

// One element, for the kernels that write C element by element.
__device__ __forceinline__ void linear_one(const LinearArgs &L, int64_t row, int64_t col, int sum) {
  float y = linear_value(sum, L.row_scale ? L.row_scale[row] : 1.0f, L.col_scale ? L.col_scale[col] : 1.0f,
                         L.bias ? L.bias[col] : 0.0f);
  switch (activation_kind(L.act)) {
    case 0: y = Activate<0>::of(L.act)(y); break;
    case 1: y = Activate<1>::of(L.act)(y); break;
    default: y = Activate<2>::of(L.act)(y); break;
  }
  if (L.R) y += load_real(L.R, row * L.ldr + col, L.type);
  store_real(L.C, row * L.ldc + col, L.type, y);
}

// What the write-back of PASSES row pieces of four columns, ROWS rows apart, needs from memory: loaded one strip of rows
// ahead, so that its latency hides behind the strip before.
template <int PASSES>
struct LinearStrip {
  v4w residual[PASSES];
  float row_scale[PASSES];
};
template <int PASSES, int ROWS, bool FULL>
__device__ __forceinline__ LinearStrip<PASSES> linear_strip(const LinearArgs &L, int64_t row, int64_t rows, int64_t col, int64_t count) {
  LinearStrip<PASSES> s;
#pragma unroll
  for (int t = 0; t < PASSES; ++t) {
    const bool here = (FULL || t * ROWS < rows) && count > 0;
    s.residual[t] = v4w{0, 0, 0, 0};  // (zeros in every type)
    if (here && L.R) s.residual[t] = linear_residual(L, row + t * ROWS, col, count);
    s.row_scale[t] = here && L.row_scale ? L.row_scale[row + t * ROWS] : 1.0f;
  }
  return s;
}
// The pieces' sums are in LDS at patch + t * ROWS * PITCH.
template <int KIND, int PASSES, int ROWS, int PITCH, bool FULL, bool STREAM>
__device__ __forceinline__ void linear_pieces(const LinearArgs &L, const Activate<KIND> act, const LinearColumns &columns,
                                              const LinearStrip<PASSES> &s, int64_t row, int64_t rows, int64_t col,
                                              int64_t count, const int32_t *patch) {
  v4i sum[PASSES];
#pragma unroll
  for (int t = 0; t < PASSES; ++t) sum[t] = *reinterpret_cast<const v4i *>(patch + t * ROWS * PITCH);
#pragma unroll
  for (int t = 0; t < PASSES; ++t)
    if ((FULL || t * ROWS < rows) && count > 0)
      linear_quad<KIND, STREAM>(L, act, columns, row + t * ROWS, col, count, sum[t], s.row_scale[t], s.residual[t]);
}

// Blocks of v_mfma_i32_16x16x64_i8 (epilogue16.h), sixteen rows at a time through the wave's patch.
// row0, col0: the first element of the sub-tile in C; rows, cols: how much of it lies inside.
template <int FM, int FN, int KIND, bool FULL>
__device__ __forceinline__ void store_linear16_as(const v4i (&acc)[FM][FN], const LinearArgs &L, int64_t row0, int64_t col0,
                                                  int64_t rows, int64_t cols, int lane, int32_t *patch) {
  constexpr int PITCH = Patch16<FN>::PITCH, LANES_PER_ROW = 4 * FN, ROWS = 64 / LANES_PER_ROW, PASSES = 16 / ROWS;
  const bool active = 64 % LANES_PER_ROW == 0 || lane < ROWS * LANES_PER_ROW;
  const int r0 = active ? lane / LANES_PER_ROW : 0, c0 = 4 * (lane % LANES_PER_ROW);
  const int64_t count = !active ? 0 : (FULL ? 4 : cols - c0);
  const LinearColumns columns = linear_columns(L, col0 + c0, count);
  const Activate<KIND> act = Activate<KIND>::of(L.act);
  LinearStrip<PASSES> strip[2];
  auto fetch = [&](int i) { return linear_strip<PASSES, ROWS, FULL>(L, row0 + i * 16 + r0, rows - (i * 16 + r0), col0 + c0, count); };
  strip[0] = fetch(0);
#pragma unroll
  for (int i = 0; i < FM; ++i) {
    if (!FULL && i * 16 >= rows) break;  // wave-uniform
    if (i + 1 < FM) strip[(i + 1) & 1] = fetch(i + 1);
    __builtin_amdgcn_sched_barrier(0);  // (the loads stay up here)
#pragma unroll
    for (int j = 0; j < FN; ++j)
      *reinterpret_cast<v4i *>(patch + (lane & 15) * PITCH + 16 * j + 4 * (lane >> 4)) = acc[i][j];
    // same wave wrote and reads: LDS operations of a wave complete in order
    if (64 % LANES_PER_ROW != 0) asm volatile("" ::: "memory");
    linear_pieces<KIND, PASSES, ROWS, PITCH, FULL, FULL && FN == 8>(L, act, columns, strip[i & 1], row0 + i * 16 + r0, rows - (i * 16 + r0),
                                                   col0 + c0, count, patch + r0 * PITCH + c0);
  }
}

// Blocks of v_mfma_i32_32x32x32_i8 (epilogue.h), one at a time through the wave's STORE_PATCH_BYTES of LDS.
template <int FM, int FN, int KIND, bool FULL>
__device__ __forceinline__ void store_linear32_as(const v16i (&acc)[FM][FN], const LinearArgs &L, int64_t row0, int64_t col0,
                                                  int64_t rows, int64_t cols, int lane, int32_t *patch) {
  const int r0 = lane >> 3, c0 = 4 * (lane & 7);
  const Activate<KIND> act = Activate<KIND>::of(L.act);
#pragma unroll
  for (int j = 0; j < FN; ++j) {
    if (!FULL && j * 32 >= cols) break;  // wave-uniform
    const int64_t count = FULL ? 4 : cols - (j * 32 + c0);
    const LinearColumns columns = linear_columns(L, col0 + j * 32 + c0, count);
    LinearStrip<4> strip[2];
    auto fetch = [&](int i) { return linear_strip<4, 8, FULL>(L, row0 + i * 32 + r0, rows - (i * 32 + r0), col0 + j * 32 + c0, count); };
    strip[0] = fetch(0);
#pragma unroll
    for (int i = 0; i < FM; ++i) {
      if (!FULL && i * 32 >= rows) break;
      if (i + 1 < FM) strip[(i + 1) & 1] = fetch(i + 1);
      __builtin_amdgcn_sched_barrier(0);  // (the loads stay up here)
#pragma unroll
      for (int q = 0; q < 4; ++q)
        *reinterpret_cast<v4i *>(patch + (lane & 31) * 36 + 8 * q + 4 * (lane >> 5)) =
            v4i{acc[i][j][4 * q], acc[i][j][4 * q + 1], acc[i][j][4 * q + 2], acc[i][j][4 * q + 3]};
      linear_pieces<KIND, 4, 8, 36, FULL, false>(L, act, columns, strip[i & 1], row0 + i * 32 + r0, rows - (i * 32 + r0),
                                          col0 + j * 32 + c0, count, patch + r0 * 36 + c0);
    }
  }
}

#define MIP_STORE_LINEAR(NAME, BLOCK)                                                                              \
  template <int FM, int FN, bool FULL>                                                                             \
  __device__ __forceinline__ void NAME(const BLOCK (&acc)[FM][FN], const LinearArgs &L, int64_t row0, int64_t col0, \
                                       int64_t rows, int64_t cols, int lane, int32_t *patch) {                     \
    switch (activation_kind(L.act)) { /* wave-uniform */                                                           \
      case 0: NAME##_as<FM, FN, 0, FULL>(acc, L, row0, col0, rows, cols, lane, patch); break;                       \
      case 1: NAME##_as<FM, FN, 1, FULL>(acc, L, row0, col0, rows, cols, lane, patch); break;                       \
      default: NAME##_as<FM, FN, 2, FULL>(acc, L, row0, col0, rows, cols, lane, patch); break;                      \
    }                                                                                                              \
  }
MIP_STORE_LINEAR(store_linear16, v4i)
MIP_STORE_LINEAR(store_linear32, v16i)
#undef MIP_STORE_LINEAR

}  // namespace mip
