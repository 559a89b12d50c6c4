// Rows of real numbers brought to 8 bits, each with a scale of its own, optionally through an RMS norm:
//     z_j = x_j w_j (w_j = 1 without a norm),  a = max_j |z_j|,  q_j = rint(127 z_j / a),
//     scale = a / 127, times 1 / sqrt(mean_j x_j^2 + eps) with a norm.
// The norm's factor is the same in every z_j and in a, so it never meets q_j: the codes do not depend on
// the order in which the squares are summed.
//
// Bound by memory: x is read once, a byte an element written.  A row stays in the registers of its workgroup
// between the reduction and the rounding where it fits (16384 numbers); longer rows are read a second time,
// through the cache.  A wave to a row up to 1024 columns, four waves up to 4096; up to 16384 sixteen waves
// where there is a workgroup of them at a time for every row (48 rows of 11008: 3.7 us against 6.8 with four), else four.
// 4096 rows of 4096 in bfloat16 with a norm: 14.4 us from memory (50 MB at 3.5 TB/s), 13 resident, 11 without a norm.  21 vector
// instructions to a number are 9 us of issue, and two rounds of workgroups, each of which loads, meets at a barrier and
// stores, do not overlap with it altogether (8192 rows 25 us, 16384 44).  4096 rows of 11008, 64 numbers to a thread and so
// four workgroups to a compute unit: 41 us from memory (3.3 TB/s), 39 resident, 30 without a norm.  A row of 4096: 2.5 us, of
// which some 2 are the launch.
#include "layer_internal.h"
#include "row_codes.h"

namespace mip {

namespace {

struct QuantizeParams {
  const void *X;
  int64_t ldx, rows, cols;
  const float *weight;  // null: no norm
  float eps;
  int8_t *Q;
  int64_t ldq;
  float *scales;
};

// x_j and w_j of eight columns from j on; what lies behind the row is zero.
template <typename T>
__device__ __forceinline__ void load_oct(const QuantizeParams &P, int64_t row, int64_t j, float (&x)[8]) {
  constexpr int TYPE = real_of<T>::type;
  if (j + 8 <= P.cols) {
    load_real8<TYPE>(P.X, row * P.ldx + j, x);
  } else {
#pragma unroll
    for (int e = 0; e < 8; ++e) x[e] = j + e < P.cols ? load_real(P.X, row * P.ldx + j + e, TYPE) : 0.0f;
  }
}
__device__ __forceinline__ void times_weight(const QuantizeParams &P, int64_t j, float (&x)[8]) {
  float w[8];
  if (j + 8 <= P.cols) {
    load_real8<REAL_F32>(P.weight, j, w);
  } else {
#pragma unroll
    for (int e = 0; e < 8; ++e) w[e] = j + e < P.cols ? P.weight[j + e] : 0.0f;
  }
#pragma unroll
  for (int e = 0; e < 8; ++e) x[e] = __fmul_rn(x[e], w[e]);
}

// WAVES to a row, ROWS rows to a workgroup; HELD: eights of columns a thread keeps, 0: none.
// NORM: through an RMS norm, whose weights are there.
template <typename T, int WAVES, int ROWS, int HELD, bool NORM>
__global__ __launch_bounds__(64 * WAVES *ROWS) void quantize_kernel(QuantizeParams P) {
  constexpr int THREADS = 64 * WAVES;
  const int lane = threadIdx.x & 63, wave = threadIdx.x / 64 % WAVES, at = threadIdx.x % THREADS;
  const int64_t row = (int64_t)blockIdx.x * ROWS + threadIdx.x / THREADS;
  const bool here = row < P.rows;
  float x[HELD ? HELD : 1][8];
  float top = 0.0f, squares = 0.0f, none = 0.0f;  // none: NaN where something is no number
  auto take = [&](int64_t j, float (&v)[8]) {
    load_oct<T>(P, row, j, v);
    if (NORM) {
#pragma unroll
      for (int e = 0; e < 8; ++e) squares += v[e] * v[e];
      times_weight(P, j, v);
    }
#pragma unroll
    for (int e = 0; e < 8; ++e) none = __builtin_fmaf(v[e], 0.0f, none);
#pragma unroll
    for (int e = 0; e < 8; e += 2) top = fmaxf(fmaxf(top, fabsf(v[e])), fabsf(v[e + 1]));
  };
  if (HELD) {
#pragma unroll
    for (int u = 0; u < HELD; ++u) {
      const int64_t j = 8 * ((int64_t)u * THREADS + at);
      if (here && j < P.cols) take(j, x[u]);
    }
  } else if (here) {
    for (int64_t j = 8 * at; j < P.cols; j += 8 * THREADS) take(j, x[0]);
  }
  if (none != 0.0f) top = __builtin_nanf("");
  auto larger = [](float a, float b) { return a != a ? a : (b <= a ? a : b); };
#pragma unroll
  for (int d = 1; d < 64; d *= 2) {
    top = larger(top, __shfl_xor(top, d));
    if (NORM) squares += __shfl_xor(squares, d);
  }
  if constexpr (WAVES > 1) {
    __shared__ float both[2][WAVES];
    if (lane == 0) {
      both[0][wave] = top;
      both[1][wave] = squares;
    }
    __syncthreads();
    top = both[0][0];
    squares = both[1][0];
#pragma unroll
    for (int w = 1; w < WAVES; ++w) {
      top = larger(top, both[0][w]);
      squares += both[1][w];
    }
  }
  if (!here) return;
  const bool finite = top < __builtin_inff();  // (false for a NaN)
  if (at == 0) {
    float scale = finite ? __fdiv_rn(top, 127.0f) : __builtin_nanf("");
    if (NORM && top != 0.0f)  // (zero stays zero, whatever eps is)
      scale *= __fdiv_rn(1.0f, __fsqrt_rn(__fdiv_rn(squares, (float)P.cols) + P.eps));
    P.scales[row] = scale;
  }
  const float by = code_range(top);
  const float a = top * by, by_127 = 127.0f * by, r = finite && top > 0.0f ? __fdiv_rn(1.0f, a) : 0.0f;
  auto put = [&](int64_t j, float (&v)[8]) { put_codes(P.Q + row * P.ldq + j, P.cols - j, v, by_127, a, r); };
  if (HELD) {
#pragma unroll
    for (int u = 0; u < HELD; ++u) {
      const int64_t j = 8 * ((int64_t)u * THREADS + at);
      if (j < P.cols) put(j, x[u]);
    }
  } else {
    for (int64_t j = 8 * at; j < P.cols; j += 8 * THREADS) {
      load_oct<T>(P, row, j, x[0]);
      if (NORM) times_weight(P, j, x[0]);
      put(j, x[0]);
    }
  }
  // From 2^-100 to 2^120 of the mean no square has passed float32, and what is lost of small ones is below 2^-40 of it.  Elsewhere
  // the first wave sums them again, in float64, which squares of float32 neither pass nor fall below.
  if (!NORM || wave != 0 || !finite || top == 0.0f) return;
  const float mean = squares * __builtin_amdgcn_rcpf((float)P.cols) + P.eps;
  if (mean >= 0x1p-100f && mean <= 0x1p120f) return;
  double sum = 0.0;
  int first = lane;
  asm volatile("" : "+v"(first));  // (its addresses are not kept over the above)
#pragma unroll 1
  for (int64_t j = first; j < P.cols; j += 64) {
    const double v = load_real(P.X, row * P.ldx + j, real_of<T>::type);
    sum += v * v;
  }
#pragma unroll
  for (int d = 1; d < 64; d *= 2) sum += __shfl_xor(sum, d);
  if (lane == 0) P.scales[row] = (float)((double)top / (127.0 * __builtin_sqrt(sum / (double)P.cols + (double)P.eps)));
}

constexpr int64_t MOST_THREADS = 1024;  // of a workgroup below, which takes a row or more

template <typename T, bool NORM>
hipError_t launch_for(const QuantizeParams &P, hipStream_t s) {
  void (*kernel)(QuantizeParams);
  unsigned threads = 256;
  int64_t rows = 1;
  if (P.cols <= 1024) { kernel = quantize_kernel<T, 1, 4, 2, NORM>; rows = 4; }
  else if (P.cols <= 4096) kernel = quantize_kernel<T, 4, 1, 2, NORM>;
  else if (P.cols > 16384) { kernel = quantize_kernel<T, 16, 1, 0, NORM>; threads = 1024; }
  else if (P.rows <= 2 * compute_units()) { kernel = quantize_kernel<T, 16, 1, 2, NORM>; threads = 1024; }
  else kernel = quantize_kernel<T, 4, 1, 8, NORM>;
  const dim3 grid((unsigned)((P.rows + rows - 1) / rows));
  return launch_with(reinterpret_cast<const void *>(kernel), grid, threads, 0, s, &P);
}

}  // namespace

hipError_t launch_quantize(int64_t rows, int64_t cols, const void *X, int64_t ldx, int type, const float *weight, float eps,
                           int8_t *Q, int64_t ldq, float *scales, hipStream_t s) {
  // (a grid has at most 2^32 - 1 threads a dimension: taller matrices in slabs)
  constexpr int64_t slab = (int64_t)1 << 21;
  static_assert(slab * MOST_THREADS < (int64_t)1 << 32, "a row to a workgroup of the most threads");
  for (int64_t i = 0; i < rows; i += slab) {
    const QuantizeParams P{static_cast<const uint8_t *>(X) + i * ldx * real_bytes(type), ldx,
                           rows - i < slab ? rows - i : slab, cols, weight, eps, Q + i * ldq, ldq, scales + i};
    const hipError_t e = type == REAL_F32    ? (weight ? launch_for<float, true>(P, s) : launch_for<float, false>(P, s))
                         : type == REAL_BF16 ? (weight ? launch_for<__bf16, true>(P, s) : launch_for<__bf16, false>(P, s))
                                             : (weight ? launch_for<_Float16, true>(P, s) : launch_for<_Float16, false>(P, s));
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}

}  // namespace mip
