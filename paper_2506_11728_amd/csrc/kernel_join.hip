// The end of a block and the norm in front of the next, row by row:
//     y = sum_j w_j X(place_j),  u = norm(y),  H = R + scale gate u,  z = norm(H),  N = z,  Q = rint(127 z / max |z|).
// A row stays in the registers of its workgroup throughout: X, R and the gate are read once and H, N and Q written once, so
// memory bounds it; the norms' weights, the same for every row, come from the caches.  8192 rows of 4096 in bfloat16 between two RMS norms,
// gated: 71 us (3.8 TB/s; vector instructions issue for 43 of them; into codes in place of values 82 and 58; 103 with residual and gate loaded behind
// the first norm, elements masked one by one and sums by shuffles), 8192 rows of eight parts of 2048 79 us (4.7 TB/s); one row of eight parts of 4096
// 6 us, of one part 5.
//
// A mean is subtracted in two steps: the sum of what is left after the first is taken along with the sum of squares, so
// that numbers far from zero keep their differences.  Sums of squares that float32 does not hold are taken again in
// float64, from the registers.
#include "layer_internal.h"
#include "row_codes.h"
#include "wave.h"

namespace mip {

namespace {

struct TwoSums {
  float a, b;
};

// Sums over the threads of a row, in the same order every time.  `room`: two words to a wave, of this call's own, so that one barrier is
// enough.
template <int WAVES>
__device__ __forceinline__ TwoSums row_sums(TwoSums s, bool both, float (*room)[2], int wave, int lane) {
  if (both) s.a = wave_sum(s.a);
  s.b = wave_sum(s.b);
  if constexpr (WAVES > 1) {
    if (lane == 0) {
      room[wave][0] = s.a;
      room[wave][1] = s.b;
    }
    __syncthreads();
    s = {0.0f, 0.0f};
#pragma unroll
    for (int w = 0; w < WAVES; ++w) {
      s.a += room[w][0];
      s.b += room[w][1];
    }
  }
  return s;
}
template <int WAVES>
__device__ __forceinline__ double row_sum(double s, double *room, int wave, int lane) {
#pragma unroll
  for (int d = 1; d < 64; d *= 2) s += __shfl_xor(s, d);
  if constexpr (WAVES > 1) {
    __syncthreads();  // (from one call to the next)
    if (lane == 0) room[wave] = s;
    __syncthreads();
    s = 0.0;
#pragma unroll
    for (int w = 0; w < WAVES; ++w) s += room[w];
  }
  return s;
}

template <typename T>
__device__ __forceinline__ void load_part(const void *p, int64_t at, int64_t count, float (&v)[8]) {
  constexpr int TYPE = real_of<T>::type;
  if (count >= 8) {
    load_real8<TYPE>(p, at, v);
  } else {
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = e < count ? load_real(p, at + e, TYPE) : 0.0f;
  }
}
template <typename T>
__device__ __forceinline__ void store_part(void *p, int64_t at, int64_t count, const float (&v)[8]) {
  constexpr int TYPE = real_of<T>::type;
  if (count >= 8) {
    store_real8<TYPE>(p, at, v);
  } else {
#pragma unroll
    for (int e = 0; e < 7; ++e)
      if (e < count) store_real(p, at + e, TYPE, v[e]);
  }
}

template <typename T>
struct eight_of {
  typedef T type __attribute__((ext_vector_type(8)));
};

// WAVES to a row, ROWS rows to a workgroup; HELD: eights of columns a thread keeps.  WHOLE: the columns are a multiple of eight, so that
// a thread's eights are there or are not; what lies behind the row is zero throughout.
template <typename T, int WAVES, int ROWS, int HELD, bool WHOLE>
__global__ __launch_bounds__(64 * WAVES *ROWS) void join_kernel(JoinArgs P) {
  constexpr int THREADS = 64 * WAVES;
  typedef typename eight_of<T>::type Eight;
  typedef float v8f __attribute__((ext_vector_type(8)));
  __shared__ float sums[4][WAVES * ROWS][2];
  __shared__ double wide_sums[WAVES * ROWS];
  const int lane = threadIdx.x & 63, wave = threadIdx.x / 64 % WAVES, at = threadIdx.x % THREADS;
  const int group = __builtin_amdgcn_readfirstlane(threadIdx.x / THREADS);
  const int64_t row = P.row0 + (int64_t)blockIdx.x * ROWS + group;
  if (row >= P.rows) return;  // (ROWS > 1: a wave to a row, nothing to wait for)
  float (*room[4])[2] = {&sums[0][group * WAVES], &sums[1][group * WAVES], &sums[2][group * WAVES], &sums[3][group * WAVES]};
  double *wide_room = &wide_sums[group * WAVES];
  auto column = [&](int u) { return 8 * (u * THREADS + at); };
  auto there = [&](int c, int e) { return WHOLE || c + e < P.cols; };  // where c is
  // eight numbers as they lie in memory: what is sent for ahead is not worked on, and so not waited for
  auto raw = [&](const void *p, int64_t from, int c) -> Eight {
    Eight x = {};
    if (c >= P.cols) return x;
    const T *q = static_cast<const T *>(p) + from + c;
    if (WHOLE || c + 8 <= P.cols) return reinterpret_cast<const real_quad<Eight> *>(q)->v;
#pragma unroll
    for (int e = 0; e < 8; ++e)
      if (c + e < P.cols) x[e] = q[e];
    return x;
  };
  const float columns = (float)(P.cols > 0 ? P.cols : 1);

  Eight residual[HELD], gates[HELD];
  const int64_t gate_row = P.gate ? row / P.gate_rows : 0;
  auto ahead = [&]() {
#pragma unroll
    for (int u = 0; u < HELD; ++u) {
      if (P.R) residual[u] = raw(P.R, row * P.ldr, column(u));
      if (P.gate) gates[u] = raw(P.gate, gate_row * P.ldg, column(u));
    }
  };
  float v[HELD][8];
#pragma unroll
  for (int u = 0; u < HELD; ++u)
#pragma unroll
    for (int e = 0; e < 8; ++e) v[u][e] = 0.0f;
  auto add = [&](const Eight (&x)[HELD], float w) {
#pragma unroll
    for (int u = 0; u < HELD; ++u) {
      if (column(u) >= P.cols) continue;
      const v8f f = __builtin_convertvector(x[u], v8f);
#pragma unroll
      for (int e = 0; e < 8; ++e) v[u][e] = there(column(u), e) ? __builtin_fmaf(w, f[e], v[u][e]) : 0.0f;
    }
  };
  // Up to 64 parts at a time: their places and weights by the lanes in one load each, their rows four at a time.
  for (int j0 = 0; j0 < P.parts; j0 += 64) {
    const int here = P.parts - j0 < 64 ? P.parts - j0 : 64;
    const int64_t j = row * P.parts + j0 + (lane < here ? lane : 0);
    const int places = P.places ? P.places[j] : 0;
    const float weights = P.weights ? P.weights[j] : 1.0f;
    if (j0 == 0) ahead();
    for (int i = 0; i < here; i += 4) {
      Eight x[4][HELD];
      float w[4];
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        w[k] = 0.0f;
        if (i + k >= here) continue;
        const int64_t place = P.places ? __builtin_amdgcn_readlane(places, i + k) : row * P.parts + j0 + i + k;
        w[k] = __int_as_float(__builtin_amdgcn_readlane(__float_as_int(weights), i + k));
        const bool has = place >= 0 && place < P.x_rows;
#pragma unroll
        for (int u = 0; u < HELD; ++u) x[k][u] = raw(P.X, has ? place * P.ldx : 0, has ? column(u) : P.cols);
      }
#pragma unroll
      for (int k = 0; k < 4; ++k)
        if (i + k < here) add(x[k], w[k]);
    }
  }

  // v normed: the differences from the mean in v, and what they are to be multiplied by (`wide`: they are multiplied already, in float64)
  struct Factor {
    float by;
    bool wide;
    double whole;
  };
  auto norm = [&](int kind, float (*room0)[2], float (*room1)[2]) -> Factor {
    const bool layer = kind == ROW_NORM_LAYER;
    float mean = 0.0f;
    TwoSums s{0.0f, 0.0f};
    if (layer) {
#pragma unroll
      for (int u = 0; u < HELD; ++u)
#pragma unroll
        for (int e = 0; e < 8; ++e) s.b += v[u][e];
      mean = __fdiv_rn(row_sums<WAVES>(s, false, room0, wave, lane).b, columns);
      s.b = 0.0f;
#pragma unroll
      for (int u = 0; u < HELD; ++u) {
        if (column(u) >= P.cols) continue;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          const float d = there(column(u), e) ? v[u][e] - mean : 0.0f;
          s.a += d;
          s.b = __builtin_fmaf(d, d, s.b);
        }
      }
    } else {
#pragma unroll
      for (int u = 0; u < HELD; ++u)
#pragma unroll
        for (int e = 0; e < 8; ++e) s.b = __builtin_fmaf(v[u][e], v[u][e], s.b);
    }
    s = row_sums<WAVES>(s, layer, room1, wave, lane);
    const float rest = layer ? __fdiv_rn(s.a, columns) : 0.0f;
    const float square = __fdiv_rn(s.b, columns) - rest * rest + P.eps;
    // (the same in the whole row; a deviation of a thousandth of the mean is left with too few bits)
    if (square >= 0x1p-100f && square <= 0x1p120f && square >= 0x1p-20f * mean * mean) {
      if (layer) {
#pragma unroll
        for (int u = 0; u < HELD; ++u)
#pragma unroll
          for (int e = 0; e < 8; ++e) v[u][e] = (v[u][e] - mean) - rest;
      }
      return {__fdiv_rn(1.0f, __fsqrt_rn(square)), false, 0.0};
    }
    double m = 0.0, sum = 0.0;
    if (layer) {
#pragma unroll
      for (int u = 0; u < HELD; ++u)
#pragma unroll
        for (int e = 0; e < 8; ++e) sum += v[u][e];
      m = row_sum<WAVES>(sum, wide_room, wave, lane) / (double)P.cols;
      sum = 0.0;
    }
#pragma unroll
    for (int u = 0; u < HELD; ++u)
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const double d = column(u) + e < P.cols ? (double)v[u][e] - m : 0.0;
        sum += d * d;
      }
    sum = row_sum<WAVES>(sum, wide_room, wave, lane);
    // (zeros stay zeros, whatever eps is)
    const double by = sum == 0.0 ? 0.0 : 1.0 / __builtin_sqrt(sum / (double)P.cols + (double)P.eps);
#pragma unroll
    for (int u = 0; u < HELD; ++u)
#pragma unroll
      for (int e = 0; e < 8; ++e) v[u][e] = (float)(((double)v[u][e] - m) * by);
    return {1.0f, true, by};
  };
  auto weigh = [&](const float *weight, const float *bias, float by) {
#pragma unroll
    for (int u = 0; u < HELD; ++u) {
      const int c = column(u);
      if (c >= P.cols) {  // (a mean has been taken off here too)
#pragma unroll
        for (int e = 0; e < 8; ++e) v[u][e] = 0.0f;
        continue;
      }
      float w[8], b[8];
      if (weight) load_part<float>(weight, c, P.cols - c, w);
      if (bias) load_part<float>(bias, c, P.cols - c, b);
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        float x = v[u][e] * by;
        if (weight) x *= w[e];
        if (bias) x += b[e];
        v[u][e] = there(c, e) ? x : 0.0f;
      }
    }
  };
  if (P.post_norm) {
    const Factor f = norm(P.post_norm, room[0], room[1]);
    weigh(P.post_weight, P.post_bias, f.by);
  }

#pragma unroll
  for (int u = 0; u < HELD; ++u) {
    const int c = column(u);
    if (c >= P.cols) continue;
    if (P.gate) {
      const v8f g = __builtin_convertvector(gates[u], v8f);
#pragma unroll
      for (int e = 0; e < 8; ++e) v[u][e] *= g[e];
    }
#pragma unroll
    for (int e = 0; e < 8; ++e) v[u][e] *= P.scale;
    if (P.R) {
      const v8f r = __builtin_convertvector(residual[u], v8f);
#pragma unroll
      for (int e = 0; e < 8; ++e) v[u][e] += r[e];
    }
#pragma unroll
    for (int e = 0; e < 8; ++e) v[u][e] = there(c, e) ? (float)(T)v[u][e] : 0.0f;
    if (P.H) store_part<T>(P.H, row * P.ldh + c, P.cols - c, v[u]);
  }
  if (!P.N && !P.Q) return;

  // Codes behind an RMS norm without a bias are those of H and the weights, and the norm's factor is in the scale alone: as
  // in rows that are brought to 8 bits by themselves.
  const bool apart = P.Q && P.norm == ROW_NORM_RMS && !P.norm_bias;
  float held[HELD][8];
  if (apart) {
#pragma unroll
    for (int u = 0; u < HELD; ++u)
#pragma unroll
      for (int e = 0; e < 8; ++e) held[u][e] = v[u][e];
  }
  Factor f{1.0f, false, 0.0};
  if (P.norm) {
    f = norm(P.norm, room[2], room[3]);
    weigh(P.norm_weight, P.norm_bias, f.by);
  }
  if (P.N) {
#pragma unroll
    for (int u = 0; u < HELD; ++u) {
      const int c = column(u);
      if (c < P.cols) store_part<T>(P.N, row * P.ldn + c, P.cols - c, v[u]);
    }
  }
  if (!P.Q) return;
  if (apart) {
#pragma unroll
    for (int u = 0; u < HELD; ++u) {
      const int c = column(u);
      if (c >= P.cols) continue;
      float w[8];
      if (P.norm_weight) load_part<float>(P.norm_weight, c, P.cols - c, w);
#pragma unroll
      for (int e = 0; e < 8; ++e) v[u][e] = P.norm_weight ? __fmul_rn(held[u][e], w[e]) : held[u][e];
    }
  }
  float top = 0.0f, none = 0.0f;  // none: NaN where something is no number
#pragma unroll
  for (int u = 0; u < HELD; ++u)
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const float z = there(column(u), e) ? v[u][e] : 0.0f;
      none = __builtin_fmaf(z, 0.0f, none);
      top = __builtin_fmaxf(top, __builtin_fabsf(z));
    }
  top = wave_most(top);
  if (__ballot(none != 0.0f)) top = __builtin_nanf("");
  if constexpr (WAVES > 1) {
    auto larger = [](float a, float b) { return a != a ? a : (b <= a ? a : b); };
    if (lane == 0) room[0][wave][0] = top;  // (every wave is behind the barrier of a later sum, or none was taken)
    __syncthreads();
    top = room[0][0][0];
#pragma unroll
    for (int w = 1; w < WAVES; ++w) top = larger(top, room[0][w][0]);
  }
  const bool finite = top < __builtin_inff();  // (false for a NaN)
  const float by = code_range(top), a = top * by, by_127 = 127.0f * by, r = finite && top > 0.0f ? __fdiv_rn(1.0f, a) : 0.0f;
#pragma unroll
  for (int u = 0; u < HELD; ++u) {
    const int c = column(u);
    if (c < P.cols) put_codes(P.Q + row * P.ldq + c, P.cols - c, v[u], by_127, a, r);
  }
  if (at == 0) {
    float scale = finite ? __fdiv_rn(top, 127.0f) : __builtin_nanf("");
    // (a 127th of the smallest numbers has few bits left, so what goes through float64 does so from the largest on)
    if (apart && finite && top != 0.0f) scale = f.wide ? (float)((double)top * f.whole / 127.0) : scale * f.by;
    P.scales[row] = scale;
  }
}

template <typename T, bool WHOLE>
hipError_t launch_for(const JoinArgs &P, hipStream_t s) {
  void (*kernel)(JoinArgs);
  unsigned threads = 256;
  int64_t rows = 1;
  // (few rows: as many waves to each as it can use)
  const bool few = P.rows - P.row0 <= 2 * compute_units();
  if (P.cols <= 512) { kernel = join_kernel<T, 1, 4, 1, WHOLE>; rows = 4; }
  else if (P.cols <= 1024 && !few) { kernel = join_kernel<T, 1, 4, 2, WHOLE>; rows = 4; }
  else if (P.cols <= 2048) kernel = join_kernel<T, 4, 1, 1, WHOLE>;
  else if (P.cols <= 4096 && !few) kernel = join_kernel<T, 4, 1, 2, WHOLE>;
  else if (P.cols <= 4096) { kernel = join_kernel<T, 8, 1, 1, WHOLE>; threads = 512; }
  else if (P.cols <= 8192 && !few) { kernel = join_kernel<T, 8, 1, 2, WHOLE>; threads = 512; }
  else if (P.cols <= 8192) { kernel = join_kernel<T, 16, 1, 1, WHOLE>; threads = 1024; }
  else { kernel = join_kernel<T, 16, 1, 2, WHOLE>; threads = 1024; }
  return launch_with(reinterpret_cast<const void *>(kernel), dim3((unsigned)((P.rows - P.row0 + rows - 1) / rows)), threads, 0, s, &P);
}

}  // namespace

hipError_t launch_join(JoinArgs P, int type, hipStream_t s) {
  // (a grid has at most 2^32 - 1 threads a dimension: taller matrices in slabs)
  constexpr int64_t slab = (int64_t)1 << 21;
  const int64_t rows = P.rows;
  for (int64_t i = 0; i < rows; i += slab) {
    P.row0 = i;
    P.rows = rows - i < slab ? rows : i + slab;
    const bool whole = P.cols % 8 == 0;
    const hipError_t e = type == REAL_F32    ? (whole ? launch_for<float, true>(P, s) : launch_for<float, false>(P, s))
                         : type == REAL_BF16 ? (whole ? launch_for<__bf16, true>(P, s) : launch_for<__bf16, false>(P, s))
                                             : (whole ? launch_for<_Float16, true>(P, s) : launch_for<_Float16, false>(P, s));
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}

}  // namespace mip
