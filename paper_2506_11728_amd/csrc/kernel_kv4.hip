// Heads of queries, keys and values between the projections of a layer and its attention: RMS norm of each
// head of queries and keys, their rotation by position, and keys and values written to the 4-bit cache; and
// rows of that cache read back.
//
// Bound by memory (every number is read once and written once); one launch, so that nothing between the
// projection and the cache goes to memory.  d / 8 lanes to a head, eight channels to a lane: a wave takes 8, 4 or
// 2 heads.  Queries are worked out in float32.  Keys and values go through float64 between their load and their
// codes: a code is a rounding to one of sixteen levels, and with the norm's sum, the rotation and the group's step at 53
// bits it is the code of the exact key, whichever order the squares are summed in.
#include "kv4.h"
#include "layer_internal.h"

namespace mip {

namespace {

template <typename F>
__device__ __forceinline__ F inverse_root(F x) {
  if constexpr (sizeof(F) == 8) return 1.0 / __builtin_sqrt(x);
  else return __fdiv_rn(1.0f, __fsqrt_rn(x));
}

// Where a slot's token lies: the head's part of its page, and the token's place in it.
struct Place {
  uint8_t *part;
  int token;
};
template <int D>
__device__ __forceinline__ Place place_of(uint8_t *cache, int64_t slot, int log_page, int kv_heads, int head) {
  const int64_t block = ((int64_t)D / 8 * 9) << log_page;
  return {cache + ((slot >> log_page) * kv_heads + head) * block, (int)(slot & ((1 << log_page) - 1))};
}

template <int D>
__device__ __forceinline__ void put_in_cache(const RopeArgs &P, int64_t token, int head, int lane, bool value,
                                             const double (&x)[8]) {
  uint32_t pair;
  const uint32_t word = kv4_encode(x, &pair);
  const int64_t slot = P.slots[token];
  if (slot < 0 || slot >= P.pages << P.log_page) return;
  const Kv4Layout L(1 << P.log_page, D);
  const Place at = place_of<D>(P.cache, slot, P.log_page, P.kv_heads, head);
  uint8_t *codes = at.part + (value ? L.values + 16 * ((at.token >> 2) * (D / 8) + lane) + 4 * (at.token & 3)
                                    : at.token * (D / 2) + 4 * lane);
  *reinterpret_cast<uint32_t *>(codes) = word;
  if ((lane & 3) == 0)
    *reinterpret_cast<uint16_t *>(at.part + (value ? L.value_pairs : L.key_pairs) +
                                  2 * (((lane >> 2) << P.log_page) + at.token)) = (uint16_t)pair;
}

// Norm and rotation of the head whose channels 8 * lane .. + 7 are x; `row`: D numbers of LDS of its own.
template <int D, typename F>
__device__ __forceinline__ void norm_and_rotate(const RopeArgs &P, const float *weight, int64_t token, int lane, F (&x)[8], F *row) {
  constexpr int LANES = D / 8;
  const int c0 = 8 * lane;
  if (weight) {
    F sum = 0;
#pragma unroll
    for (int e = 0; e < 8; ++e) sum += x[e] * x[e];
#pragma unroll
    for (int d = 1; d < LANES; d *= 2) sum += __shfl_xor(sum, d);
    const F root = inverse_root(sum / (F)D + (F)P.eps);
#pragma unroll
    for (int e = 0; e < 8; ++e) x[e] = x[e] * root * (F)weight[c0 + e];
  }
  if (P.rot == 0) return;
  const int64_t position = P.positions[token];
  const bool known = position >= 0 && position < P.table_rows;
  const int half = P.rot / 2;
  const float *cosine = P.cosine + (known ? position : 0) * half, *sine = P.sine + (known ? position : 0) * half;
  const float nan = __builtin_nanf("");  // a position outside the table: nothing to turn by
  if (P.style == ROTATE_STYLE_PAIRS) {
#pragma unroll
    for (int e = 0; e < 8; e += 2) {
      if (c0 + e >= P.rot) continue;
      const F c = known ? cosine[c0 / 2 + e / 2] : nan, s = known ? sine[c0 / 2 + e / 2] : nan;
      const F a = x[e], b = x[e + 1];
      x[e] = a * c - b * s;
      x[e + 1] = b * c + a * s;
    }
    return;
  }
#pragma unroll
  for (int e = 0; e < 8; ++e) row[c0 + e] = x[e];
  // same wave wrote and reads: LDS operations of a wave complete in order
  __builtin_amdgcn_wave_barrier();
  asm volatile("" ::: "memory");
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    const int c = c0 + e;
    if (c >= P.rot) continue;
    const bool second = c >= half;
    const int j = second ? c - half : c;
    const F other = row[second ? j : j + half];
    const F cs = known ? cosine[j] : nan, sn = known ? sine[j] : nan;
    x[e] = second ? x[e] * cs + other * sn : x[e] * cs - other * sn;
  }
  __builtin_amdgcn_wave_barrier();
  asm volatile("" ::: "memory");
}

template <int TYPE, typename F>
__device__ __forceinline__ void load_head(const void *p, int64_t at, F (&x)[8]) {
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    const v4f v = load_real4(p, at + 4 * h, TYPE);
#pragma unroll
    for (int e = 0; e < 4; ++e) x[4 * h + e] = v[e];
  }
}
template <int TYPE, typename F>
__device__ __forceinline__ void store_head(void *p, int64_t at, const F (&x)[8]) {
#pragma unroll
  for (int h = 0; h < 2; ++h)
    store_real4(p, at + 4 * h, TYPE, v4f{(float)x[4 * h], (float)x[4 * h + 1], (float)x[4 * h + 2], (float)x[4 * h + 3]});
}

template <int D, int TYPE>
__global__ __launch_bounds__(256) void rope_kernel(RopeArgs P) {
  constexpr int LANES = D / 8, HEADS = 256 / LANES;  // of a workgroup
  __shared__ double rows[HEADS][D];
  const int lane = threadIdx.x % LANES, mine = threadIdx.x / LANES;
  const int64_t token = P.token0 + blockIdx.x / P.blocks;
  int head = (int)(blockIdx.x % P.blocks) * HEADS + mine;
  if (head < P.q_heads) {
    float x[8];
    load_head<TYPE>(P.Q, token * P.ldq + head * D + 8 * lane, x);
    norm_and_rotate<D>(P, P.q_weight, token, lane, x, reinterpret_cast<float *>(rows[mine]));
    store_head<TYPE>(P.Qo, token * P.ldqo + head * D + 8 * lane, x);
    return;
  }
  head -= P.q_heads;
  if (head < P.kv_heads) {
    if (!P.Ko && !P.cache) return;
    double x[8];
    load_head<TYPE>(P.K, token * P.ldk + head * D + 8 * lane, x);
    norm_and_rotate<D>(P, P.k_weight, token, lane, x, rows[mine]);
    if (P.Ko) store_head<TYPE>(P.Ko, token * P.ldko + head * D + 8 * lane, x);
    if (P.cache) put_in_cache<D>(P, token, head, lane, false, x);
    return;
  }
  head -= P.kv_heads;
  if (head < P.kv_heads && P.cache) {
    double x[8];
    load_head<TYPE>(P.V, token * P.ldv + head * D + 8 * lane, x);
    put_in_cache<D>(P, token, head, lane, true, x);
  }
}

template <int D, int TYPE>
__global__ __launch_bounds__(256) void kv4_read_kernel(Kv4ReadArgs P) {
  constexpr int LANES = D / 8, HEADS = 256 / LANES;
  const int lane = threadIdx.x % LANES;
  const int64_t token = P.token0 + blockIdx.x / P.blocks;
  const int both = (int)(blockIdx.x % P.blocks) * HEADS + threadIdx.x / LANES;
  if (both >= 2 * P.kv_heads) return;
  const bool value = both >= P.kv_heads;
  const int head = value ? both - P.kv_heads : both;
  void *to = value ? P.V : P.K;
  if (!to) return;
  const int64_t slot = P.slots[token];
  float x[8] = {0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f};
  if (slot >= 0 && slot < P.pages << P.log_page) {
    const Kv4Layout L(1 << P.log_page, D);
    const Place at = place_of<D>(const_cast<uint8_t *>(P.cache), slot, P.log_page, P.kv_heads, head);
    const uint32_t word = *reinterpret_cast<const uint32_t *>(
        at.part + (value ? L.values + 16 * ((at.token >> 2) * (D / 8) + lane) + 4 * (at.token & 3)
                         : at.token * (D / 2) + 4 * lane));
    const uint32_t pair = *reinterpret_cast<const uint16_t *>(at.part + (value ? L.value_pairs : L.key_pairs) +
                                                              2 * (((lane >> 2) << P.log_page) + at.token));
    const float s = kv4_step(pair);
    const int z = kv4_zero(pair);
#pragma unroll
    for (int e = 0; e < 8; ++e) x[e] = s * (float)((int)((word >> (4 * e)) & 15) - z);
  }
  store_head<TYPE>(to, token * (value ? P.ldv : P.ldk) + head * D + 8 * lane, x);
}

// A launch takes as many tokens as a grid holds.
template <typename ARGS>
hipError_t launch_tokens(void (*const (&kernels)[3][3])(ARGS), ARGS P, int64_t tokens, int head_dim, int type, int heads,
                         hipStream_t s) {
  const int per = 256 / (head_dim / 8);
  P.blocks = (heads + per - 1) / per;
  const int64_t most = ((int64_t)1 << 23) / P.blocks > 0 ? ((int64_t)1 << 23) / P.blocks : 1;
  void (*kernel)(ARGS) = kernels[head_dim == 64 ? 0 : (head_dim == 128 ? 1 : 2)][type];
  for (int64_t t = 0; t < tokens; t += most) {
    P.token0 = t;
    const int64_t here = tokens - t < most ? tokens - t : most;
    const hipError_t e = launch_with(reinterpret_cast<const void *>(kernel), dim3((unsigned)(here * P.blocks)), 256, 0, s, &P);
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}

#define MIP_BY_TYPE(K, D) {K<D, REAL_F32>, K<D, REAL_BF16>, K<D, REAL_F16>}

}  // namespace

hipError_t launch_rope(const RopeArgs &P, int64_t tokens, int head_dim, int type, hipStream_t s) {
  static void (*const kernels[3][3])(RopeArgs) = {MIP_BY_TYPE(rope_kernel, 64), MIP_BY_TYPE(rope_kernel, 128),
                                                  MIP_BY_TYPE(rope_kernel, 256)};
  const int heads = P.q_heads + (P.cache ? 2 : (P.Ko ? 1 : 0)) * P.kv_heads;
  return heads ? launch_tokens(kernels, P, tokens, head_dim, type, heads, s) : hipSuccess;
}

hipError_t launch_kv4_read(const Kv4ReadArgs &P, int64_t tokens, int head_dim, int type, hipStream_t s) {
  static void (*const kernels[3][3])(Kv4ReadArgs) = {MIP_BY_TYPE(kv4_read_kernel, 64), MIP_BY_TYPE(kv4_read_kernel, 128),
                                                     MIP_BY_TYPE(kv4_read_kernel, 256)};
  return launch_tokens(kernels, P, tokens, head_dim, type, 2 * P.kv_heads, s);
}

}  // namespace mip
