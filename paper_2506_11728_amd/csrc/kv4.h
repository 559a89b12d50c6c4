// The cache of keys and values in 4 bits: its form and its layout.
//
// Form.  32 channels of one token and head are a group:  x ~ s (n - z), n in 0 .. 15, z in -127 .. 127, s a
// float16 with three bits behind its leading one (eight bits: the float16's sign is 0 and its last seven bits
// are 0), so 4.5 bits a channel.  n - z has at most eight significant bits and s four: s (n - z) is exact in
// float16, which is what the matrix instructions that read the cache take, and nothing is rounded again on the
// way.  Zero is a value of every group.
//   s = max( (max - min) / 15, max |x| / 112 ), rounded up to such a number (to a multiple of 2^-17 below 2^-14)
//   z = -rint(min / s),  n = min(max(rint(x / s) + z, 0), 15)
// |x| is cut at 57344, so that s (n - z) stays finite in float16; a group with an infinity or NaN has a NaN for s.
//
// Layout.  A page holds `page` tokens (a power of two, 16 or more) of every head; a head's part of it is
//   the keys' codes      page x d / 2 bytes, token by token; channel 8 w + e is the e-th nibble, from the lowest
//                        bits on, of the token's word w
//   the keys' pairs      d / 32 groups x page tokens x (s >> 7 of its float16, z): 2 bytes
//   the values' codes    the same words with four tokens interleaved: word w of token t at 16 (t / 4 * d / 8 + w) + 4 (t % 4)
//   the values' pairs    as the keys'
// A wave that multiplies keys takes 16 bytes of one token to a lane; one that multiplies values needs, for a
// channel, the tokens in a row: four tokens of eight channels are 16 bytes in a row.
#pragma once
#include "real.h"

namespace mip {

struct Kv4Layout {
  int64_t key_pairs, values, value_pairs, block;  // bytes from the start of a head's part, and of the whole part
  __host__ __device__ Kv4Layout(int page, int d)
      : key_pairs((int64_t)page * d / 2), values((int64_t)page * d / 16 * 9),
        value_pairs((int64_t)page * d / 16 * 17), block((int64_t)page * d / 8 * 9) {}
};

constexpr double KV4_TOP = 57344.0;

// x of the lane that CTRL, a data-parallel primitive's control, names.
template <int CTRL>
__device__ __forceinline__ float of_lane(float x) {
  return __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(x), CTRL, 0xf, 0xf, true));
}
constexpr int LANE_XOR_1 = 0xb1, LANE_XOR_2 = 0x4e, LANE_MIRROR_8 = 0x141, LANE_MIRROR_16 = 0x140;

__device__ __forceinline__ float least3(float a, float b, float c) { return __builtin_fminf(__builtin_fminf(a, b), c); }
__device__ __forceinline__ float most3(float a, float b, float c) { return __builtin_fmaxf(__builtin_fmaxf(a, b), c); }

// num / s, correctly rounded (r is 1 / s, correctly rounded; Markstein's theorem).
__device__ __forceinline__ float kv4_quotient(float num, float s, float r) {
  const float q = num * r;
  return __builtin_fmaf(__builtin_fmaf(-q, s, num), r, q);
}

// A lane's eight channels of a group that four neighbouring lanes hold: the word of codes, and the pair of the
// group (in every lane).  All four lanes call it.  `error`: a bound on what is wrong with a channel.  With one, `unsure` is set
// where it, or the roundings here, could move a code or the step, and where a channel is no number, which may be one that
// float32 cannot hold before it is cut: there the caller does it again in float64.  Without one, for
// numbers of 16 bits, it is exact: their quotients by four significant bits are further from the middle between two codes
// than a rounding, or on it, and whether a step is large enough is asked of products and a difference that are not rounded.
__device__ __forceinline__ uint32_t kv4_encode(float (&x)[8], float error, uint32_t *pair, bool *unsure) {
  float lo = least3(x[0], x[1], x[2]), hi = most3(x[0], x[1], x[2]), none = 0.0f;
#pragma unroll
  for (int e = 3; e < 7; e += 2) {
    lo = least3(lo, x[e], x[e + 1]);
    hi = most3(hi, x[e], x[e + 1]);
  }
#pragma unroll
  for (int e = 0; e < 8; ++e) none = __builtin_fmaf(x[e], 0.0f, none);  // (NaN if one is none)
  lo = __builtin_fminf(lo, x[7]);
  hi = __builtin_fmaxf(hi, x[7]);
  lo = __builtin_fminf(lo, of_lane<LANE_XOR_1>(lo));
  hi = __builtin_fmaxf(hi, of_lane<LANE_XOR_1>(hi));
  none += of_lane<LANE_XOR_1>(none);
  lo = __builtin_fminf(lo, of_lane<LANE_XOR_2>(lo));
  hi = __builtin_fmaxf(hi, of_lane<LANE_XOR_2>(hi));
  none += of_lane<LANE_XOR_2>(none);
  constexpr float TOP = (float)KV4_TOP;
  if (hi > TOP || lo < -TOP) {
    lo = __builtin_amdgcn_fmed3f(lo, -TOP, TOP);
    hi = __builtin_amdgcn_fmed3f(hi, -TOP, TOP);
#pragma unroll
    for (int e = 0; e < 8; ++e) x[e] = __builtin_amdgcn_fmed3f(x[e], -TOP, TOP);
  }
  const float most = __builtin_fmaxf(hi, -lo), least = __builtin_fminf(hi, -lo);
  const float step = __builtin_fmaxf((hi - lo) * (float)(1.0 / 15), most * (float)(1.0 / 112));
  // the unit of four significant bits of x: a power of two, at least 2^-17
  auto unit_of = [](float of) {
    return __builtin_fmaxf(__int_as_float((__float_as_int(of) & 0x7f800000) - (3 << 23)), 0x1p-17f);
  };
  const float unit = unit_of(step), units = step * __int_as_float((254 << 23) - __float_as_int(unit));
  // rounded up from a little less than the step, and up by one unit more where that is too small
  const float low = __builtin_ceilf(units * (float)(1.0 - 0x1p-20)) * unit;
  const float s = 15.0f * low - most >= least && 112.0f * low >= most ? low : low + unit_of(low);
  const float over = s > 0.0f ? s : 1.0f, near = __builtin_amdgcn_rcpf(over);
  const float r = __builtin_fmaf(__builtin_fmaf(-over, near, 1.0f), near, near);  // (correctly rounded for four bits)
  const float z = __builtin_rintf(kv4_quotient(-lo, over, r));
  constexpr float WHOLE = 12582912.0f;  // 1.5 2^23: added to a number, it leaves the nearest whole one in the lowest bits
  const int from = (int)z - __float_as_int(WHOLE);
  uint32_t word = 0;
  float off = 0.0f;
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    const float t = kv4_quotient(x[e], over, r), w = t + WHOLE;
    off = __builtin_fmaxf(off, fabsf(t - (w - WHOLE)));
    const int n = __float_as_int(w) + from;
    word |= (uint32_t)(n < 0 ? 0 : (n > 15 ? 15 : n)) << (4 * e);
  }
  const bool number = none == 0.0f;
  // (of the step: a seventh of twice the error)
  *unsure = error > 0.0f && (!number || off >= 0.5f - error * r * 1.0625f - most * r * 0x1p-21f ||
            (step > 0.0f && fabsf(units - __builtin_rintf(units)) * unit <= error * 0.25f + step * 0x1p-21f));
  const uint16_t half = __builtin_bit_cast(uint16_t, (_Float16)s);  // (exact)
  *pair = number ? (uint32_t)(half >> 7) | ((uint32_t)(int)z & 0xff) << 8 : 0xff;
  return number ? word : 0;
}

// The same in float64.
__device__ __forceinline__ uint32_t kv4_encode(const double (&x)[8], uint32_t *pair) {
  double lo = 0, hi = 0, v[8];
  int bad = 0;
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    bad |= !(x[e] - x[e] == 0);
    v[e] = x[e] > KV4_TOP ? KV4_TOP : (x[e] < -KV4_TOP ? -KV4_TOP : x[e]);
    lo = e == 0 || v[e] < lo ? v[e] : lo;
    hi = e == 0 || v[e] > hi ? v[e] : hi;
  }
#pragma unroll
  for (int d = 1; d < 4; d *= 2) {
    const double l = __shfl_xor(lo, d), h = __shfl_xor(hi, d);
    lo = l < lo ? l : lo;
    hi = h > hi ? h : hi;
    bad |= __shfl_xor(bad, d);
  }
  if (bad) {
    *pair = 0xff;
    return 0;
  }
  const double most = hi > -lo ? hi : -lo, range = (hi - lo) / 15, size = most / 112, step = range > size ? range : size;
  const double s = step < 0x1p-14 ? __builtin_ceil(step * 0x1p17) * 0x1p-17
                                  : __longlong_as_double((__double_as_longlong(step) + ((1LL << 49) - 1)) & ~((1LL << 49) - 1));
  const double over = s > 0 ? s : 1.0, z = -__builtin_rint(lo / over);
  uint32_t word = 0;
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    double n = __builtin_rint(v[e] / over) + z;
    n = n < 0 ? 0 : (n > 15 ? 15 : n);
    word |= (uint32_t)(int)n << (4 * e);
  }
  const uint16_t half = __builtin_bit_cast(uint16_t, (_Float16)(float)s);  // (exact)
  *pair = (uint32_t)(half >> 7) | ((uint32_t)(int)z & 0xff) << 8;
  return word;
}

__device__ __forceinline__ float kv4_step(uint32_t pair) {
  return (float)__builtin_bit_cast(_Float16, (uint16_t)((pair & 0xff) << 7));
}
__device__ __forceinline__ int kv4_zero(uint32_t pair) { return (int)(int8_t)(pair >> 8); }

}  // namespace mip
