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

// num / s, correctly rounded (r is 1 / s, correctly rounded; Markstein's theorem).
template <typename F>
__device__ __forceinline__ F kv4_quotient(F num, F s, F r) {
  const F q = num * r;
  if constexpr (sizeof(F) == 8) return __builtin_fma(__builtin_fma(-q, s, num), r, q);
  else return __builtin_fmaf(__builtin_fmaf(-q, s, num), r, q);
}

// A lane's eight channels of a group that four neighbouring lanes hold: the word of codes, and the pair of the
// group (in every lane).  All four lanes call it.  In float32, `unsure` is set where an error of `error` in a channel, and of
// the roundings here, could move a code or the step: there the caller does it again in float64.  (Without an error,
// numbers of 16 bits leave nothing to be unsure of but the step: their quotients by four significant bits are
// further from the middle between two codes than a rounding, or on it.)
template <typename F>
__device__ __forceinline__ uint32_t kv4_encode(const F (&x)[8], F error, uint32_t *pair, bool *unsure) {
  constexpr bool WIDE = sizeof(F) == 8;
  F lo = 0, hi = 0, v[8];
  int bad = 0;
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    bad |= !(x[e] - x[e] == 0);
    v[e] = x[e] > (F)KV4_TOP ? (F)KV4_TOP : (x[e] < -(F)KV4_TOP ? -(F)KV4_TOP : x[e]);
    lo = e == 0 || v[e] < lo ? v[e] : lo;
    hi = e == 0 || v[e] > hi ? v[e] : hi;
  }
#pragma unroll
  for (int d = 1; d < 4; d *= 2) {
    const F l = __shfl_xor(lo, d), h = __shfl_xor(hi, d);
    lo = l < lo ? l : lo;
    hi = h > hi ? h : hi;
    bad |= __shfl_xor(bad, d);
  }
  *unsure = false;
  if (bad) {
    *pair = 0xff;
    return 0;
  }
  const F most = hi > -lo ? hi : -lo;
  const F range = WIDE ? (hi - lo) / 15 : (hi - lo) * (F)(1.0 / 15), size = WIDE ? most / 112 : most * (F)(1.0 / 112);
  const F step = range > size ? range : size;
  F s;
  if constexpr (WIDE) {
    s = step < 0x1p-14 ? __builtin_ceil(step * 0x1p17) * 0x1p-17
                       : __longlong_as_double((__double_as_longlong(step) + ((1LL << 49) - 1)) & ~((1LL << 49) - 1));
  } else {
    const float wide = step * 0x1p17f, off = error * 0x1p15f + wide * 0x1p-21f;  // (of step: a seventh of twice the error)
    if (step < 0x1p-14f) {
      s = __builtin_ceilf(wide) * 0x1p-17f;
      *unsure = step > 0.0f && fabsf(wide - __builtin_rintf(wide)) <= off;
    } else {
      s = __int_as_float((__float_as_int(step) + 0xfffff) & ~0xfffff);
      const float below = __int_as_float(__float_as_int(step) & ~0xfffff);  // the nearest such numbers on either side
      *unsure = (step - below) * 0x1p17f <= off || (s - step) * 0x1p17f <= off;
    }
  }
  const F over = s > 0 ? s : (F)1, r = (F)1 / over;
  const F z = -__builtin_rint(kv4_quotient(lo, over, r));
  const F doubt = (F)0.5 - error * r * (F)1.0625 - (error > 0 ? most * r * (F)0x1p-21 : (F)0);
  uint32_t word = 0;
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    const F t = kv4_quotient(v[e], over, r), whole = WIDE ? __builtin_rint(t) : __builtin_rintf(t);
    if (!WIDE && error > 0) *unsure |= fabsf(t - whole) >= doubt;
    F n = whole + z;
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
