// A row's codes of 8 bits, as every operator that writes them forms them.
#pragma once
#include "real.h"

namespace mip {

template <typename T>
struct real_of;
template <> struct real_of<float> { static constexpr int type = REAL_F32; };
template <> struct real_of<__bf16> { static constexpr int type = REAL_BF16; };
template <> struct real_of<_Float16> { static constexpr int type = REAL_F16; };

struct __attribute__((packed, aligned(1))) byte_oct { uint64_t v; };

// The quotient 127 z / a, correctly rounded: the reciprocal r of a is, and one step of Newton's iteration on the quotient
// then is as well (Markstein's theorem), where nothing underflows; then the nearest whole number, ties to even, in the
// lowest byte (1.5 2^23 leaves no bits for fractions).
__device__ __forceinline__ uint32_t code_of(float z, float by, float a, float r) {
  const float num = __fmul_rn(z, by), q = num * r;
  return __float_as_uint(__fadd_rn(__builtin_fmaf(__builtin_fmaf(-q, a, num), r, q), 12582912.0f));
}
// the lowest bytes of four words
__device__ __forceinline__ uint32_t four_bytes(uint32_t a, uint32_t b, uint32_t c, uint32_t d) {
  return __builtin_amdgcn_perm(__builtin_amdgcn_perm(d, c, 0x0c0c0400u), __builtin_amdgcn_perm(b, a, 0x0c0c0400u), 0x05040100u);
}

// far from 1, a power of two keeps the reciprocal and the products in range, and changes no quotient
__device__ __forceinline__ float code_range(float top) { return top < 0x1p-60f ? 0x1p60f : (top > 0x1p60f ? 0x1p-60f : 1.0f); }

// The bytes of eight numbers, `count` of which exist, at q (of any alignment); r 0: zeros.
__device__ __forceinline__ void put_codes(int8_t *q, int64_t count, const float (&v)[8], float by_127, float a, float r) {
  uint32_t n[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) n[e] = code_of(v[e], by_127, a, r);
  const uint64_t both = (uint64_t)four_bytes(n[4], n[5], n[6], n[7]) << 32 | four_bytes(n[0], n[1], n[2], n[3]);
  const uint64_t word = r != 0.0f ? both : 0;
  if (count >= 8) {
    reinterpret_cast<byte_oct *>(q)->v = word;
  } else {
#pragma unroll
    for (int e = 0; e < 7; ++e)
      if (e < count) q[e] = (int8_t)(word >> (8 * e));
  }
}

}  // namespace mip
