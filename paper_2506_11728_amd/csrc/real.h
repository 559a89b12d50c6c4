// Real numbers as the operators around the integer products take and give them: float32, bfloat16
// or float16 in memory, float32 in registers.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

namespace mip {

enum RealType { REAL_F32 = 0, REAL_BF16 = 1, REAL_F16 = 2 };  // MIPGEMM_F32, MIPGEMM_BF16, MIPGEMM_F16
inline bool real_type_ok(int t) { return t >= REAL_F32 && t <= REAL_F16; }
inline int64_t real_bytes(int t) { return t == REAL_F32 ? 4 : 2; }

typedef float v4f __attribute__((ext_vector_type(4)));
typedef float v2f __attribute__((ext_vector_type(2)));
typedef _Float16 v2h __attribute__((ext_vector_type(2)));
typedef _Float16 v4h __attribute__((ext_vector_type(4)));
typedef _Float16 v8h __attribute__((ext_vector_type(8)));
typedef __bf16 v4b __attribute__((ext_vector_type(4)));

// Four numbers in a row at any element's address.
template <typename V>
struct __attribute__((packed, aligned(2))) real_quad { V v; };

__device__ __forceinline__ v4f load_real4(const void *p, int64_t at, int type) {
  if (type == REAL_F32) return reinterpret_cast<const real_quad<v4f> *>(static_cast<const float *>(p) + at)->v;
  if (type == REAL_BF16)
    return __builtin_convertvector(reinterpret_cast<const real_quad<v4b> *>(static_cast<const __bf16 *>(p) + at)->v, v4f);
  return __builtin_convertvector(reinterpret_cast<const real_quad<v4h> *>(static_cast<const _Float16 *>(p) + at)->v, v4f);
}
// Eight in a row: one load of 16 bytes in a 16-bit type, two in float32.
template <int TYPE>
__device__ __forceinline__ void load_real8(const void *p, int64_t at, float (&x)[8]) {
  typedef __bf16 v8b __attribute__((ext_vector_type(8)));
  typedef float v8f __attribute__((ext_vector_type(8)));
  v8f v;
  if constexpr (TYPE == REAL_F32) v = reinterpret_cast<const real_quad<v8f> *>(static_cast<const float *>(p) + at)->v;
  else if constexpr (TYPE == REAL_BF16)
    v = __builtin_convertvector(reinterpret_cast<const real_quad<v8b> *>(static_cast<const __bf16 *>(p) + at)->v, v8f);
  else v = __builtin_convertvector(reinterpret_cast<const real_quad<v8h> *>(static_cast<const _Float16 *>(p) + at)->v, v8f);
#pragma unroll
  for (int e = 0; e < 8; ++e) x[e] = v[e];
}
template <int TYPE>
__device__ __forceinline__ void store_real8(void *p, int64_t at, const float (&x)[8]) {
  typedef __bf16 v8b __attribute__((ext_vector_type(8)));
  typedef float v8f __attribute__((ext_vector_type(8)));
  const v8f v = {x[0], x[1], x[2], x[3], x[4], x[5], x[6], x[7]};
  if constexpr (TYPE == REAL_F32) reinterpret_cast<real_quad<v8f> *>(static_cast<float *>(p) + at)->v = v;
  else if constexpr (TYPE == REAL_BF16)
    reinterpret_cast<real_quad<v8b> *>(static_cast<__bf16 *>(p) + at)->v = __builtin_convertvector(v, v8b);
  else reinterpret_cast<real_quad<v8h> *>(static_cast<_Float16 *>(p) + at)->v = __builtin_convertvector(v, v8h);
}
__device__ __forceinline__ float load_real(const void *p, int64_t at, int type) {
  if (type == REAL_F32) return static_cast<const float *>(p)[at];
  if (type == REAL_BF16) return (float)static_cast<const __bf16 *>(p)[at];
  return (float)static_cast<const _Float16 *>(p)[at];
}
typedef uint32_t v4w __attribute__((ext_vector_type(4), aligned(2)));
typedef uint32_t v2w __attribute__((ext_vector_type(2), aligned(2)));
template <bool STREAM = false>  // non-temporal
__device__ __forceinline__ void store_real4(void *p, int64_t at, int type, v4f v) {
  if (type == REAL_F32) {
    v4w *to = reinterpret_cast<v4w *>(static_cast<float *>(p) + at);
    const v4w w = __builtin_bit_cast(v4w, v);
    if (STREAM) __builtin_nontemporal_store(w, to);
    else *to = w;
    return;
  }
  v2w *to = reinterpret_cast<v2w *>(static_cast<uint16_t *>(p) + at);
  const v2w w = type == REAL_BF16 ? __builtin_bit_cast(v2w, __builtin_convertvector(v, v4b))
                                  : __builtin_bit_cast(v2w, __builtin_convertvector(v, v4h));
  if (STREAM) __builtin_nontemporal_store(w, to);
  else *to = w;
}
__device__ __forceinline__ void store_real(void *p, int64_t at, int type, float v) {
  if (type == REAL_F32) static_cast<float *>(p)[at] = v;
  else if (type == REAL_BF16) static_cast<__bf16 *>(p)[at] = (__bf16)v;
  else static_cast<_Float16 *>(p)[at] = (_Float16)v;
}

}  // namespace mip
