// Heads of queries, keys and values between the projections of a layer and its attention: RMS norm of each
// head of queries and keys, their rotation by position, and keys and values written to the 4-bit cache; and
// rows of that cache read back.
//
// Bound by memory (every number is read once and written once); one launch, so that nothing between the
// projection and the cache goes to memory.  d / 8 lanes to a head, eight channels to a lane: a wave takes 8, 4 or
// 2 heads.  All of it is worked out in float32; where a key's code or a group's step lies so near the middle between
// two that float32's roundings could decide it, the wave's heads are done again in float64 (some waves in a hundred): the
// codes are those of the exact keys, whichever order the squares are summed in.
#include "kv4.h"
#include "layer_internal.h"

namespace mip {

namespace {

// 1 / sqrt(x): the instruction and one step of Newton's iteration in float32.
template <typename F>
__device__ __forceinline__ F inverse_root(F x) {
  if constexpr (sizeof(F) == 8) {
    return 1.0 / __builtin_sqrt(x);
  } else {
    const float r = __builtin_amdgcn_rsqf(x), better = r * __builtin_fmaf(-0.5f * x * r, r, 1.5f);
    return r > 0.0f && r < __builtin_inff() ? better : r;
  }
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
__device__ __forceinline__ void put_in_cache(const RopeArgs &P, int64_t slot, int head, int lane, bool value, uint32_t word,
                                             uint32_t pair) {
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

// What a lane's eight channels are turned by: y(c) cosine + y(partner) sine, the sine negative for a pair's first.
struct Turn {
  float cosine[8], sine[8];
  int partner;  // HALVES, rot_dim a multiple of 16: the first of the channels that the lane's meet
};
template <int D>
__device__ __forceinline__ Turn turn_of(const RopeArgs &P, int64_t token, int c0) {
  Turn t;
  t.partner = 0;
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    t.cosine[e] = 1.0f;
    t.sine[e] = 0.0f;
  }
  if (P.rot == 0) return t;
  const int64_t position = P.positions[token];
  const bool known = position >= 0 && position < P.table_rows;
  const int half = P.rot / 2;
  const float *cosine = P.cosine + (known ? position : 0) * half, *sine = P.sine + (known ? position : 0) * half;
  if (c0 < P.rot) {
    if (P.style == ROTATE_STYLE_HALVES && half % 8 == 0) {
      const int j = c0 < half ? c0 : c0 - half;
      t.partner = c0 < half ? c0 + half : j;
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const v4f c = load_real4(cosine, j + 4 * h, REAL_F32), s = load_real4(sine, j + 4 * h, REAL_F32);
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          t.cosine[4 * h + e] = c[e];
          t.sine[4 * h + e] = c0 < half ? -s[e] : s[e];
        }
      }
    } else if (P.style == ROTATE_STYLE_PAIRS && c0 + 8 <= P.rot) {
      const v4f c = load_real4(cosine, c0 / 2, REAL_F32), s = load_real4(sine, c0 / 2, REAL_F32);
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        t.cosine[e] = c[e / 2];
        t.sine[e] = e % 2 ? s[e / 2] : -s[e / 2];
      }
    } else {
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const int c = c0 + e;
        if (c >= P.rot) continue;
        const bool first = P.style == ROTATE_STYLE_PAIRS ? e % 2 == 0 : c < half;
        const int j = P.style == ROTATE_STYLE_PAIRS ? c / 2 : (first ? c : c - half);
        t.cosine[e] = cosine[j];
        t.sine[e] = first ? -sine[j] : sine[j];
      }
    }
  }
  if (!known) {  // a position outside the table: nothing to turn by
#pragma unroll
    for (int e = 0; e < 8; ++e) t.cosine[e] = __builtin_nanf("");
  }
  return t;
}

// Norm and rotation of the head whose channels 8 * lane .. + 7 are x; `row`: D numbers of LDS of its own.  Returns, for
// float32, a bound on what its roundings can have moved a channel by: those of the sum of squares (a chain of 8 + log2
// LANES additions), the root, two products and the rotation are below 16 of 2^-24 of the head's largest.
template <int D, typename F>
__device__ __forceinline__ F norm_and_rotate(const RopeArgs &P, const float *weight, const float (&gain)[8], const Turn &turn,
                                                int lane, F (&x)[8], F *row) {
  constexpr int LANES = D / 8;
  const int c0 = 8 * lane;
  if (weight) {
    F sum = 0;
#pragma unroll
    for (int e = 0; e < 8; ++e) sum += x[e] * x[e];
#pragma unroll
    for (int d = 1; d < LANES; d *= 2) sum += __shfl_xor(sum, d);
    const F root = inverse_root(sum * (F)(1.0 / D) + (F)P.eps);
#pragma unroll
    for (int e = 0; e < 8; ++e) x[e] = x[e] * root * (F)gain[e];
  }
  F largest = 0;
  if constexpr (sizeof(F) == 4) {
#pragma unroll
    for (int e = 0; e < 8; ++e) largest = fmaxf(largest, fabsf(x[e]));
#pragma unroll
    for (int d = 1; d < LANES; d *= 2) largest = fmaxf(largest, __shfl_xor(largest, d));
    largest *= 0x1p-20f;
  }
  if (P.rot == 0) return largest;
  F other[8];
  if (P.style == ROTATE_STYLE_PAIRS) {
#pragma unroll
    for (int e = 0; e < 8; ++e) other[e] = x[e ^ 1];
  } else {
    typedef F v4 __attribute__((ext_vector_type(4)));
#pragma unroll
    for (int g = 0; g < 2; ++g)
      *reinterpret_cast<v4 *>(row + c0 + 4 * g) = v4{x[4 * g], x[4 * g + 1], x[4 * g + 2], x[4 * g + 3]};
    // same wave wrote and reads: LDS operations of a wave complete in order
    __builtin_amdgcn_wave_barrier();
    asm volatile("" ::: "memory");
    if (P.rot % 16 == 0) {  // (then the channels that a lane's meet are eight in a row)
#pragma unroll
      for (int g = 0; g < 2; ++g) {
        const v4 y = *reinterpret_cast<const v4 *>(row + turn.partner + 4 * g);
#pragma unroll
        for (int e = 0; e < 4; ++e) other[4 * g + e] = y[e];
      }
    } else {
      const int half = P.rot / 2;
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const int c = c0 + e;
        other[e] = c < P.rot ? row[c < half ? c + half : c - half] : (F)0;
      }
    }
    __builtin_amdgcn_wave_barrier();
    asm volatile("" ::: "memory");
  }
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    const F y = x[e] * (F)turn.cosine[e] + other[e] * (F)turn.sine[e];
    if (c0 + e < P.rot) x[e] = y;
  }
  return largest;
}

template <int D, int TYPE>
__global__ __launch_bounds__(256, 4) void rope_kernel(RopeArgs P) {
  constexpr int LANES = D / 8, HEADS = 256 / LANES;  // of a workgroup at a time
  __shared__ __attribute__((aligned(16))) double rows[HEADS][D];
  const int lane = threadIdx.x % LANES, mine = threadIdx.x / LANES, c0 = 8 * lane;
  const int64_t token = P.token0 + blockIdx.x / P.blocks;
  const int heads = P.q_heads + (P.cache ? 2 : (P.Ko ? 1 : 0)) * P.kv_heads, step = HEADS * P.blocks;
  const int first = (int)(blockIdx.x % P.blocks) * HEADS + mine;
  // a head's numbers are on their way while the one before is worked on
  auto fetch = [&](int head, float (&x)[8]) {
    const int k = head - P.q_heads, v = k - P.kv_heads;
    if (head >= heads) return;
    if (k < 0) load_real8<TYPE>(P.Q, token * P.ldq + head * D + c0, x);
    else if (v < 0) load_real8<TYPE>(P.K, token * P.ldk + k * D + c0, x);
    else load_real8<TYPE>(P.V, token * P.ldv + v * D + c0, x);
  };
  float next[8] = {}, q_gain[8], k_gain[8];
  fetch(first, next);
  const Turn turn = turn_of<D>(P, token, c0);
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    q_gain[e] = P.q_weight ? P.q_weight[c0 + e] : 1.0f;
    k_gain[e] = P.k_weight ? P.k_weight[c0 + e] : 1.0f;
  }
  const int64_t slot = P.cache ? P.slots[token] : -1;
  for (int head = first; head < heads; head += step) {
    float x[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) x[e] = next[e];
    fetch(head + step, next);
    const int k = head - P.q_heads, v = k - P.kv_heads;
    if (k < 0) {
      norm_and_rotate<D>(P, P.q_weight, q_gain, turn, lane, x, reinterpret_cast<float *>(rows[mine]));
      store_real8<TYPE>(P.Qo, token * P.ldqo + head * D + c0, x);
      continue;
    }
    uint32_t word = 0, pair = 0;
    bool unsure = P.Ko != nullptr;  // (keys that leave as numbers are worked out in float64)
    if (!unsure) {
      float y[8], error = 0.0f;
#pragma unroll
      for (int e = 0; e < 8; ++e) y[e] = x[e];
      if (v < 0) error = norm_and_rotate<D>(P, P.k_weight, k_gain, turn, lane, y, reinterpret_cast<float *>(rows[mine]));
      else if (TYPE == REAL_F32) error = 1e-38f;  // (none, but the quotients' own rounding counts)
      word = kv4_encode(y, error, &pair, &unsure);
    }
    if (__any(unsure)) {
      double y[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) y[e] = x[e];
      if (v < 0) norm_and_rotate<D>(P, P.k_weight, k_gain, turn, lane, y, rows[mine]);
      if (v < 0 && P.Ko) {
#pragma unroll
        for (int e = 0; e < 8; ++e) x[e] = (float)y[e];
        store_real8<TYPE>(P.Ko, token * P.ldko + k * D + c0, x);
      }
      word = kv4_encode(y, 0.0, &pair, &unsure);
    }
    if (P.cache) put_in_cache<D>(P, slot, v < 0 ? k : v, lane, v >= 0, word, pair);
  }
}

template <int D, int TYPE>
__global__ __launch_bounds__(256) void kv4_read_kernel(Kv4ReadArgs P) {
  constexpr int LANES = D / 8, HEADS = 256 / LANES;
  const int lane = threadIdx.x % LANES;
  const int64_t token = P.token0 + blockIdx.x / P.blocks;
  const int64_t slot = P.slots[token];
  for (int both = (int)(blockIdx.x % P.blocks) * HEADS + threadIdx.x / LANES; both < 2 * P.kv_heads; both += HEADS * P.blocks) {
    const bool value = both >= P.kv_heads;
    const int head = value ? both - P.kv_heads : both;
    void *to = value ? P.V : P.K;
    if (!to) continue;
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
    store_real8<TYPE>(to, token * (value ? P.ldv : P.ldk) + head * D + 8 * lane, x);
  }
}

// A launch takes as many tokens as a grid holds.
template <typename ARGS>
hipError_t launch_tokens(void (*const (&kernels)[3][3])(ARGS), ARGS P, int64_t tokens, int head_dim, int type, int heads,
                         hipStream_t s) {
  const int per = 256 / (head_dim / 8);
  // a workgroup to a token, which shares what the token is turned by, where there are enough of them
  P.blocks = tokens >= 8 * compute_units() ? 1 : (heads + per - 1) / per;
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
