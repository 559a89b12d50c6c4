// Heads of queries, keys and values between the projections of a layer and its attention: RMS norm of each
// head of queries and keys, their rotation by position, and keys and values written to the 4-bit cache; and
// rows of that cache read back.
//
// Every number is read once and written once, in one launch, so that nothing between the projection and the cache
// goes to memory: 8192 tokens of 32 heads of queries and 8 of keys and values, 128 channels in bfloat16, would take
// 34 us at the rate of a copy.  They take 54 resident, bound by vector instructions (some 260 for a wave's heads, 41 us of
// issue), and 70 from memory (177 MB at 2.5 TB/s), where a wave waits for its numbers besides.  In float32 93, with rotations that
// are no multiple of 16 133, with keys as numbers, all of which go through float64, 82.  d / 8 lanes to a head, eight channels to a lane:
// a wave takes 8, 4 or 2 heads at a time, all of one kind, so that what kind they are is decided by scalar branches.
// What a rotation joins to a lane's channels is loaded a second time (from the first cache) rather than passed between
// lanes: through LDS the kernel took 88 us.  Weights and rotation become one factor for each channel and one for its
// partner, once for a token and kind; the sums of squares meet in registers.
//
// All of it is worked out in float32; where a key's code or a group's step lies so near the middle between two that
// float32's roundings could decide it, the wave's turn is done again in float64 (one turn in fifty to a hundred): the
// codes are those of the exact keys, whichever order the squares are summed in.  So is a turn, of queries too, with a head whose mean of
// squares float32 cannot hold, or holds to few bits.
#include "kv4.h"
#include "layer_internal.h"

namespace mip {

namespace {

// 1 / sqrt(x): the instruction and one step of Newton's iteration.
__device__ __forceinline__ float inverse_root(float x) {
  const float r = __builtin_amdgcn_rsqf(x), better = r * __builtin_fmaf(-0.5f * x * r, r, 1.5f);
  return r > 0.0f && r < __builtin_inff() ? better : r;
}

// Eight numbers as they lie in memory.
template <int TYPE>
struct Raw {
  static constexpr int WORDS = TYPE == REAL_F32 ? 8 : 4;
  uint32_t w[WORDS];
  __device__ __forceinline__ void load(const void *from, int64_t at) {
    const v4w *p = reinterpret_cast<const v4w *>(static_cast<const uint8_t *>(from) + at * (WORDS / 2));
#pragma unroll
    for (int g = 0; g < WORDS / 4; ++g) {
      const v4w v = p[g];
#pragma unroll
      for (int e = 0; e < 4; ++e) w[4 * g + e] = v[e];
    }
  }
  __device__ __forceinline__ void load_one(const void *from, int64_t at, int e) {
    if constexpr (TYPE == REAL_F32) w[e] = static_cast<const uint32_t *>(from)[at];
    else w[e / 2] = (e % 2 ? w[e / 2] & 0xffff : 0) | (uint32_t)static_cast<const uint16_t *>(from)[at] << (e % 2 * 16);
  }
  __device__ __forceinline__ float operator[](int e) const {
    if constexpr (TYPE == REAL_F32) return __int_as_float((int)w[e]);
    if constexpr (TYPE == REAL_BF16) return __int_as_float((int)(e % 2 ? w[e / 2] & 0xffff0000u : w[e / 2] << 16));
    return (float)__builtin_bit_cast(v2h, w[e / 2])[e % 2];
  }
  // either of two neighbours in the other's place
  __device__ __forceinline__ Raw swapped() const {
    Raw r;
#pragma unroll
    for (int i = 0; i < WORDS; ++i) r.w[i] = TYPE == REAL_F32 ? w[i ^ 1] : w[i] >> 16 | w[i] << 16;
    return r;
  }
};

// Where a slot's token lies: the head's part of its page, and the token's place in it.
struct Place {
  uint8_t *part;
  int token;
};
template <int D>
__device__ __forceinline__ Place place_of(uint8_t *cache, int64_t slot, int log_page, int kv_heads, int head) {
  const uint32_t block = (uint32_t)(D / 8 * 9) << log_page;  // (1024 heads of it stay below 2^32)
  return {cache + (slot >> log_page) * (int64_t)(block * (uint32_t)kv_heads) + block * (uint32_t)head,
          (int)(slot & ((1 << log_page) - 1))};
}
// Bytes from there to a lane's word of codes, and to its group's pair.
template <int D>
__device__ __forceinline__ uint32_t word_at(int token, int lane, bool value, int log_page) {
  const uint32_t values = (uint32_t)(D / 16 * 9) << log_page;
  return value ? values + 16 * ((token >> 2) * (D / 8) + lane) + 4 * (token & 3) : (uint32_t)(token * (D / 2) + 4 * lane);
}
template <int D>
__device__ __forceinline__ uint32_t pair_at(int token, int lane, bool value, int log_page) {
  return ((uint32_t)(value ? D / 16 * 17 : D / 2) << log_page) + 2 * (((lane >> 2) << log_page) + token);
}

template <int D>
__device__ __forceinline__ void put_in_cache(const RopeArgs &P, int64_t slot, int head, int lane, bool value, uint32_t word,
                                             uint32_t pair) {
  if (slot < 0 || slot >= P.pages << P.log_page) return;
  const Place at = place_of<D>(P.cache, slot, P.log_page, P.kv_heads, head);
  *reinterpret_cast<uint32_t *>(at.part + word_at<D>(at.token, lane, value, P.log_page)) = word;
  if ((lane & 3) == 0) *reinterpret_cast<uint16_t *>(at.part + pair_at<D>(at.token, lane, value, P.log_page)) = (uint16_t)pair;
}

// What becomes of a lane's eight channels but for the root: y(c) = x(c) weight cosine + x(partner) its weight sine, the sine
// negative for a pair's first.
struct Turn {
  float cosine[8], sine[8], own[8], other[8];
};
template <bool EIGHTS>
__device__ __forceinline__ Turn turn_of(const RopeArgs &P, int64_t token, int c0, const float *weight) {
  Turn t;
  // (worked out anew for each kind of head: its addresses, kept over the loop over heads, would take its registers)
  asm volatile("" : "+v"(c0));
  const int half = P.rot / 2;
  const bool pairs = P.style == ROTATE_STYLE_PAIRS;
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    t.cosine[e] = t.own[e] = t.other[e] = 1.0f;
    t.sine[e] = 0.0f;
  }
  auto load8 = [](const float *from, int at, float (&to)[8]) { load_real8<REAL_F32>(from, at, to); };
  if (weight) load8(weight, c0, t.own);
  // a position outside the tables: none of the head's channels is a number, not even one that is not turned
  auto in_tables = [&](int64_t position) { return position >= 0 && position < P.table_rows; };
  if (c0 >= P.rot) {
    if (P.rot > 0 && !in_tables(P.positions[token])) {
#pragma unroll
      for (int e = 0; e < 8; ++e) t.cosine[e] = __builtin_nanf("");
    }
    return t;
  }
  const int64_t position = P.positions[token];
  const bool known = in_tables(position);
  const float *cosine = P.cosine + (known ? position : 0) * half, *sine = P.sine + (known ? position : 0) * half;
  auto partner = [&](int c) { return pairs ? c ^ 1 : (c < half ? c + half : c - half); };
  if (!known) {
#pragma unroll
    for (int e = 0; e < 8; ++e) t.cosine[e] = __builtin_nanf("");
  } else if constexpr (!EIGHTS) {
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const int c = c0 + e;
      if (c >= P.rot) continue;
      const bool first = pairs ? e % 2 == 0 : c < half;
      const int j = pairs ? c / 2 : (first ? c : c - half);
      t.cosine[e] = cosine[j];
      t.sine[e] = first ? -sine[j] : sine[j];
      if (weight) t.other[e] = weight[partner(c)];
    }
  } else if (pairs) {
    const v4f c = load_real4(cosine, c0 / 2, REAL_F32), s = load_real4(sine, c0 / 2, REAL_F32);
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      t.cosine[e] = c[e / 2];
      t.sine[e] = e % 2 ? s[e / 2] : -s[e / 2];
      t.other[e] = t.own[e ^ 1];
    }
  } else {
    const bool first = c0 < half;
    const int j = first ? c0 : c0 - half;
    load8(cosine, j, t.cosine);
    load8(sine, j, t.sine);
#pragma unroll
    for (int e = 0; e < 8; ++e) t.sine[e] = first ? -t.sine[e] : t.sine[e];
    if (weight) load8(weight, partner(c0), t.other);
  }
  return t;
}

// The same for all lanes of a head.
template <int LANES>
__device__ __forceinline__ float sum_of_head(float x) {
  x += of_lane<LANE_XOR_1>(x);
  x += of_lane<LANE_XOR_2>(x);
  x += of_lane<LANE_MIRROR_8>(x);
  if (LANES > 8) x += of_lane<LANE_MIRROR_16>(x);
  if (LANES > 16) x += __shfl_xor(x, 16);
  return x;
}

// Whether float32 held the mean of squares, eps in it, well whose inverse root this is: from 2^-100 to 2^120.  No square is
// past it then, and what is lost of small ones is below 2^-40 of the mean.  (As a whole number: one subtraction, one comparison,
// and NaN is out.)
__device__ __forceinline__ bool mean_was_held(float root) {
  return __float_as_uint(root) - ((127u - 60u) << 23) <= (110u << 23);
}

// EIGHTS: a lane's eight channels meet eight in a row, or are none that are rotated (the number of rotated channels is a
// multiple of 16, of 8 in pairs); else they are looked for one by one.
// (five waves to a SIMD where the registers allow it: 67 us with the reading back of the cache, 74 with four)
template <int D, int TYPE, bool EIGHTS>
__global__ __launch_bounds__(256, EIGHTS && TYPE != REAL_F32 && D < 256 ? 5 : 4) void rope_kernel(RopeArgs P) {
  constexpr int LANES = D / 8, HEADS = 64 / LANES;  // of a wave at a time, all of one kind: queries, keys or values
  int lane = threadIdx.x % LANES, c0 = 8 * lane, mine = threadIdx.x % 64 / LANES;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int64_t token = P.token0 + blockIdx.x / P.blocks;
  const int step = 4 * P.blocks, first = (int)(blockIdx.x % P.blocks) * 4 + wave;
  const int q_turns = (P.q_heads + HEADS - 1) / HEADS, kv_turns = (P.kv_heads + HEADS - 1) / HEADS;
  const int turns = q_turns + (P.cache ? 2 : (P.Ko ? 1 : 0)) * kv_turns;
  const int half = P.rot / 2;
  const bool pairs = P.style == ROTATE_STYLE_PAIRS;
  // A turn's kind of heads, and the lane's of them: behind the last one the last again, which is not written.
  struct Turned { int kind, head; bool here; };
  auto of_turn = [&](int turn) {
    const int kind = turn < q_turns ? 0 : (turn < q_turns + kv_turns ? 1 : 2);
    const int count = kind ? P.kv_heads : P.q_heads;
    const int head = (turn - (kind ? q_turns : 0) - (kind == 2 ? kv_turns : 0)) * HEADS + mine;
    return Turned{kind, head < count ? head : count - 1, head < count};
  };
  // A head's numbers, and those that the rotation joins to them: on their way while the head before is worked on.
  struct Numbers { Raw<TYPE> own, other; } now = {}, next = {};
  constexpr int SIZE = TYPE == REAL_F32 ? 4 : 2;
  auto fetch = [&](int turn, Numbers &x) {
    if (turn >= turns) return;
    const Turned t = of_turn(turn);
    const void *all = t.kind == 0 ? P.Q : (t.kind == 1 ? P.K : P.V);
    const uint8_t *row = static_cast<const uint8_t *>(all) + token * (t.kind == 0 ? P.ldq : (t.kind == 1 ? P.ldk : P.ldv)) * SIZE;
    const uint32_t at = (uint32_t)(t.head * D + c0);
    x.own.load(row, at);
    if (pairs || t.kind == 2) return;
    if (EIGHTS) {
      if (c0 < P.rot) x.other.load(row, c0 < half ? at + half : at - half);
    } else {
#pragma unroll
      for (int e = 0; e < 8; ++e)
        if (c0 + e < P.rot) x.other.load_one(row, c0 + e < half ? at + e + half : at + e - half, e);
    }
  };
  auto join = [&](Numbers &x) {
    if (pairs) x.other = x.own.swapped();
    if (P.rot == D) return;
    constexpr int EACH = 8 / Raw<TYPE>::WORDS;  // (what is not rotated: not even an infinity times zero)
#pragma unroll
    for (int i = 0; i < Raw<TYPE>::WORDS; ++i) x.other.w[i] = c0 + EACH * i < P.rot ? x.other.w[i] : 0;
  };
  fetch(first, next);
  const int64_t slot = P.cache ? P.slots[token] : -1;
  auto write = [&](const Turned &t, const float (&y)[8]) {
    uint8_t *row = static_cast<uint8_t *>(t.kind ? P.Ko : P.Qo) + token * (t.kind ? P.ldko : P.ldqo) * SIZE;
    if (t.here) store_real8<TYPE>(row, (uint32_t)(t.head * D + c0), y);
  };
  float own_by[8], other_by[8];  // of the kind of head that was the last: weights and rotation in one
  int known = -1;
  uint64_t again = 0, bit = 1;  // the turns (64 at most) that are to be done in float64
  for (int turn = first; turn < turns; turn += step, bit <<= 1) {
    now = next;
    fetch(turn + step, next);
    const Turned t = of_turn(turn);
    if (t.kind == 1 && P.Ko) {  // (keys that leave as numbers are worked out in float64)
      again |= bit;
      continue;
    }
    float y[8], error = TYPE == REAL_F32 ? 1e-38f : 0.0f;  // (of values none, but in 32 bits the quotients' own rounding counts)
    if (t.kind < 2) {
      const float *weight = t.kind ? P.k_weight : P.q_weight;
      if (known != t.kind) {
        known = t.kind;
        const Turn by = turn_of<EIGHTS>(P, token, c0, weight);
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          own_by[e] = by.cosine[e] * by.own[e];
          other_by[e] = by.sine[e] * by.other[e];
        }
      }
      join(now);
      // What float32's roundings can have moved a channel by: those of the sum of squares (a chain of 8 + log2 LANES
      // additions, halved by the root), the root's, the weight's and three products' are below 20 of 2^-24 of the larger of
      // its two terms.
      float sum = 0.0f, largest = 0.0f;
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const float x = now.own[e], p = x * own_by[e];
        sum = __builtin_fmaf(x, x, sum);
        y[e] = __builtin_fmaf(now.other[e], other_by[e], p);
        if (t.kind) largest = most3(largest, fabsf(p), fabsf(y[e]));
      }
      const float root = weight ? inverse_root(sum_of_head<LANES>(sum) * (float)(1.0 / D) + P.eps) : 1.0f;
      if (__any(!mean_was_held(root))) {
        again |= bit;
        continue;
      }
#pragma unroll
      for (int e = 0; e < 8; ++e) y[e] *= root;
      if (t.kind == 0) {
        write(t, y);
        continue;
      }
      largest = __builtin_fmaxf(largest, of_lane<LANE_XOR_1>(largest));
      largest = __builtin_fmaxf(largest, of_lane<LANE_XOR_2>(largest));
      error = largest * root * 0x1.4p-20f;
    } else {
#pragma unroll
      for (int e = 0; e < 8; ++e) y[e] = now.own[e];
    }
    uint32_t pair;
    bool unsure;
    const uint32_t word = kv4_encode(y, error, &pair, &unsure);
    if (__any(unsure)) again |= bit;
    else if (t.here) put_in_cache<D>(P, slot, t.head, lane, t.kind == 2, word, pair);
  }
  if (!again) return;
  bit = 1;
  // (the same once more, which is cheaper than a register over the loop above: with one spilled it takes 67 us instead of 65)
  const int in_wave = __builtin_amdgcn_mbcnt_hi(~0u, __builtin_amdgcn_mbcnt_lo(~0u, 0u));
  lane = in_wave % LANES;
  c0 = 8 * lane;
  mine = in_wave / LANES;
  for (int turn = first; turn < turns; turn += step, bit <<= 1) {
    const Turned t = of_turn(turn);
    if (!(again & bit)) continue;
    fetch(turn, now);
    double z[8];
    if (t.kind < 2) {
      const float *weight = t.kind ? P.k_weight : P.q_weight;
      join(now);
      double sum = 0.0, root = 1.0;
#pragma unroll
      for (int e = 0; e < 8; ++e) sum += (double)now.own[e] * now.own[e];
#pragma unroll
      for (int d = 1; d < LANES; d *= 2) sum += __shfl_xor(sum, d);
      if (weight) root = 1.0 / __builtin_sqrt(sum * (1.0 / D) + (double)P.eps);
      const Turn by = turn_of<EIGHTS>(P, token, c0, weight);
      float y[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        z[e] = root * ((double)now.own[e] * by.own[e] * by.cosine[e] + (double)now.other[e] * by.other[e] * by.sine[e]);
        y[e] = (float)z[e];
      }
      if (t.kind == 0 || P.Ko) write(t, y);
      if (t.kind == 0) continue;
    } else {
#pragma unroll
      for (int e = 0; e < 8; ++e) z[e] = now.own[e];
    }
    uint32_t pair;
    const uint32_t word = kv4_encode(z, &pair);
    if (P.cache && t.here) put_in_cache<D>(P, slot, t.head, lane, t.kind == 2, word, pair);
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
      const Place at = place_of<D>(const_cast<uint8_t *>(P.cache), slot, P.log_page, P.kv_heads, head);
      const uint32_t word = *reinterpret_cast<const uint32_t *>(at.part + word_at<D>(at.token, lane, value, P.log_page));
      const uint32_t pair = *reinterpret_cast<const uint16_t *>(at.part + pair_at<D>(at.token, lane, value, P.log_page));
      const float s = kv4_step(pair);
      const int z = kv4_zero(pair);
#pragma unroll
      for (int e = 0; e < 8; ++e) x[e] = s * (float)((int)((word >> (4 * e)) & 15) - z);
    }
    store_real8<TYPE>(to, token * (value ? P.ldv : P.ldk) + head * D + 8 * lane, x);
  }
}

// A launch takes as many tokens as a grid holds.  groups: workgroups that a token has work for.
template <typename ARGS>
hipError_t launch_tokens(void (*const (&kernels)[3][3])(ARGS), ARGS P, int64_t tokens, int head_dim, int type, int groups,
                         hipStream_t s) {
  // a workgroup to a token, which shares what the token is turned by, where there are enough of them (8192 tokens and
  // their reading back 67 us, 85 with a workgroup to every four turns), and to 64 turns of a wave, which it has a bit for
  P.blocks = tokens >= 8 * compute_units() ? (groups + 63) / 64 : groups;
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

template <int D, int TYPE>
constexpr auto rope_ones = rope_kernel<D, TYPE, false>;
template <int D, int TYPE>
constexpr auto rope_eights = rope_kernel<D, TYPE, true>;

#define MIP_BY_TYPE(K, D) {K<D, REAL_F32>, K<D, REAL_BF16>, K<D, REAL_F16>}

}  // namespace

hipError_t launch_rope(const RopeArgs &P, int64_t tokens, int head_dim, int type, hipStream_t s) {
  static void (*const kernels[2][3][3])(RopeArgs) = {
      {MIP_BY_TYPE(rope_ones, 64), MIP_BY_TYPE(rope_ones, 128), MIP_BY_TYPE(rope_ones, 256)},
      {MIP_BY_TYPE(rope_eights, 64), MIP_BY_TYPE(rope_eights, 128), MIP_BY_TYPE(rope_eights, 256)}};
  const bool eights = P.rot % (P.style == ROTATE_STYLE_PAIRS ? 8 : 16) == 0;
  const int per = 512 / head_dim;  // heads that a wave takes at a time
  const int turns = (P.q_heads + per - 1) / per + (P.cache ? 2 : (P.Ko ? 1 : 0)) * ((P.kv_heads + per - 1) / per);
  return turns ? launch_tokens(kernels[eights], P, tokens, head_dim, type, (turns + 3) / 4, s) : hipSuccess;
}

hipError_t launch_kv4_read(const Kv4ReadArgs &P, int64_t tokens, int head_dim, int type, hipStream_t s) {
  static void (*const kernels[3][3])(Kv4ReadArgs) = {MIP_BY_TYPE(kv4_read_kernel, 64), MIP_BY_TYPE(kv4_read_kernel, 128),
                                                     MIP_BY_TYPE(kv4_read_kernel, 256)};
  return launch_tokens(kernels, P, tokens, head_dim, type, (2 * P.kv_heads * head_dim + 2047) / 2048, s);
}

}  // namespace mip
