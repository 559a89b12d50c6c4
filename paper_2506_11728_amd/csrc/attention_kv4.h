// Attention over the 4-bit cache (kv4.h): what its kernels share.
//
//     o(i) = sum over t of p(i, t) v(t) / sum over t of p(i, t),   p(i, t) = exp(scale q(i) . k(t) - max)
// in one pass over the keys, with the running maximum and sum of the softmax in float32.  The queries of
// all heads that share a key head are the rows of one product: row = query * shared + head.
//
// The products are float16 matrix instructions on the cache's own numbers: a code's nibble under the exponent of
// 1024 or of 64 is the float16 1024 + n (64 + n), the zero point is subtracted and the step multiplied in float16,
// and both are exact.  What is rounded is p: to float16, eleven bits, which is what the instruction takes beside the values.  That is
// an eighth of the output's own rounding in bfloat16 and as much as it in float16 (one query of 301 keys: 2.7e-4 of the result
// instead of 2.0e-4).  Its sum, one more column of the product with the values, is of the rounded p.
//
// Of the kernels for few rows and for 256 channels, which are what follows here (kernel_attention_wide.hip has its own form
// of it): the instructions are v_mfma_f32_16x16x32_f16.  Queries in bfloat16 are multiplied by a power of two that
// brings the row's largest below 32768 and are exact as float16 wherever they are not 2^-24 times smaller than that;
// the power is taken back in the scale of the scores.
//
// Operand layout of the instruction: lane l gives row (column) l % 16, eight k from 8 (l / 16) on; the result has
// column l % 16 and rows 4 (l / 16) .. + 3.  Any order of k will do that both operands share.
//   scores, transposed (tokens x rows):  lane l takes token l % 16 of a tile of sixteen and d / 4 channels in a row,
//     which are 16 bytes of its codes (8 at d = 64) and belong to one group, so one step and zero point.
//   output (rows x channels): the scores' result is the operand already (row l % 16, tokens 4 (l / 16) .. + 3 of two
//     tiles), and lane l takes for it, from the same eight tokens, the channels of its word l % 16, one of
//     the word's eight nibbles to an instruction.
#pragma once
#include <type_traits>

#include "kv4.h"
#include "layer_internal.h"

namespace mip {

typedef int v2i __attribute__((ext_vector_type(2)));
typedef int v4i __attribute__((ext_vector_type(4)));
typedef uint32_t v4u __attribute__((ext_vector_type(4)));

template <int D>
struct Kv4Shape {
  static constexpr int UNITS = D / 128 > 0 ? D / 128 : 1;   // of 128 channels
  static constexpr int WORDS = D >= 128 ? 4 : 2;            // a lane's words of a key, per unit
  static constexpr int NIBBLES = D >= 128 ? 8 : 4;          // a lane's channels of a value, per unit
  static constexpr int KEY_STEPS = UNITS * WORDS;           // instructions for the scores of a tile
  static constexpr int CHANNELS = UNITS * NIBBLES;          // instructions for the output of two tiles
  // channel of a query that meets nibble e of word w, unit u of lane group h
  __host__ __device__ static constexpr int key_channel(int u, int w, int h, int e) {
    return D >= 128 ? 128 * u + 32 * h + 8 * w + e : 16 * h + 8 * w + e;
  }
  // channel that instruction (u, j) gives column c of the output
  __host__ __device__ static constexpr int value_channel(int u, int j, int c) {
    return D >= 128 ? 128 * u + 8 * c + j : 4 * c + j;
  }
};

// Codes of a tile's keys and of the values of four of its tokens, and their pairs, as they come from memory.
template <int D>
struct Kv4Tile {
  using S = Kv4Shape<D>;
  uint32_t key[S::UNITS][S::WORDS];
  uint32_t key_pair[S::UNITS];
  v4u value[S::UNITS];
  v2i value_pair[S::UNITS];
};

// part: the head's part of the tile's page; first: the tile's first token in the page.  A lane's offsets
// in a part that do not depend on the tile are worked out once.
template <int D>
struct Kv4Reader {
  using S = Kv4Shape<D>;
  uint32_t key, key_pair[S::UNITS], value, value_pair[S::UNITS];  // bytes
  __device__ __forceinline__ Kv4Reader(int log_page, int lane) {
    const int c = lane & 15, h = lane >> 4, page = 1 << log_page;
    const Kv4Layout L(page, D);
    key = c * (D / 2) + h * (4 * S::WORDS);
    value = (uint32_t)L.values + 16 * (h * (D / 8) + (D >= 128 ? c : c >> 1));
#pragma unroll
    for (int u = 0; u < S::UNITS; ++u) {
      key_pair[u] = (uint32_t)L.key_pairs + 2 * (((D >= 128 ? 4 * u + h : h >> 1) << log_page) + c);
      value_pair[u] = (uint32_t)L.value_pairs + 2 * (((D >= 128 ? 4 * u + (c >> 2) : c >> 3) << log_page) + 4 * h);
    }
  }
  // COUNT words of a key from instruction `from` on (all of them of one unit), and its group's pair
  template <int COUNT>
  __device__ __forceinline__ void load_keys(const uint8_t *part, int first, int from, uint32_t (&w)[COUNT], uint32_t &pair) const {
    static_assert(COUNT == 1 || COUNT == 2 || COUNT == 4, "whole loads");
    const int u = from / S::WORDS;
    const uint8_t *k = part + first * (D / 2) + key + 64 * u + 4 * (from % S::WORDS);
    if constexpr (COUNT == 4) {
      const v4u x = *reinterpret_cast<const v4u *>(k);
#pragma unroll
      for (int i = 0; i < 4; ++i) w[i] = x[i];
    } else if constexpr (COUNT == 2) {
      const v2i x = *reinterpret_cast<const v2i *>(k);
      w[0] = x[0];
      w[1] = x[1];
    } else {
      w[0] = *reinterpret_cast<const uint32_t *>(k);
    }
    pair = *reinterpret_cast<const uint16_t *>(part + 2 * first + (u ? key_pair[S::UNITS - 1] : key_pair[0]));
  }
  __device__ __forceinline__ void load_values(const uint8_t *part, int first, int unit, v4u &w, v2i &pair) const {
    w = *reinterpret_cast<const v4u *>(part + first * (D / 2) + value + 256 * unit);
    pair = *reinterpret_cast<const v2i *>(part + 2 * first + (unit ? value_pair[S::UNITS - 1] : value_pair[0]));
  }
  __device__ __forceinline__ void load_values(const uint8_t *part, int first, v4u (&w)[S::UNITS], v2i (&pair)[S::UNITS]) const {
#pragma unroll
    for (int u = 0; u < S::UNITS; ++u) load_values(part, first, u, w[u], pair[u]);
  }
  __device__ __forceinline__ void load_keys(const uint8_t *part, int first, Kv4Tile<D> &t) const {
#pragma unroll
    for (int u = 0; u < S::UNITS; ++u) load_keys<S::WORDS>(part, first, u * S::WORDS, t.key[u], t.key_pair[u]);
  }
};

__device__ __forceinline__ v2h as_halves(uint32_t w) { return __builtin_bit_cast(v2h, w); }

// 1024 and 64 as float16 in both halves of a word, in registers the compiler knows nothing of: as literals beside
// their masks they would take an instruction of their own.
struct Kv4Exponents {
  uint32_t e1024, e64;
  __device__ __forceinline__ Kv4Exponents() : e1024(0x64006400u), e64(0x54005400u) { asm volatile("" : "+v"(e1024), "+v"(e64)); }
};

// Steps and negated zero points of two pairs (one in either half of `pairs`).
struct Kv4Scale {
  v2h s, z1024, z64;  // s, -(1024 + z), -(64 + z)
  Kv4Scale() = default;
  __device__ __forceinline__ explicit Kv4Scale(uint32_t pairs) {
    step(pairs);
    zero(pairs);
  }
  __device__ __forceinline__ void step(uint32_t pairs) { s = as_halves((pairs & 0x00ff00ffu) << 7); }
  __device__ __forceinline__ void zero(uint32_t pairs) {
    // z + 128 under the exponent of -1024, less the 128
    z1024 = as_halves(((pairs >> 8) & 0x00ff00ffu) ^ 0xe480e480u) + (_Float16)128.0f;
    z64 = z1024 + (_Float16)960.0f;
  }
  // nibbles at bits 0 and 16, and at bits 4 and 20
  __device__ __forceinline__ v2h low_sum(uint32_t w, const Kv4Exponents &k) const { return as_halves((w & 0x000f000fu) | k.e1024) + z1024; }
  __device__ __forceinline__ v2h high_sum(uint32_t w, const Kv4Exponents &k) const { return as_halves((w & 0x00f000f0u) | k.e64) + z64; }
  __device__ __forceinline__ v2h low(uint32_t w, const Kv4Exponents &k) const { return low_sum(w, k) * s; }
  __device__ __forceinline__ v2h high(uint32_t w, const Kv4Exponents &k) const { return high_sum(w, k) * s; }
};

__device__ __forceinline__ v8h join(v2h a, v2h b, v2h c, v2h d) {
  return v8h{a[0], a[1], b[0], b[1], c[0], c[1], d[0], d[1]};
}

// Operand of the scores from word w of a lane's keys: channels in the order 0 4 1 5 2 6 3 7.
__device__ __forceinline__ v8h key_operand(uint32_t w, const Kv4Scale &g, const Kv4Exponents &k) {
  const uint32_t x = w >> 8;
  return join(g.low(w, k), g.high(w, k), g.low(x, k), g.high(x, k));
}

// Operands of the output from the values of two tiles: instruction j of unit u, tokens in the order of the
// score's result.
template <int D>
struct Kv4Values {
  using S = Kv4Shape<D>;
  Kv4Scale g[4];
  uint32_t selector;  // bytes of the first pair of channels (d = 64: a lane takes half a word)
  const v4u a, b;
  __device__ __forceinline__ Kv4Values(v4u a, v4u b, v2i pa, v2i pb, int lane)
      : g{Kv4Scale(pa[0]), Kv4Scale(pa[1]), Kv4Scale(pb[0]), Kv4Scale(pb[1])},
        selector(0x0c040c00u + (D >= 128 ? 0u : (lane & 1) * 0x00020002u)), a(a), b(b) {}
  // channels 2 k and 2 k + 1 of the lane
  __device__ __forceinline__ void pair(int k, const Kv4Exponents &x, v8h &even, v8h &odd) const {
    const uint32_t sel = selector + k * 0x00010001u;
    const uint32_t x0 = __builtin_amdgcn_perm(a[1], a[0], sel), x1 = __builtin_amdgcn_perm(a[3], a[2], sel);
    const uint32_t x2 = __builtin_amdgcn_perm(b[1], b[0], sel), x3 = __builtin_amdgcn_perm(b[3], b[2], sel);
    even = join(g[0].low(x0, x), g[1].low(x1, x), g[2].low(x2, x), g[3].low(x3, x));
    odd = join(g[0].high(x0, x), g[1].high(x1, x), g[2].high(x2, x), g[3].high(x3, x));
  }
};

// Values that are no numbers: a step that is an infinity or NaN.  A product with them is none either, whatever it is multiplied
// by, also by the zero of a row that does not see them: where some row of a tile does not see all of its keys they are made
// zeros, and what sees them is made NaN afterwards, by a product of two patterns of ones and zeros.
//   no_number: ones, in float16, where a half of `pairs` has such a step; numbers_of: zeros there
__device__ __forceinline__ uint32_t no_step(uint32_t pairs) { return (((pairs & 0x00ff00ffu) + 0x00080008u) >> 8) & 0x00010001u; }
__device__ __forceinline__ uint32_t no_number(uint32_t pairs) { return no_step(pairs) * 0x3c00u; }
__device__ __forceinline__ uint32_t numbers_of(uint32_t pairs) { return pairs & ~(no_step(pairs) * 0xffffu); }
// what a lane's row sees of its eight tokens, two times four that are APART apart: `room` of them from the first on
template <int APART>
__device__ __forceinline__ v8h seen_tokens(int room) {
  v8h r;
#pragma unroll
  for (int e = 0; e < 8; ++e) r[e] = APART * (e / 4) + e % 4 < room ? (_Float16)1.0f : (_Float16)0.0f;
  return r;
}

__device__ __forceinline__ v4f multiply(v8h a, v8h b, v4f c) { return __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, 0, 0, 0); }

// bit e: row 4 (l / 16) + e sees something of the pattern's column l % 16
__device__ __forceinline__ uint32_t seen_of(v8h tokens, v8h pattern) {
  const v4f count = multiply(tokens, pattern, v4f{0.0f, 0.0f, 0.0f, 0.0f});
  uint32_t bits = 0;
#pragma unroll
  for (int e = 0; e < 4; ++e) bits |= count[e] > 0.0f ? 1u << e : 0;
  return bits;
}

// A request as the kernels see it: its rows of queries, its keys.  The device's numbers are cut to what the
// host was told, so that no value of theirs reads or writes outside the buffers.
struct Request {
  int64_t q0;       // first row of Q
  int queries, keys;
};
__device__ __forceinline__ Request request_of(const AttentionArgs &P, int r) {
  int64_t a = P.q_starts[r], b = P.q_starts[r + 1];
  a = a < 0 ? 0 : (a > P.q_rows ? P.q_rows : a);
  b = b < a ? a : (b > P.q_rows ? P.q_rows : b);
  int64_t queries = b - a, keys = P.kv_lengths[r];
  queries = queries > P.max_q ? P.max_q : queries;
  keys = keys < 0 ? 0 : (keys > P.max_kv ? P.max_kv : keys);
  return {a, (int)queries, (int)keys};
}
// Of so many keys those that the table can name.
__device__ __forceinline__ int named_of(const AttentionArgs &P, int keys) { return keys < P.named_kv ? keys : P.named_kv; }
// Where a range from `begin` on ends, of the tokens that are seen (begin + span can pass 31 bits where max_kv nearly does).
__device__ __forceinline__ int range_end(const AttentionArgs &P, int begin, int seen) {
  return P.partials && seen > begin && seen - begin > P.span ? begin + P.span : seen;
}
// Where a request's keys and values of one head lie.
struct Pages {
  typedef const __attribute__((address_space(4))) int32_t *table_ptr;
  table_ptr table;
  const uint8_t *head;  // the head's part of page 0
  uint32_t bytes;       // from page to page (at most 1024 heads of 294912)
  int last, pages, log_page;
  __device__ __forceinline__ Pages(const AttentionArgs &P, int r, int of, int64_t block)
      : table((table_ptr)(uintptr_t)(P.block_table + r * P.table_stride)), head(P.cache + of * block),
        bytes((uint32_t)(P.kv_heads * block)), last((int)P.table_stride - 1), pages(P.pages), log_page(P.log_page) {}
  // What the table says of a token's page: through the scalar cache (the table is not written while a kernel reads it),
  // and asked for well ahead of the page's own loads, which would otherwise begin with a wait for it.
  __device__ __forceinline__ int of(int token) const {
    const int at = __builtin_amdgcn_readfirstlane(token) >> log_page;
    return table[at < last ? at : last];
  }
  // whether it names a page there
  __device__ __forceinline__ bool named(int page, int token) const {
    return (unsigned)page < (unsigned)pages && (token >> log_page) <= last;
  }
  // the page, or one that is there to be read
  __device__ __forceinline__ const uint8_t *part(int page, bool named) const { return head + (uint64_t)(uint32_t)(named ? page : 0) * bytes; }
  __device__ __forceinline__ int within(int token) const { return token & ((1 << log_page) - 1); }
  // Whether a lane's row sees a key among so many tokens, none of them past the table: one whose page it names.
  __device__ __forceinline__ bool any_named(int tokens) const {
    for (int t = 0; t < tokens; t += 1 << log_page)
      if ((unsigned)table[t >> log_page] < (unsigned)pages) return true;
    return false;
  }
  // The same asked by a whole wave, 64 pages at a time: the first such token, or 2^31 - 1.
  __device__ __forceinline__ int first_named(int tokens) const {
    const int count = tokens > 0 ? ((tokens - 1) >> log_page) + 1 : 0;
    for (int from = 0; from < count; from += 64) {
      const int at = from + (int)__builtin_amdgcn_mbcnt_hi(~0u, __builtin_amdgcn_mbcnt_lo(~0u, 0u));
      const uint64_t found = __ballot(at < count && (unsigned)table[at < count ? at : 0] < (unsigned)pages);
      if (found) return (from + __builtin_ctzll(found)) << log_page;
    }
    return 0x7fffffff;
  }
};

// What a row's output is multiplied by that has no sum of p.  The sum is zero where the row sees no key, whose output is zeros, and
// where every score is minus infinity, which is also what masks one: those of an infinite query against keys of the other sign, or
// past float32.  That is no number, and here, once a row, is where the two are told apart.
__device__ __forceinline__ float of_no_sum(bool sees_a_key) { return sees_a_key ? __builtin_nanf("") : 0.0f; }

// A range's result for a row in scratch memory: D sums, then base and sum of the softmax.
template <int D>
constexpr int PARTIAL = D + 4;

constexpr float LOWEST = -3.402823466e38f;
// p is 2^(score - base) in float16, base the row's maximum less HEAD when it was last set: up to 2^LIMIT before
// the sums have to be rescaled, and not lost before it is 2^-31 of the largest.
constexpr float HEAD = 7.0f, LIMIT = 15.0f;

// Queries of a row as operands of the scores, and what a score is multiplied by to be a power of two's exponent.
// at: the row's first channel in Q; here: whether the row exists (else zeros).
template <int D, int TYPE>
__device__ __forceinline__ float load_queries(const AttentionArgs &P, int64_t at, bool here, int h, v8h (&q)[Kv4Shape<D>::KEY_STEPS]) {
  using S = Kv4Shape<D>;
  constexpr int ORDER[8] = {0, 4, 1, 5, 2, 6, 3, 7};
  v4f x[S::KEY_STEPS][2];
  float top = 0.0f;
#pragma unroll
  for (int i = 0; i < S::KEY_STEPS; ++i)
#pragma unroll
    for (int half = 0; half < 2; ++half) {
      x[i][half] = v4f{0.0f, 0.0f, 0.0f, 0.0f};
      if (here) x[i][half] = load_real4(P.Q, at + S::key_channel(i / S::WORDS, i % S::WORDS, h, 4 * half), TYPE);
#pragma unroll
      for (int e = 0; e < 4; ++e) top = fmaxf(top, fabsf(x[i][half][e]));
    }
  float by = 1.0f, back = 1.0f;
  if (TYPE == REAL_BF16) {
    top = fmaxf(top, __shfl_xor(top, 16));
    top = fmaxf(top, __shfl_xor(top, 32));
    int e = (__float_as_int(top) >> 23) - 127;  // top < 2^(e + 1)
    e = e < -100 ? -100 : e;
    by = __int_as_float((127 + 14 - e) << 23);
    back = __int_as_float((127 - 14 + e > 0 ? 127 - 14 + e : 1) << 23);
  }
#pragma unroll
  for (int i = 0; i < S::KEY_STEPS; ++i)
#pragma unroll
    for (int e = 0; e < 8; ++e) q[i][e] = (_Float16)(x[i][ORDER[e] / 4][ORDER[e] % 4] * by);
  // (never zero, which would make a NaN of a masked score)
  return fmaxf(P.scale * 1.4426950408889634f * back, 1.2e-38f);
}

// p of N times 32 keys for a wave's RT times sixteen rows (lane: row l % 16, tokens 4 (l / 16) .. + 3 of two tiles) from
// their scores, as operands of the output.  Only where a score has risen past LIMIT do the lanes of a row have
// to agree on a new base (top), and are its sums rescaled.  far: some base is so large that float32 holds no fractions of
// it.
template <int RT, int N, int SUMS>
__device__ __forceinline__ void weights(const v4f (&score)[RT][N][2], const float (&scale)[RT], float (&top)[RT], bool &far,
                                        v4f (&out)[RT][SUMS], int h, v8h (&p)[RT][N]) {
  float x[RT][N][8];
  // A fused multiply-add keeps what the product's rounding would lose, but against a base that is a rounded product
  // itself the difference of two large numbers is no longer zero where they are equal: past 2^20 both are rounded.
  auto exponents = [&](auto rounded) {
#pragma unroll
    for (int t = 0; t < RT; ++t)
#pragma unroll
      for (int n = 0; n < N; ++n)
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          const float s = score[t][n][e / 4][e % 4];
          x[t][n][e] = decltype(rounded)::value ? __fsub_rn(__fmul_rn(s, scale[t]), top[t]) : __builtin_fmaf(s, scale[t], -top[t]);
        }
  };
  if (far) exponents(std::true_type{});
  else exponents(std::false_type{});
  float largest = LOWEST;
#pragma unroll
  for (int t = 0; t < RT; ++t)
#pragma unroll
    for (int n = 0; n < N; ++n)
#pragma unroll
      for (int e = 0; e < 8; ++e) largest = fmaxf(largest, x[t][n][e]);
  if (__any(largest > LIMIT)) {
    far = false;
#pragma unroll
    for (int t = 0; t < RT; ++t) {
      largest = LOWEST;
#pragma unroll
      for (int n = 0; n < N; ++n)
#pragma unroll
        for (int e = 0; e < 8; ++e) largest = fmaxf(largest, __fmul_rn(score[t][n][e / 4][e % 4], scale[t]));
      largest = fmaxf(largest, __shfl_xor(largest, 16));
      largest = fmaxf(largest, __shfl_xor(largest, 32));
      const float moved = largest - HEAD > top[t] ? largest - HEAD : top[t];
      const float less = __builtin_amdgcn_exp2f(top[t] - moved);
      top[t] = moved;
      far |= __any(fabsf(moved) > 1048576.0f);
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const float by = __shfl(less, 4 * h + e);
#pragma unroll
        for (int j = 0; j < SUMS; ++j) out[t][j][e] *= by;
      }
    }
    if (far) exponents(std::true_type{});
    else exponents(std::false_type{});
  }
#pragma unroll
  for (int t = 0; t < RT; ++t)
#pragma unroll
    for (int n = 0; n < N; ++n)
#pragma unroll
      for (int e = 0; e < 8; ++e) p[t][n][e] = (_Float16)__builtin_amdgcn_exp2f(x[t][n][e]);
}

}  // namespace mip
