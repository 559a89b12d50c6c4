// Attention over the 4-bit cache for many rows of 64 or 128 channels: prompts and their chunks.
//
// A workgroup of eight waves takes 256 rows of one request and key head, 32 to a wave; tiles of 64 keys are brought
// from codes to float16 once for all of them, each wave its share, and lie in LDS as the operands of
// v_mfma_f32_32x32x16_f16, 1 KB each, so that every read is sixteen bytes a lane in a row.
//
// A SIMD has two waves, one of either half of the workgroup, and the halves run half a tile apart, held there by a
// barrier after every half: while one wave keeps the matrix unit busy (output of a tile, scores of the next), the other works
// out the weights of its tile.  A wave's share of the codes to come is unpacked between the matrix instructions, two or three
// vector instructions after each: beside the weights it made that half twice as long as this one.  The matrix half goes before
// the other where both could issue (290 us instead of 304).
//
// 2048 queries of 32 heads over 8192 keys of 8, 128 channels: 255 to 290 us by the card, 830 to 940 TFLOP/s (338 with the codes
// beside the weights, 380 with 16 x 16 x 32 instructions and 128 rows).  What bounds it is issue: a wave and tile takes 36 matrix
// instructions of 32 clocks, some 240 vector and 140 scalar ones, so a half takes about 2000 clocks, not the 1152 of the
// matrix unit; and the first rows' workgroups, which see a quarter fewer keys, leave their units an eighth of the time.
// In bfloat16 the scale of the scores is multiplied into the queries (rounded to float16's eleven bits, three more than
// theirs), and the base of the softmax is one more term of their sums: they come out as exponents.
//
// Layout: lane l of an operand gives row (column) l % 32 and eight k from 8 (l / 32) on; the result has column
// l % 32 and rows 8 (v / 4) + 4 (l / 32) + v % 4 in its sixteen registers v.
//   scores, transposed: token l % 32 of a block of 32, half of its channels in a row to either half of the wave;
//   output: a score's result is the operand already (registers 0 .. 7 and 8 .. 15 the two sixteens of a block), and
//     lane l takes for it, from the same eight tokens, half (d = 64: a quarter) of a word of codes.
#include "attention_kv4.h"

namespace mip {

namespace {

typedef float v16f __attribute__((ext_vector_type(16)));

__device__ __forceinline__ v16f multiply32(v8h a, v8h b, v16f c) { return __builtin_amdgcn_mfma_f32_32x32x16_f16(a, b, c, 0, 0, 0); }
__device__ __forceinline__ v16f all16(float x) { return v16f{x, x, x, x, x, x, x, x, x, x, x, x, x, x, x, x}; }

// ONE: a tile lies in one page (pages of 64 tokens or more).
template <int D, int TYPE, bool ONE>
__global__ __launch_bounds__(512, 2) void attention_wide_kernel(AttentionArgs P) {
  constexpr int ROWS = 256, TILE = 64;
  constexpr int KEY_STEPS = D / 16, KEYS = 2 * KEY_STEPS;      // operands of a block's, of a tile's scores
  constexpr int COLUMNS = D / 32, VALUES = 4 * COLUMNS;        // of sixteen tokens', of a tile's output
  constexpr int KEY_EACH = KEY_STEPS / 4, PARTS = COLUMNS / 2;  // a wave's operands of keys; waves to sixteen tokens of values
  constexpr bool FOLD = TYPE == REAL_BF16;
  constexpr float FAR = FOLD ? 32768.0f : 1048576.0f;  // past what float16 holds, or float32 with fractions
  extern __shared__ __attribute__((aligned(16))) uint8_t smem[];
  // values that are no numbers: patterns of tile i % 4's sixteens, and i + 1 for a sixteen that has one
  __shared__ __attribute__((aligned(16))) uint8_t none[4][4][1024];
  __shared__ int has_none[4][4];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int c = lane & 31, h = lane >> 5;
  const int range = blockIdx.x % P.ranges, r = blockIdx.z;
  // the last rows of a prompt see the most keys: they begin first
  const int of_all = P.first + (int)(gridDim.x / P.ranges) - 1 - (int)(blockIdx.x / P.ranges);
  const int head = of_all % P.kv_heads, row0 = of_all / P.kv_heads * ROWS;
  // a wave's share: keys of block `wave % 2`, a quarter of their channels; values of the sixteen `wave % 4`
  const int key_block = wave & 1, key_part = wave >> 1, unit = wave & 3, value_part = wave >> 2;
  const int begin = range * P.span;
  const Kv4Layout L(1 << P.log_page, D);
  const Pages pages(P, r, head, L.block);
  int key_page[2] = {pages.of(ONE ? begin : begin + 32 * key_block), pages.of(begin + 32 * key_block + 16)};
  int value_page = pages.of(begin + 16 * unit);
  const Request req = request_of(P, r);
  const int rows = req.queries * P.shared;
  if (row0 >= rows) return;
  const int before = req.keys - req.queries + 1;  // keys that the first query sees
  auto sees_of = [&](int row) { return before + row / P.shared; };
  const int seen = named_of(P, sees_of(row0 + ROWS < rows ? row0 + ROWS - 1 : rows - 1));
  const int end = range_end(P, begin, seen);
  if (range > 0 && begin >= end) return;

  // queries: lane's row, channels D / 2 h + 8 i + 0 4 1 5 2 6 3 7 in operand i
  // (a row that is none sees what the last one does, so that it needs no mask, and is not written)
  const int wave_row = row0 + 32 * wave;
  const bool here = wave_row + c < rows;
  const int row = here ? wave_row + c : rows - 1, query = row / P.shared, sees = before + query;
  // the fewest and the most keys that a row of the wave sees
  const int fewest = wave_row < rows ? sees_of(wave_row) : 0;
  const int most = wave_row < rows ? sees_of((wave_row + 32 < rows ? wave_row + 32 : rows) - 1) : 0;
  v8h q[KEY_STEPS];
  float back;  // what a score is multiplied by to be an exponent
  bool folded = FOLD;
  {
    constexpr int ORDER[8] = {0, 4, 1, 5, 2, 6, 3, 7};
    const int64_t at = (req.q0 + query) * P.ldq + (int64_t)(head * P.shared + (row - query * P.shared)) * D + D / 2 * h;
    float x[KEY_STEPS][8], most_of_row = 0.0f;
#pragma unroll
    for (int i = 0; i < KEY_STEPS; ++i) {
#pragma unroll
      for (int e = 0; e < 8; ++e) x[i][e] = 0.0f;
      if (here) load_real8<TYPE>(P.Q, at + 8 * i, x[i]);
#pragma unroll
      for (int e = 0; e < 8; ++e) most_of_row = fmaxf(most_of_row, fabsf(x[i][e]));
    }
    const float whole = P.scale * 1.4426950408889634f;
    float by = 1.0f;
    back = whole;
    if (FOLD) {
      most_of_row = fmaxf(most_of_row, __shfl_xor(most_of_row, 32));
      const float scaled = most_of_row * whole;
      // (outside float16's better part: a power of two instead, and the scale afterwards)
      folded = !__any(!(scaled == 0.0f || (scaled >= 0.0625f && scaled < 32768.0f)));
      if (folded) {
        by = whole;
        back = 1.0f;
      } else {
        int e = (__float_as_int(most_of_row) >> 23) - 127;
        e = e < -100 ? -100 : e;
        by = __int_as_float((127 + 14 - e) << 23);
        back = whole * __int_as_float((127 - 14 + e > 0 ? 127 - 14 + e : 1) << 23);
      }
    }
    back = fmaxf(back, 1.2e-38f);  // (never zero, which would make a NaN of a masked score)
#pragma unroll
    for (int i = 0; i < KEY_STEPS; ++i)
#pragma unroll
      for (int e = 0; e < 8; ++e) q[i][e] = (_Float16)(x[i][ORDER[e]] * by);
  }
  float base = LOWEST;
  bool far = true;  // some base is past FAR (the first is)
  v16f out[COLUMNS + 1];  // the last: sums of p
#pragma unroll
  for (int j = 0; j <= COLUMNS; ++j) out[j] = all16(0.0f);
  // the base, taken off by one more instruction of the scores where they come out as exponents: in three parts, which
  // hold all bits of it
  v8h less_base = {};
  auto set_less_base = [&](bool on) {
    const float x = on && h == 0 ? -base : 0.0f;
    const _Float16 hi = (_Float16)x, mid = (_Float16)(x - (float)hi);
    less_base[0] = hi;
    less_base[1] = mid;
    less_base[2] = (_Float16)(x - (float)hi - (float)mid);
  };
  const _Float16 one = (_Float16)1.0f;
  const v8h ones = {one, one, one, one, one, one, one, one};

  // a lane's places in a page: offsets that do not depend on the tile
  const int key_group = D == 128 ? 2 * h + (key_part >> 1) : h, word = D == 128 ? c >> 1 : c >> 2;
  const int key_token = ONE ? 32 * key_block + c : c & 15, value_token = ONE ? 16 * unit : 0;
  const uint32_t key_at = (uint32_t)(key_token * (D / 2) + (D / 4) * h + 4 * KEY_EACH * key_part);
  const uint32_t key_pair_at = (uint32_t)(L.key_pairs + 2 * ((key_group << P.log_page) + key_token));
  const uint32_t value_at = (uint32_t)(L.values + value_token * (D / 2) + 16 * (h * (D / 8) + word));
  const uint32_t value_pair_at = (uint32_t)(L.value_pairs + 2 * (((word >> 2) << P.log_page) + value_token + 4 * h));
  // the byte of a value's word that the lane's channels are in, of two tokens
  const uint32_t byte = 0x0c040c00u + (uint32_t)(D == 128 ? 2 * (c & 1) + value_part : c & 3) * 0x00010001u;
  const Kv4Exponents exponents;
  const int tiles = end > begin ? (end - begin + TILE - 1) / TILE : 0;
  // whether the table names all the pages that are read here (if not, every tile asks it again)
  bool whole = true;
  if (tid < 16) has_none[tid >> 2][tid & 3] = 0;
  for (int i = (begin >> P.log_page) + tid; i < (end + (1 << P.log_page) - 1) >> P.log_page; i += 512)
    whole = whole && pages.named(pages.table[i < pages.last ? i : pages.last], i << P.log_page);
  whole = __syncthreads_and(whole);
  // (past the last tile, the last again: what it becomes is not used)
  auto first_of = [&](int tile) { return begin + (tile < tiles ? tile : tiles - 1) * TILE; };
  uint32_t key[KEY_EACH], key_pair;
  v4u value[2];
  v2i value_pair[2];
  int tile_room = 0, value_room = 16;  // tokens that there are from the tile's first on, and of the sixteen
  struct Place { const uint8_t *codes, *pairs; } keys_at = {}, keys_at_16 = {}, values_at = {};
  auto place = [&](int page, int token, int &room) {
    const int in = pages.within(token);
    const bool exists = pages.named(page, token);
    const uint8_t *part = pages.part(page, exists);
    room = exists ? end - token : 0;
    return Place{part + in * (D / 2), part + 2 * in};
  };
  auto place_keys = [&](int tile) {
    const int first = first_of(tile) + (ONE ? 0 : 32 * key_block);
    keys_at = place(key_page[0], first, tile_room);
    if (!ONE) keys_at_16 = place(key_page[1], first + 16, tile_room);
  };
  auto fetch_keys = [&] {
    const uint8_t *codes = keys_at.codes, *pairs = keys_at.pairs;
    if (!ONE) {
      codes = c & 16 ? keys_at_16.codes : codes;
      pairs = c & 16 ? keys_at_16.pairs : pairs;
    }
    if constexpr (KEY_EACH == 2) {
      const v2i w = *reinterpret_cast<const v2i *>(codes + key_at);
      key[0] = w[0];
      key[1] = w[1];
    } else {
      key[0] = *reinterpret_cast<const uint32_t *>(codes + key_at);
    }
    key_pair = *reinterpret_cast<const uint16_t *>(pairs + key_pair_at);
  };
  auto place_values = [&](int tile) {
    if constexpr (ONE) {  // (the place of the keys that were the last to be placed)
      values_at = keys_at;
      value_room = tile_room - 16 * unit;
    } else {
      values_at = place(value_page, first_of(tile) + 16 * unit, value_room);
    }
  };
  auto fetch_values = [&] {
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      value[i] = *reinterpret_cast<const v4u *>(values_at.codes + value_at + i * (4 * D));
      value_pair[i] = *reinterpret_cast<const v2i *>(values_at.pairs + value_pair_at + 16 * i);
    }
  };
  // what lies behind the last key, and in pages that are none, is no number: a step of zero makes it zero
  auto cut_values = [&](int tile) {
    if (value_room < 16) {
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const int exist = value_room - 8 * i - 4 * h;
        if (exist < 4) value_pair[i][1] &= exist < 3 ? 0 : 0x0000ffff;
        if (exist < 2) value_pair[i][0] &= exist < 1 ? 0 : 0x0000ffff;
      }
    }
    if (tile < tiles && begin + tile * TILE + TILE > sees_of(row0)) {  // some row may not see all of its keys
      v2i &a = value_pair[0], &b = value_pair[1];
      if (__any(no_step(a[0]) | no_step(a[1]) | no_step(b[0]) | no_step(b[1]))) {  // (two waves find and write the same)
        has_none[tile & 3][unit] = tile + 1;
        *reinterpret_cast<v4u *>(none[tile & 3][unit] + 16 * lane) = v4u{no_number(a[0]), no_number(a[1]), no_number(b[0]), no_number(b[1])};
        a = v2i{(int)numbers_of(a[0]), (int)numbers_of(a[1])};
        b = v2i{(int)numbers_of(b[0]), (int)numbers_of(b[1])};
      }
    }
  };
  // Beside tile `tile`: the operands of its values and of the keys after it, from the codes that were fetched, in slices
  // of two or three instructions, which is what goes between two of the matrix unit.  (A code is multiplied one slice after
  // the zero point is added: packed, the two would need a pause between them.)
  constexpr int KEY_SLICES = 3 + 4 * KEY_EACH, SLICES = KEY_SLICES + 11 + 4 * PARTS;
  Kv4Scale g[5];
  uint32_t x[4];
  v2h part[4];
  auto slice = [&](int tile, int i) {
    if (i < KEY_SLICES) {
      if (i == 0) g[4].step(key_pair * 0x00010001u);
      if (i == 1) g[4].zero(key_pair * 0x00010001u);
      const int of = (i - 2) / 4, e = (i - 2) & 3;
      if (i > 2) part[(e + 3) & 3] *= g[4].s;
      if (i > 2 && e == 0) {
        uint8_t *to = smem + (((tile + 1) & 1) * KEYS + key_block * KEY_STEPS + key_part * KEY_EACH + of - 1) * 1024 + 16 * lane;
        *reinterpret_cast<v8h *>(to) = join(part[0], part[1], part[2], part[3]);
      }
      if (i >= 2 && of < KEY_EACH) {
        const uint32_t w = key[of] >> (e & 2 ? 8 : 0);
        part[e] = e & 1 ? g[4].high_sum(w, exponents) : g[4].low_sum(w, exponents);
      }
    } else if (i < KEY_SLICES + 2) {
      const int of = i - KEY_SLICES;
      x[2 * of] = __builtin_amdgcn_perm(value[of][1], value[of][0], byte);
      x[2 * of + 1] = __builtin_amdgcn_perm(value[of][3], value[of][2], byte);
      if (PARTS == 1) {  // (one operand to a wave: of the upper four bits for the last four)
        x[2 * of] >>= 4 * value_part;
        x[2 * of + 1] >>= 4 * value_part;
      }
    } else if (i < KEY_SLICES + 10) {
      const int e = (i - KEY_SLICES - 2) / 2;
      if ((i - KEY_SLICES) & 1) g[e].zero(value_pair[e / 2][e & 1]);
      else g[e].step(value_pair[e / 2][e & 1]);
    } else {
      const int from = i - KEY_SLICES - 10, of = from / 4, e = from & 3;
      if (from > 0) part[(e + 3) & 3] *= g[(e + 3) & 3].s;
      if (from > 0 && e == 0) {
        uint8_t *to = smem + (2 * KEYS + (tile & 1) * VALUES + unit * COLUMNS + PARTS * value_part + of - 1) * 1024 + 16 * lane;
        *reinterpret_cast<v8h *>(to) = join(part[0], part[1], part[2], part[3]);
      }
      if (of < PARTS) part[e] = of ? g[e].high_sum(x[e], exponents) : g[e].low_sum(x[e], exponents);
    }
  };
  // the pages of the tiles that come after those: asked for at the start of a half, since its end waits for them
  int next_key_page[2] = {0, 0}, next_value_page = 0;
  auto ask = [&](int of_keys, int of_values) {
    if constexpr (ONE) {
      next_key_page[0] = pages.of(first_of(of_keys));
    } else {
#pragma unroll
      for (int i = 0; i < 2; ++i) next_key_page[i] = pages.of(first_of(of_keys) + 32 * key_block + 16 * i);
      next_value_page = pages.of(first_of(of_values) + 16 * unit);
    }
    __builtin_amdgcn_sched_barrier(0);
  };
  auto told = [&] {
    key_page[0] = next_key_page[0];
    key_page[1] = next_key_page[1];
    value_page = next_value_page;
  };

  v16f score[2];
  v8h p[4];
  // Output of the values in one stage and scores of the keys in another, as one run of operands: each is read LOOK
  // before it is used, and beside(0), beside(1) .. go between them, in this order and no other (left to itself the compiler
  // reads two operands and waits for them).
  auto multiply_tiles = [&](auto values_tag, auto keys_tag, int value_stage, int key_stage, auto beside) {
    constexpr int V = decltype(values_tag)::value ? VALUES : 0, N = V + (decltype(keys_tag)::value ? KEYS : 0), LOOK = 4;
    const uint8_t *values = smem + (2 * KEYS + value_stage * VALUES) * 1024 + 16 * lane;
    const uint8_t *keys = smem + key_stage * (KEYS * 1024) + 16 * lane;
    auto read = [&](int i) {
      return *reinterpret_cast<const v8h *>(i < V ? values + i * 1024 : keys + ((i - V) / 2 + ((i - V) & 1) * KEY_STEPS) * 1024);
    };
    v8h ring[LOOK];
    // (two at a time and the second first, so that one wait is enough for both)
    auto read_two = [&](int i) {
      ring[(i + 1) % LOOK] = read(i + 1);
      __builtin_amdgcn_sched_barrier(0);
      ring[i % LOOK] = read(i);
      __builtin_amdgcn_sched_barrier(0);
    };
#pragma unroll
    for (int i = 0; i < LOOK; i += 2) read_two(i);
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const v8h operand = ring[i % LOOK];
      if (i < V) {
        const int u = i / COLUMNS, j = i % COLUMNS;
        if (j == 0) out[COLUMNS] = multiply32(p[u], ones, out[COLUMNS]);
        out[j] = multiply32(p[u], operand, out[j]);
      } else {
        const int b = (i - V) & 1, w = (i - V) / 2;
        if (w == 0) score[b] = FOLD ? multiply32(ones, less_base, all16(0.0f)) : all16(0.0f);
        score[b] = multiply32(operand, q[w], score[b]);
      }
      if (i % 2 && i - 1 + LOOK < N) read_two(i - 1 + LOOK);
#pragma unroll
      for (int k = i * SLICES / N; k < (i + 1) * SLICES / N; ++k) beside(k);
      __builtin_amdgcn_sched_barrier(0);
    }
  };
  // NaN in the rows that see a value of the tile that is no number
  auto mark_none = [&](int tile) {
    if (begin + tile * TILE + TILE <= sees_of(row0)) return;  // (the others' keys count too: what is made zero is for all)
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      if (__builtin_amdgcn_readfirstlane(has_none[tile & 3][u]) != tile + 1) continue;
      const v8h tokens = seen_tokens<8>(sees - (begin + tile * TILE + 16 * u + 4 * h));
      const v8h pattern = *reinterpret_cast<const v8h *>(none[tile & 3][u] + 16 * lane);
      const v16f count = multiply32(tokens, pattern, all16(0.0f));
#pragma unroll
      for (int v = 0; v < 16; ++v)
#pragma unroll
        for (int j = 0; j < COLUMNS; ++j) out[j][v] = count[v] > 0.0f ? __builtin_nanf("") : out[j][v];
    }
  };
  auto mask_scores = [&](int tile) {
    const int token = begin + tile * TILE;
    if (token + TILE > fewest || !whole) {
      int sees_of_it[4] = {sees, sees, sees, sees};  // of the tile's sixteens
      if (!whole) {
#pragma unroll
        for (int i = 0; i < 4; ++i) sees_of_it[i] = pages.named(pages.of(token + 16 * i), token + 16 * i) ? sees : 0;
      }
#pragma unroll
      for (int b = 0; b < 2; ++b)
#pragma unroll
        for (int v = 0; v < 16; ++v) {
          const int room = sees_of_it[2 * b + v / 8] - (token + 32 * b + 4 * h);
          score[b][v] = 8 * (v / 4) + v % 4 < room ? score[b][v] : -__builtin_inff();
        }
    }
  };
  // Scores to exponents (in place), their base moved where one has risen past LIMIT, and p from them.
  auto weights = [&] {
    auto each = [&](auto change) {
#pragma unroll
      for (int b = 0; b < 2; ++b)
#pragma unroll
        for (int v = 0; v < 16; ++v) score[b][v] = change(score[b][v]);
    };
    auto largest = [&] {
      float m = LOWEST;
#pragma unroll
      for (int b = 0; b < 2; ++b)
#pragma unroll
        for (int v = 0; v < 16; ++v) m = fmaxf(m, score[b][v]);
      return m;
    };
    float less = 1.0f;
    bool moved = false;
    if (far) {
      // (fused, the multiplication would keep what its rounding loses, but against a base that is a rounded product itself the
      // difference of two large numbers is no longer zero where they are equal)
      each([&](float s) { return __fmul_rn(s, back); });
      float m = largest();
      if (__any(m - base > LIMIT)) {
        m = fmaxf(m, __shfl_xor(m, 32)) - HEAD;
        m = m > base ? m : base;
        less = __builtin_amdgcn_exp2f(base - m);
        base = m;
        moved = true;
      }
      each([&](float s) { return __fsub_rn(s, base); });
      far = __any(fabsf(base) > FAR) || (FOLD && !folded);
      if (FOLD) set_less_base(!far);  // from the next tile on
    } else {
      if (!FOLD) each([&](float s) { return __builtin_fmaf(s, back, -base); });
      float m = largest();
      if (__any(m > LIMIT)) {
        m = fmaxf(m, __shfl_xor(m, 32));
        const float rise = m > HEAD ? m - HEAD : 0.0f;
        less = __builtin_amdgcn_exp2f(-rise);
        base += rise;
        each([&](float s) { return s - rise; });
        moved = true;
        far = __any(fabsf(base) > FAR);
        if (FOLD) set_less_base(!far);
      }
    }
    if (moved) {
#pragma unroll
      for (int v = 0; v < 16; ++v) {
        const float by = __shfl(less, 8 * (v / 4) + 4 * h + v % 4);
#pragma unroll
        for (int j = 0; j <= COLUMNS; ++j) out[j][v] *= by;
      }
    }
#pragma unroll
    for (int u = 0; u < 4; ++u)
#pragma unroll
      for (int e = 0; e < 8; ++e) p[u][e] = (_Float16)__builtin_amdgcn_exp2f(score[u / 2][8 * (u % 2) + e]);
  };
  // (not __syncthreads: loads from memory stay in flight across it)
  auto half_done = [] { asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory"); };

  // Half h of the first four waves is the output of tile h / 2 - 1 and the scores of tile h / 2 where h is even, the weights of
  // tile h / 2 where it is odd; the other four are one half behind.  Beside the former, which leaves a wave four in five of
  // the instructions it can issue, go the codes: the values of tile i and the keys of tile i + 1, read from 2 i + 2 on,
  // are written in the halves 2 i and 2 i + 1, after the last reads of the tiles whose stages they take.
  if (tiles > 0) {
    ask(1, 1);
    place_keys(0);
    fetch_keys();
    place_values(0);
    fetch_values();
#pragma unroll
    for (int i = 0; i < KEY_SLICES; ++i) slice(-1, i);
    told();
    place_keys(1);
    fetch_keys();
    ask(2, 1);
    cut_values(0);
    half_done();
    told();
    if (wave >> 2) half_done();
    for (int tile = 0; tile < tiles; ++tile) {
      const bool sees_any = begin + tile * TILE < most;
      auto beside = [&](int i) { slice(tile, i); };
      __builtin_amdgcn_s_setprio(1);
      if (sees_any && tile > 0) {
        multiply_tiles(std::true_type{}, std::true_type{}, (tile - 1) & 1, tile & 1, beside);
      } else if (sees_any) {
        multiply_tiles(std::false_type{}, std::true_type{}, 0, 0, beside);
      } else {
#pragma unroll
        for (int i = 0; i < SLICES; ++i) beside(i);
      }
      __builtin_amdgcn_s_setprio(0);
      half_done();
      place_values(tile + 1);
      fetch_values();
      __builtin_amdgcn_sched_barrier(0);
      if (sees_any) mask_scores(tile);
      place_keys(tile + 2);
      fetch_keys();
      ask(tile + 3, tile + 2);  // (behind the scores' one read of LDS, whose wait would include it)
      if (sees_any) weights();
      cut_values(tile + 1);
      told();
      half_done();
      // (the rows of a wave that see nothing of the next tile end here)
      if (sees_any) mark_none(tile);
      if (sees_any && (tile + 1 == tiles || begin + (tile + 1) * TILE >= most))
        multiply_tiles(std::true_type{}, std::false_type{}, tile & 1, 0, [](int) {});
    }
    if (!(wave >> 2)) half_done();
  }

  float nothing = 0.0f;  // of a row without a sum (lane: row l % 32)
  bool no_sum = false;
#pragma unroll
  for (int v = 0; v < 16; ++v) no_sum = no_sum || out[COLUMNS][v] == 0.0f;
  if (!P.partials && __any(no_sum)) nothing = of_no_sum(pages.first_named(seen) < sees);
#pragma unroll
  for (int v = 0; v < 16; ++v) {
    const int row_in = 8 * (v / 4) + 4 * h + v % 4, at_row = wave_row + row_in;
    const float l = out[COLUMNS][v], m = __shfl(base, row_in), none_of = __shfl(nothing, row_in);
    if (at_row >= rows) continue;
    const int of = at_row / P.shared, within = at_row - of * P.shared;
    float o[COLUMNS];
#pragma unroll
    for (int j = 0; j < COLUMNS; ++j) o[j] = out[j][v];
    if (P.partials) {
      const int64_t row_of_all = ((req.q0 + of) * P.kv_heads + head) * P.shared + within;
      float *to = P.partials + (row_of_all * P.ranges + range) * PARTIAL<D>;
      if (c == 0) *reinterpret_cast<v2f *>(to + D) = v2f{m, l};
#pragma unroll
      for (int j = 0; j < COLUMNS; j += 2) *reinterpret_cast<v2f *>(to + COLUMNS * c + j) = v2f{o[j], o[j + 1]};
    } else {
      const float by = l != 0.0f ? 1.0f / l : none_of;
      const int64_t at = (req.q0 + of) * P.ldo + (int64_t)(head * P.shared + within) * D + COLUMNS * c;
      if constexpr (COLUMNS == 4) {
        store_real4(P.O, at, TYPE, v4f{o[0], o[1], o[2], o[3]} * by);
      } else {
#pragma unroll
        for (int j = 0; j < COLUMNS; ++j) store_real(P.O, at + j, TYPE, o[j] * by);
      }
    }
  }
}

}  // namespace

template <bool ONE>
static AttentionKernel wide_of(int head_dim, int type) {
  if (head_dim == 64) return type == REAL_BF16 ? attention_wide_kernel<64, REAL_BF16, ONE> : attention_wide_kernel<64, REAL_F16, ONE>;
  return type == REAL_BF16 ? attention_wide_kernel<128, REAL_BF16, ONE> : attention_wide_kernel<128, REAL_F16, ONE>;
}

AttentionKernel attention_wide(int head_dim, int type, int log_page) {
  return log_page >= 6 ? wide_of<true>(head_dim, type) : wide_of<false>(head_dim, type);
}

}  // namespace mip
