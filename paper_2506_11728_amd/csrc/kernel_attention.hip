// Attention over the 4-bit cache: the kernel for few rows (single tokens and drafted ones), the one for many
// (prompts and their chunks), and the one that joins ranges of keys.
//
// Few rows: bound by the cache's bytes where there are enough keys (one query of 32 heads over 131001 keys of 8: 34 us from memory,
// 151 MB at 4.4 TB/s, and 31 where they lie in the last-level cache; joining its 128 ranges 4.3 more), by unequal requests where
// those differ (32 of 174 to 8192 keys, 3 % more bytes: 42 us; the vector instructions that make float16 of the codes are
// 20 us of issue in either), and by first loads and last sums in short calls (301 keys 6.0 us).  Ranges are cut by the bound
// max_kv and rows by max_q: 4096 keys take 9.6 us under a bound of 4096 and 15 under one of 131072.  A workgroup takes the rows of one request and key head (16 or 32 of them; more rows,
// more workgroups, which find the codes in L2) and a range of its keys; its four waves take steps of 32 keys in turn, each with a
// running maximum, sum and output of its own, which meet in LDS at the end.  Where requests and heads are too few to
// occupy the device the keys are cut into ranges, and a second, small kernel joins them.
#include "attention_kv4.h"

namespace mip {

namespace {

constexpr int WAVES = 4, STEP = 32;  // keys of a wave's step: two tiles

template <int D, int TYPE, int RT>
__global__ __launch_bounds__(64 * WAVES, D <= 128 && RT == 1 ? 4 : (D == 256 && RT == 2 ? 1 : 2)) void attention_rows_kernel(AttentionArgs P) {
  using S = Kv4Shape<D>;
  extern __shared__ __attribute__((aligned(16))) uint8_t smem[];
  auto sums = reinterpret_cast<float (*)[16][D + 4]>(smem);  // a wave's: sixteen rows
  __shared__ float tops[WAVES][16], totals[WAVES][16];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int c = lane & 15, h = lane >> 4;
  // (heads before ranges: neighbours go to different dies, and the ranges of short requests are empty from some on)
  const int here = gridDim.x / P.ranges, range = blockIdx.x / here, of_all = P.first + blockIdx.x % here, r = blockIdx.z;
  const int head = of_all % P.kv_heads, tile = of_all / P.kv_heads;
  // (the first pages are on their way with the request's numbers)
  const int begin = range * P.span, mine = begin + wave * STEP;
  const Pages pages(P, r, head, Kv4Layout(1 << P.log_page, D).block);
  int page[2] = {pages.of(mine), pages.of(mine + 16)};
  const Request req = request_of(P, r);
  const int rows = req.queries * P.shared, row0 = tile * (16 * RT);
  if (row0 >= rows) return;
  // keys that any row of the tile sees
  const int last_query = (row0 + 16 * RT < rows ? row0 + 16 * RT - 1 : rows - 1) / P.shared;
  const int seen = named_of(P, req.keys - req.queries + last_query + 1);
  const int end = range_end(P, begin, seen);
  if (range > 0 && begin >= end) return;

  v8h q[RT][S::KEY_STEPS];
  float scale[RT], top[RT];
  bool far = true;  // (the first base is)
  int sees[RT];  // keys that the row sees
  v4f out[RT][S::CHANNELS + 1];  // the last: sums of p
  uint32_t lost = 0;  // four bits to a row tile and unit: rows that have seen a value that is no number
  int fewest = 0x7fffffff;
#pragma unroll
  for (int t = 0; t < RT; ++t) {
    // (a row that is none sees what the last one does, so that it needs no mask, and is not written)
    const int of_row = row0 + 16 * t + c, row = of_row < rows ? of_row : rows - 1, query = row / P.shared;
    const int64_t at = (req.q0 + query) * P.ldq + (int64_t)(head * P.shared + (row - query * P.shared)) * D;
    scale[t] = load_queries<D, TYPE>(P, at, of_row < rows, h, q[t]);
    sees[t] = req.keys - req.queries + query + 1;
    const int least = row0 + 16 * t < rows ? req.keys - req.queries + (row0 + 16 * t) / P.shared + 1 : fewest;
    fewest = least < fewest ? least : fewest;
    top[t] = LOWEST;
#pragma unroll
    for (int j = 0; j <= S::CHANNELS; ++j) out[t][j] = v4f{0.0f, 0.0f, 0.0f, 0.0f};
  }

  const _Float16 one = (_Float16)1.0f;
  const v8h ones = {one, one, one, one, one, one, one, one};
  const Kv4Exponents exponents;
  const Kv4Reader<D> reader(P.log_page, lane);
  const int steps = end > begin ? (end - begin + STEP - 1) / STEP : 0;
  // The codes of two tiles.  The keys of a wave's next step are on their way from its scores on, the values from its output
  // on: where they are needed the registers are free, and four waves to a SIMD cover the rest.
  Kv4Tile<D> now[2];
  bool named[2] = {false, false}, known[2];  // the table names a page for the tile
  const uint8_t *at[2];
  int in[2];
  auto fetch_keys = [&](int step) {
    const int token = begin + step * STEP;
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      const int first = token + 16 * u;
      named[u] = pages.named(page[u], first);
      at[u] = pages.part(page[u], named[u]);
      in[u] = pages.within(first);
      reader.load_keys(at[u], in[u], now[u]);
      page[u] = pages.of(first + WAVES * STEP);  // for the step after
    }
  };
  auto fetch_values = [&] {
#pragma unroll
    for (int u = 0; u < 2; ++u) reader.load_values(at[u], in[u], now[u].value, now[u].value_pair);
  };
  if (wave < steps) {
    fetch_keys(wave);
    fetch_values();
  }
  for (int step = wave; step < steps; step += WAVES) {
    known[0] = named[0];
    known[1] = named[1];
    const int token = begin + step * STEP;

    v4f score[RT][1][2];
#pragma unroll
    for (int u = 0; u < 2; ++u) {
#pragma unroll
      for (int t = 0; t < RT; ++t) score[t][0][u] = v4f{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
      for (int n = 0; n < S::UNITS; ++n) {
        const Kv4Scale g(now[u].key_pair[n] * 0x00010001u);
#pragma unroll
        for (int w = 0; w < S::WORDS; ++w) {
          const v8h k = key_operand(now[u].key[n][w], g, exponents);
#pragma unroll
          for (int t = 0; t < RT; ++t) score[t][0][u] = multiply(k, q[t][n * S::WORDS + w], score[t][0][u]);
        }
      }
    }
    if (step + WAVES < steps) fetch_keys(step + WAVES);
    if (token + STEP > fewest || !known[0] || !known[1]) {  // wave-uniform: some row does not see all of them
#pragma unroll
      for (int u = 0; u < 2; ++u)
#pragma unroll
        for (int t = 0; t < RT; ++t) {
          const int room = (known[u] ? sees[t] : 0) - (token + 16 * u + 4 * h);
#pragma unroll
          for (int e = 0; e < 4; ++e) score[t][0][u][e] = e < room ? score[t][0][u][e] : -__builtin_inff();
        }
      // what lies behind the last key, and in pages that are none, is no number: a step of zero makes it zero
#pragma unroll
      for (int u = 0; u < 2; ++u) {
        const int exist = known[u] ? end - (token + 16 * u + 4 * h) : 0;
#pragma unroll
        for (int n = 0; n < S::UNITS; ++n) {
          if (exist < 4) now[u].value_pair[n][1] &= exist < 3 ? 0 : 0x0000ffff;
          if (exist < 2) now[u].value_pair[n][0] &= exist < 1 ? 0 : 0x0000ffff;
        }
      }
    }
    v8h p[RT][1];
    weights(score, scale, top, far, out, h, p);
#pragma unroll
    for (int t = 0; t < RT; ++t) out[t][S::CHANNELS] = multiply(p[t][0], ones, out[t][S::CHANNELS]);
    if (token + STEP > fewest) {
      uint32_t any = 0;
#pragma unroll
      for (int n = 0; n < S::UNITS; ++n)
#pragma unroll
        for (int u = 0; u < 2; ++u) any |= no_step(now[u].value_pair[n][0]) | no_step(now[u].value_pair[n][1]);
      if (__any(any)) {
#pragma unroll
        for (int n = 0; n < S::UNITS; ++n) {
          v2i &a = now[0].value_pair[n], &b = now[1].value_pair[n];
          const v4u none = {no_number(a[0]), no_number(a[1]), no_number(b[0]), no_number(b[1])};
#pragma unroll
          for (int t = 0; t < RT; ++t) {
            const v8h tokens = seen_tokens<16>(sees[t] - (token + 4 * h));
            lost |= seen_of(tokens, __builtin_bit_cast(v8h, none)) << (4 * (t * S::UNITS + n));
          }
          a = v2i{(int)numbers_of(a[0]), (int)numbers_of(a[1])};
          b = v2i{(int)numbers_of(b[0]), (int)numbers_of(b[1])};
        }
      }
    }
#pragma unroll
    for (int n = 0; n < S::UNITS; ++n) {
      const Kv4Values<D> values(now[0].value[n], now[1].value[n], now[0].value_pair[n], now[1].value_pair[n], lane);
#pragma unroll
      for (int k = 0; k < S::NIBBLES / 2; ++k) {
        v8h even, odd;
        values.pair(k, exponents, even, odd);
#pragma unroll
        for (int t = 0; t < RT; ++t) {
          v4f &a = out[t][n * S::NIBBLES + 2 * k], &b = out[t][n * S::NIBBLES + 2 * k + 1];
          a = multiply(p[t][0], even, a);
          b = multiply(p[t][0], odd, b);
        }
      }
    }
    if (step + WAVES < steps) fetch_values();
  }

  // the waves' results meet: thread 16 row + part takes D / 16 channels in a row of one row
  const int row_in = tid >> 4, part = tid & 15;
#pragma unroll
  for (int t = 0; t < RT; ++t) {
    if (t > 0) __syncthreads();
    if (h == 0) tops[wave][c] = top[t];
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      if (c == 0) totals[wave][4 * h + e] = out[t][S::CHANNELS][e];
#pragma unroll
      for (int j = 0; j < S::CHANNELS; ++j)
        sums[wave][4 * h + e][S::value_channel(j / S::NIBBLES, j % S::NIBBLES, c)] =
            lost >> (4 * (t * S::UNITS + j / S::NIBBLES) + e) & 1 ? __builtin_nanf("") : out[t][j][e];
    }
    __syncthreads();
    const int row = row0 + 16 * t + row_in;
    float m = tops[0][row_in], l = 0.0f, o[D / 16];
#pragma unroll
    for (int w = 1; w < WAVES; ++w) m = fmaxf(m, tops[w][row_in]);
#pragma unroll
    for (int i = 0; i < D / 16; ++i) o[i] = 0.0f;
#pragma unroll
    for (int w = 0; w < WAVES; ++w) {
      const float by = __builtin_amdgcn_exp2f(tops[w][row_in] - m);
      l += by * totals[w][row_in];
#pragma unroll
      for (int i = 0; i < D / 16; ++i) o[i] += by * sums[w][row_in][part * (D / 16) + i];
    }
    if (row >= rows) continue;
    const int query = row / P.shared, within = row - query * P.shared;
    if (P.partials) {
      const int64_t row_of_all = ((int64_t)(req.q0 + query) * P.kv_heads + head) * P.shared + within;
      float *to = P.partials + (row_of_all * P.ranges + range) * PARTIAL<D>;
#pragma unroll
      for (int i = 0; i < D / 16; i += 4)
        *reinterpret_cast<v4f *>(to + part * (D / 16) + i) = v4f{o[i], o[i + 1], o[i + 2], o[i + 3]};
      if (part == 0) *reinterpret_cast<v2f *>(to + D) = v2f{m, l};
    } else {
      const float by = l != 0.0f ? 1.0f / l : of_no_sum(pages.any_named(named_of(P, req.keys - req.queries + query + 1)));
      const int64_t at = (req.q0 + query) * P.ldo + (int64_t)(head * P.shared + within) * D + part * (D / 16);
#pragma unroll
      for (int i = 0; i < D / 16; i += 4)
        store_real4(P.O, at + i, TYPE, v4f{o[i], o[i + 1], o[i + 2], o[i + 3]} * by);
    }
  }
}

// The kernel for many rows of 256 channels.  A workgroup of eight waves takes 128 rows of one request and key head; tiles of
// 64 keys are brought from codes to float16 once for all of them, each wave its share, and lie in LDS as the operands the
// instructions take, 1 KB each, so that every read is sixteen bytes a lane in a row.
//
// A SIMD has two waves, one of either half of the workgroup, and the halves run half a tile apart, held there by a
// barrier after every half: while one wave keeps the matrix unit busy (output of a tile, scores of the next), the other
// has the vector unit to itself (weights of a tile, its share of the codes to come).  Side by side they take the
// two units in turns.  2048 queries of 16 heads over 4096 keys of 4: 177 us, 580 TFLOP/s.
template <int TYPE>
__global__ __launch_bounds__(512, 2) void attention_tiles_kernel(AttentionArgs P) {
  constexpr int D = 256;
  using S = Kv4Shape<D>;
  constexpr int RT = 1, W = 8, TILE = 64, KEYS = 4 * S::KEY_STEPS, VALUES = 2 * S::CHANNELS;  // operands of a tile
  constexpr int KEY_PARTS = W / 4, KEY_EACH = S::KEY_STEPS / KEY_PARTS;  // a wave's share of a tile of sixteen keys
  constexpr int VALUE_EACH = S::CHANNELS / 2 / (W / 2);  // and of the values of two
  extern __shared__ __attribute__((aligned(16))) uint8_t smem[];
  __shared__ int named[2][4];  // whether the table names a page for the tiles of sixteen of a stage
  // values that are no numbers: patterns of tile i % 4's steps and units, and i + 1 where there is one
  __shared__ __attribute__((aligned(16))) uint8_t none[4][2][S::UNITS][1024];
  __shared__ int has_none[4][2][S::UNITS];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int c = lane & 15, h = lane >> 4;
  const int range = blockIdx.x % P.ranges, r = blockIdx.z;
  // the last rows of a prompt see the most keys: they begin first
  const int of_all = P.first + (int)(gridDim.x / P.ranges) - 1 - (int)(blockIdx.x / P.ranges);
  const int head = of_all % P.kv_heads, row0 = of_all / P.kv_heads * (16 * RT * W);
  const int key_tile = wave & 3, key_part = wave >> 2, step = wave & 1, value_part = wave >> 1;
  const int begin = range * P.span;
  const Pages pages(P, r, head, Kv4Layout(1 << P.log_page, D).block);
  int key_page = pages.of(begin + 16 * key_tile);
  int value_page[2] = {pages.of(begin + 32 * step), pages.of(begin + 32 * step + 16)};
  const Request req = request_of(P, r);
  const int rows = req.queries * P.shared;
  if (row0 >= rows) return;
  const int before = req.keys - req.queries + 1;  // keys that the first query sees
  auto sees_of = [&](int row) { return before + row / P.shared; };
  const int seen = named_of(P, sees_of(row0 + 16 * RT * W < rows ? row0 + 16 * RT * W - 1 : rows - 1));
  const int end = range_end(P, begin, seen);
  if (range > 0 && begin >= end) return;

  const int wave_row = row0 + wave * (16 * RT);
  v8h q[RT][S::KEY_STEPS];
  float scale[RT], top[RT];
  bool far = true;  // (the first base is)
  int sees[RT];
  v4f out[RT][S::CHANNELS + 1];  // the last: sums of p
  uint32_t lost = 0;  // four bits to a row tile and unit: rows that have seen a value that is no number
#pragma unroll
  for (int t = 0; t < RT; ++t) {
    const int of_row = wave_row + 16 * t + c, row = of_row < rows ? of_row : rows - 1, query = row / P.shared;
    const int64_t at = (req.q0 + query) * P.ldq + (int64_t)(head * P.shared + (row - query * P.shared)) * D;
    scale[t] = load_queries<D, TYPE>(P, at, of_row < rows, h, q[t]);
    sees[t] = before + query;
    top[t] = LOWEST;
#pragma unroll
    for (int j = 0; j <= S::CHANNELS; ++j) out[t][j] = v4f{0.0f, 0.0f, 0.0f, 0.0f};
  }
  // the fewest and the most keys that a row of the wave sees
  const int wave_end = wave_row + 16 * RT < rows ? wave_row + 16 * RT : rows;
  const int fewest = wave_row < rows ? sees_of(wave_row) : 0, most = wave_row < rows ? sees_of(wave_end - 1) : 0;

  const _Float16 one = (_Float16)1.0f;
  const v8h ones = {one, one, one, one, one, one, one, one};
  const Kv4Exponents exponents;
  const Kv4Reader<D> reader(P.log_page, lane);
  const int tiles = end > begin ? (end - begin + TILE - 1) / TILE : 0;
  // a wave's share: keys of tile `wave % 4`, a quarter of the channels of the values of the tiles 2 (wave % 2) and the one after
  const int unit = value_part * VALUE_EACH / (S::NIBBLES / 2);
  uint32_t key[KEY_EACH], key_pair;
  v4u value[2];
  v2i value_pair[2];
  bool key_named;
  // (past the last tile, the last again: what it becomes is not used)
  auto first_of = [&](int tile) { return begin + (tile < tiles ? tile : tiles - 1) * TILE; };
  auto fetch_keys = [&](int tile) {
    const int first = first_of(tile) + 16 * key_tile;
    key_named = pages.named(key_page, first);
    reader.template load_keys<KEY_EACH>(pages.part(key_page, key_named), pages.within(first), key_part * KEY_EACH, key, key_pair);
  };
  // the pages of the tiles that come after those: asked for at the start of a half, since its end waits for them
  int next_key_page = 0, next_value_page[2] = {0, 0};
  auto ask = [&](int of_keys, int of_values) {
    next_key_page = pages.of(first_of(of_keys) + 16 * key_tile);
#pragma unroll
    for (int i = 0; i < 2; ++i) next_value_page[i] = pages.of(first_of(of_values) + 32 * step + 16 * i);
    __builtin_amdgcn_sched_barrier(0);
  };
  auto told = [&] {
    key_page = next_key_page;
#pragma unroll
    for (int i = 0; i < 2; ++i) value_page[i] = next_value_page[i];
  };
  auto fetch_values = [&](int tile) {
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const int first = first_of(tile) + 32 * step + 16 * i;
      const bool exists = pages.named(value_page[i], first);
      reader.load_values(pages.part(value_page[i], exists), pages.within(first), unit, value[i], value_pair[i]);
      // what lies behind the last key, and in pages that are none, is no number: a step of zero makes it zero
      const int exist = exists ? end - first - 4 * h : 0;
      if (exist < 4) value_pair[i][1] &= exist < 3 ? 0 : 0x0000ffff;
      if (exist < 2) value_pair[i][0] &= exist < 1 ? 0 : 0x0000ffff;
    }
  };
  auto unpack_keys = [&](int stage) {
    uint8_t *to = smem + stage * (KEYS * 1024) + 16 * lane;
    const Kv4Scale g(key_pair * 0x00010001u);
#pragma unroll
    for (int i = 0; i < KEY_EACH; ++i)
      *reinterpret_cast<v8h *>(to + (key_tile * S::KEY_STEPS + key_part * KEY_EACH + i) * 1024) = key_operand(key[i], g, exponents);
    if (key_part == 0) named[stage][key_tile] = key_named;
  };
  auto unpack_values = [&](int tile) {
    const int stage = tile & 1;
    if (tile < tiles && begin + tile * TILE + TILE > sees_of(row0)) {  // some row may not see all of its keys
      v2i &a = value_pair[0], &b = value_pair[1];
      if (__any(no_step(a[0]) | no_step(a[1]) | no_step(b[0]) | no_step(b[1]))) {  // (two waves find and write the same)
        has_none[tile & 3][step][unit] = tile + 1;
        int at = 16 * lane;
        asm volatile("" : "+v"(at));  // (its addresses are not kept over the loop)
        *reinterpret_cast<v4u *>(none[tile & 3][step][unit] + at) = v4u{no_number(a[0]), no_number(a[1]), no_number(b[0]), no_number(b[1])};
        a = v2i{(int)numbers_of(a[0]), (int)numbers_of(a[1])};
        b = v2i{(int)numbers_of(b[0]), (int)numbers_of(b[1])};
      }
    }
    uint8_t *to = smem + (2 * KEYS + stage * VALUES + step * S::CHANNELS) * 1024 + 16 * lane;
    const Kv4Values<D> values(value[0], value[1], value_pair[0], value_pair[1], lane);
#pragma unroll
    for (int i = 0; i < VALUE_EACH; ++i) {
      const int pair = value_part * VALUE_EACH + i;
      v8h even, odd;
      values.pair(pair % (S::NIBBLES / 2), exponents, even, odd);
      *reinterpret_cast<v8h *>(to + (2 * pair) * 1024) = even;
      *reinterpret_cast<v8h *>(to + (2 * pair + 1) * 1024) = odd;
    }
  };
  v4f score[RT][2][2];
  v8h p[RT][2];
  // Output of the values in one stage (VALUES_TOO) and scores of the keys in another, as one run of operands: each is read
  // LOOK before it is used, in this order and no other, since left to itself the compiler reads two and waits for
  // them.
  auto multiply_tiles = [&](auto values_tag, auto keys_tag, int value_stage, int key_stage) {
    constexpr int V = decltype(values_tag)::value ? VALUES : 0, N = V + (decltype(keys_tag)::value ? KEYS : 0), LOOK = 3;
    const uint8_t *values = smem + (2 * KEYS + value_stage * VALUES) * 1024 + 16 * lane;
    const uint8_t *keys = smem + key_stage * (KEYS * 1024) + 16 * lane;
    auto read = [&](int i) { return *reinterpret_cast<const v8h *>(i < V ? values + i * 1024 : keys + (i - V) * 1024); };
    v8h ring[LOOK];
#pragma unroll
    for (int i = 0; i < LOOK; ++i) ring[i] = read(i);
#pragma unroll
    for (int i = 0; i < N; ++i) {
#pragma unroll
      for (int t = 0; t < RT; ++t) {
        if (i < V) {
          const int half = i / S::CHANNELS, j = i % S::CHANNELS;
          if (j == 0) out[t][S::CHANNELS] = multiply(p[t][half], ones, out[t][S::CHANNELS]);
          out[t][j] = multiply(p[t][half], ring[i % LOOK], out[t][j]);
        } else {
          const int u = (i - V) / S::KEY_STEPS, w = (i - V) % S::KEY_STEPS;
          if (w == 0) score[t][u / 2][u % 2] = v4f{0.0f, 0.0f, 0.0f, 0.0f};
          score[t][u / 2][u % 2] = multiply(ring[i % LOOK], q[t][w], score[t][u / 2][u % 2]);
        }
      }
      if (i + LOOK < N) ring[i % LOOK] = read(i + LOOK);
      __builtin_amdgcn_sched_barrier(0);
    }
  };
  // NaN in the rows that see a value of the tile that is no number
  auto mark_none = [&](int tile) {
    if (begin + tile * TILE + TILE <= sees_of(row0)) return;  // (the others' keys count too: what is made zero is for all)
#pragma unroll
    for (int half = 0; half < 2; ++half) {
#pragma unroll
      for (int n = 0; n < S::UNITS; ++n) {
        if (__builtin_amdgcn_readfirstlane(has_none[tile & 3][half][n]) != tile + 1) continue;
        int at = 16 * lane;
        asm volatile("" : "+v"(at));
        const v8h pattern = *reinterpret_cast<const v8h *>(none[tile & 3][half][n] + at);
#pragma unroll
        for (int t = 0; t < RT; ++t) {
          const v8h tokens = seen_tokens<16>(sees[t] - (begin + tile * TILE + 32 * half + 4 * h));
          lost |= seen_of(tokens, pattern) << (4 * (t * S::UNITS + n));
        }
      }
    }
  };
  auto mask_scores = [&](int tile) {
    const int token = begin + tile * TILE;
    const v4i all_named = *reinterpret_cast<const v4i *>(named[tile & 1]);
    if (token + TILE > fewest || !__builtin_amdgcn_readfirstlane(all_named[0] & all_named[1] & all_named[2] & all_named[3])) {
#pragma unroll
      for (int u = 0; u < 4; ++u)
#pragma unroll
        for (int t = 0; t < RT; ++t) {
          const int room = (all_named[u] ? sees[t] : 0) - (token + 16 * u + 4 * h);
#pragma unroll
          for (int e = 0; e < 4; ++e) score[t][u / 2][u % 2][e] = e < room ? score[t][u / 2][u % 2][e] : -__builtin_inff();
        }
    }
  };

  // (not __syncthreads: loads from memory stay in flight across it)
  auto half_done = [] { asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory"); };

  // Half h of the first four waves is the output of tile h / 2 - 1 and the scores of tile h / 2 where h is even, the weights of
  // tile h / 2 where it is odd; the other four are one half behind.  With two stages each, the keys of a tile and
  // the values of the tile before are read in the halves 2 i and 2 i + 1.  The first four write the values of tile i
  // and the keys of i + 1 in half 2 i + 1, the others the same in half 2 i, ahead of it by a tile: after the last
  // reads of what they overwrite, before the first of theirs.
  const int ahead = wave >> 2;
  if (tid < 8 * S::UNITS) has_none[tid & 3][tid >> 2 & 1][tid >> 3] = 0;
  if (tiles > 0) {
    ask(1, 1);
    fetch_keys(0);
    unpack_keys(0);
    fetch_values(0);
    told();
    fetch_keys(1);
    ask(2, 1);
    half_done();
    told();
    if (ahead) {
      ask(3, 2);
      unpack_values(0);
      unpack_keys(1);
      fetch_values(1);
      fetch_keys(2);
      half_done();
      told();
    }
    for (int tile = 0; tile < tiles; ++tile) {
      const bool sees_any = begin + tile * TILE < most;
      if (sees_any) {
        if (tile > 0) multiply_tiles(std::true_type{}, std::true_type{}, (tile - 1) & 1, tile & 1);
        else multiply_tiles(std::false_type{}, std::true_type{}, 0, 0);
      }
      half_done();
      if (sees_any) mask_scores(tile);
      ask(tile + ahead + 3, tile + ahead + 2);  // (behind the scores' one read of LDS, whose wait would include it)
      if (sees_any) weights(score, scale, top, far, out, h, p);
      unpack_values(tile + ahead);
      unpack_keys((tile + ahead + 1) & 1);
      fetch_values(tile + ahead + 1);
      fetch_keys(tile + ahead + 2);
      told();
      half_done();
      // (the rows of a wave that see nothing of the next tile end here)
      if (sees_any) mark_none(tile);
      if (sees_any && (tile + 1 == tiles || begin + (tile + 1) * TILE >= most))
        multiply_tiles(std::true_type{}, std::false_type{}, tile & 1, 0);
    }
    if (!ahead) half_done();
  }

#pragma unroll
  for (int t = 0; t < RT; ++t) {
    float nothing = 0.0f;  // of a row without a sum (lane: row l % 16)
    const v4f l_of = out[t][S::CHANNELS];
    if (!P.partials && __any(l_of[0] == 0.0f || l_of[1] == 0.0f || l_of[2] == 0.0f || l_of[3] == 0.0f))
      nothing = of_no_sum(pages.first_named(seen) < sees[t]);
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const int row = wave_row + 16 * t + 4 * h + e;
      const float l = l_of[e], m = __shfl(top[t], 4 * h + e), none_of = __shfl(nothing, 4 * h + e);
      if (row >= rows) continue;
      const int query = row / P.shared, within = row - query * P.shared;
      const float by = P.partials ? 1.0f : (l != 0.0f ? 1.0f / l : none_of);
      const int64_t at = (req.q0 + query) * P.ldo + (int64_t)(head * P.shared + within) * D;
      float *to = nullptr;
      if (P.partials) {
        const int64_t row_of_all = ((req.q0 + query) * P.kv_heads + head) * P.shared + within;
        to = P.partials + (row_of_all * P.ranges + range) * PARTIAL<D>;
        if (c == 0) *reinterpret_cast<v2f *>(to + D) = v2f{m, l};
      }
#pragma unroll
      for (int j = 0; j < S::CHANNELS; j += 4) {
        const v4f o = v4f{out[t][j][e], out[t][j + 1][e], out[t][j + 2][e], out[t][j + 3][e]} *
                      (lost >> (4 * (t * S::UNITS + j / S::NIBBLES) + e) & 1 ? __builtin_nanf("") : by);
        const int channel = S::value_channel(j / S::NIBBLES, j % S::NIBBLES, c);
        if (P.partials) *reinterpret_cast<v4f *>(to + channel) = o;
        else store_real4(P.O, at + channel, TYPE, o);
      }
    }
  }
}

// The ranges of one row and head joined: a workgroup to a row, D / 4 lanes to a range, in turn, then the first wave.  Two
// loads deep and a launch: 3 to 5 us.  (Cut by channels as well, 32 ranges at a time, 192 ranges took 39.4 us instead of 41.1
// with the kernel before, 3 ranges of 2048 rows 34.7 instead of 29.5.)
template <int D, int TYPE>
__global__ __launch_bounds__(256) void attention_join_kernel(AttentionArgs P) {
  constexpr int LANES = D / 4, GROUPS = 256 / LANES;
  __shared__ v4f sums[GROUPS][LANES];
  __shared__ float tops[GROUPS], totals[GROUPS];
  const int at = threadIdx.x % LANES, group = threadIdx.x / LANES;
  const int of_all = P.first + blockIdx.x, r = blockIdx.z;
  const int head = of_all % (P.kv_heads * P.shared), query = of_all / (P.kv_heads * P.shared);
  const Request req = request_of(P, r);
  if (query >= req.queries) return;
  const int seen = named_of(P, req.keys - req.queries + query + 1);
  // (every range that the row's tile went through has written; those that hold none of the row's keys, a sum of zero)
  const int ranges = seen <= 0 ? 1 : (seen - 1) / P.span + 1;
  const float *from = P.partials + ((req.q0 + query) * P.kv_heads * P.shared + head) * (int64_t)P.ranges * PARTIAL<D>;
  float m = LOWEST, l = 0.0f;
  v4f o = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll 4
  for (int i = group; i < ranges; i += GROUPS) {
    const v2f ml = *reinterpret_cast<const v2f *>(from + (int64_t)i * PARTIAL<D> + D);
    const v4f x = *reinterpret_cast<const v4f *>(from + (int64_t)i * PARTIAL<D> + 4 * at);
    const float top = fmaxf(m, ml[0]), a = __builtin_amdgcn_exp2f(m - top), b = __builtin_amdgcn_exp2f(ml[0] - top);
    o = o * a + x * b;
    l = l * a + ml[1] * b;
    m = top;
  }
  sums[group][at] = o;
  if (at == 0) {
    tops[group] = m;
    totals[group] = l;
  }
  __syncthreads();
  if (threadIdx.x >= 64) return;
  // the first wave: a lane takes four channels of some of the groups
  constexpr int PARTS = 64 / LANES;
  m = tops[0];
#pragma unroll
  for (int w = 1; w < GROUPS; ++w) m = fmaxf(m, tops[w]);
  l = 0.0f;
  o = v4f{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
  for (int w = 0; w < GROUPS / PARTS; ++w) {
    const int of = w * PARTS + group;
    const float by = __builtin_amdgcn_exp2f(tops[of] - m);
    o += sums[of][at] * by;
    l += totals[of] * by;
  }
#pragma unroll
  for (int d = LANES; d < 64; d *= 2) {
    l += __shfl_xor(l, d);
#pragma unroll
    for (int e = 0; e < 4; ++e) o[e] += __shfl_xor(o[e], d);
  }
  float by = 1.0f / l;
  if (__any(l == 0.0f)) by = of_no_sum(Pages(P, r, 0, 0).first_named(seen) < seen);  // (the sum is the same in all lanes)
  if (group == 0) store_real4(P.O, (req.q0 + query) * P.ldo + (int64_t)head * D + 4 * at, TYPE, o * by);
}

// `count` things, `each` workgroups to one, as many in a launch as a grid holds.
hipError_t launch_in_slabs(void (*kernel)(AttentionArgs), AttentionArgs P, int64_t count, int64_t each, int requests,
                           unsigned threads, size_t lds, hipStream_t s) {
  const int64_t most = ((int64_t)1 << 22) / each > 0 ? ((int64_t)1 << 22) / each : 1;
  for (int64_t i = 0; i < count; i += most) {
    P.first = (int)i;
    const int64_t here = count - i < most ? count - i : most;
    const hipError_t e = launch_with(reinterpret_cast<const void *>(kernel), dim3((unsigned)(here * each), 1, (unsigned)requests),
                                     threads, lds, s, &P);
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}

// How a call is cut: rows to a workgroup, and the keys into ranges of `span`.
struct Cut {
  bool tiles;  // the kernel for many rows
  int rows, ranges, span;
};
Cut cut_call(int64_t requests, int64_t kv_heads, int64_t shared, int head_dim, int64_t max_q, int64_t max_kv) {
  const int64_t rows = max_q * shared;
  Cut cut;
  // The kernels for many rows bring a tile of keys to float16 once for all of them, but put one workgroup on a compute unit and
  // hold its waves together with barriers: 8 requests of up to 8192 keys, 96 rows of 128 channels, take 73 us with them and 49
  // with the kernel for few; 256 rows 88 and 97.  In 256 channels, where the kernel for few has registers for two workgroups
  // at most, 36 rows 83 and 97.
  cut.tiles = rows > (head_dim == 256 ? 32 : 128);
  cut.rows = cut.tiles ? (head_dim == 256 ? 128 : 256) : (rows <= 16 ? 16 : 32);
  const int64_t groups = requests * kv_heads * ((rows + cut.rows - 1) / cut.rows);
  const int64_t round = cut.tiles ? 64 : WAVES * STEP;  // keys between two barriers, or of all waves' steps
  // Workgroups to a compute unit that are asked for.  Many rows: one, as many as fit.  Few rows of one request: as many as
  // fit at once (131001 keys of 8 heads 36.5 us, 41.4 with six).  Of several, whose lengths may differ, six (32 requests of
  // up to 8192 keys, half of them there: 44.8 us, 57.7 with four).
  const int64_t fit = cut.tiles ? 1 : (head_dim <= 128 && cut.rows == 16 ? 4 : 2);
  int64_t want = ((cut.tiles || requests == 1 ? fit : 6) * compute_units() + groups - 1) / groups;
  // Rounds that a range has at least: what a workgroup begins and ends with takes as long as some of them.  While there is
  // less than a workgroup to a compute unit, two (4096 keys 11.4 us, 12.0 with four; 5000 of 256 channels 13.7, 16.0),
  // but four and less stay whole (301 keys 6.4 us, 10.3 in two, of which joining them is 3).
  auto ranges_of = [&](int64_t least) { return (max_kv + least * round - 1) / (least * round); };
  int64_t most = ranges_of(cut.tiles ? 8 : 4);
  if (!cut.tiles && most > 1) {
    const int64_t each = (compute_units() + groups - 1) / groups, fine = ranges_of(2) < each ? ranges_of(2) : each;
    most = most > fine ? most : fine;
  }
  if (want > most) want = most;
  if (want < 1) want = 1;
  int64_t each = (max_kv + want - 1) / want;
  each = (each + round - 1) / round * round;
  if (each < round) each = round;
  cut.span = (int)each;
  cut.ranges = (int)((max_kv + each - 1) / each);
  if (cut.ranges < 1) cut.ranges = 1;
  return cut;
}

template <int D, int TYPE>
hipError_t launch_for(const AttentionArgs &P, const Cut &cut, int requests, hipStream_t s) {
  const int64_t rows = (int64_t)P.max_q * P.shared, groups = (rows + cut.rows - 1) / cut.rows * P.kv_heads;
  AttentionKernel kernel;
  unsigned threads = 256;
  size_t lds = (size_t)WAVES * 16 * (D + 4) * 4;
  if (cut.tiles) {
    if constexpr (D == 256) kernel = attention_tiles_kernel<TYPE>;
    else kernel = attention_wide(D, TYPE, P.log_page);
    threads = 512;
    lds = (size_t)(D / 4) * 2048;
  } else {
    kernel = cut.rows == 16 ? attention_rows_kernel<D, TYPE, 1> : attention_rows_kernel<D, TYPE, 2>;
  }
  // (in 256 channels what is not dynamic leaves just that much)
  hipError_t e = allow_dynamic_lds(reinterpret_cast<const void *>(kernel), lds + (D == 256 ? 0 : 18432));
  if (e == hipSuccess) e = launch_in_slabs(kernel, P, groups, P.ranges, requests, threads, lds, s);
  if (e != hipSuccess || !P.partials) return e;
  return launch_in_slabs(attention_join_kernel<D, TYPE>, P, (int64_t)P.max_q * P.kv_heads * P.shared, 1, requests, 256, 0, s);
}

}  // namespace

size_t attention_scratch(int64_t requests, int64_t kv_heads, int64_t shared, int head_dim, int64_t max_q, int64_t max_kv) {
  const int ranges = cut_call(requests, kv_heads, shared, head_dim, max_q, max_kv).ranges;
  return ranges > 1 ? (size_t)(requests * max_q * kv_heads * shared) * (size_t)ranges * (size_t)(head_dim + 4) * 4 + 16 : 0;
}

hipError_t launch_attention(AttentionArgs P, int requests, int head_dim, int type, void *ws, size_t ws_bytes, hipStream_t s) {
  const Cut cut = cut_call(requests, P.kv_heads, P.shared, head_dim, P.max_q, P.max_kv);
  P.ranges = cut.ranges;
  P.span = cut.span;
  const size_t skip = (16 - reinterpret_cast<uintptr_t>(ws) % 16) % 16;
  const size_t need = (size_t)P.q_rows * (size_t)(P.kv_heads * P.shared) * (size_t)P.ranges * (size_t)(head_dim + 4) * 4;
  if (P.ranges > 1 && ws && ws_bytes >= skip && ws_bytes - skip >= need) {
    P.partials = reinterpret_cast<float *>(static_cast<uint8_t *>(ws) + skip);
  } else {
    P.partials = nullptr;
    P.ranges = 1;
    P.span = 0;
  }
  // (requests go to grid.z)
  const int most = 65535;
  for (int r = 0; r < requests; r += most) {
    AttentionArgs A = P;
    A.q_starts += r;
    A.kv_lengths += r;
    A.block_table += (int64_t)r * P.table_stride;
    const int here = requests - r < most ? requests - r : most;
    hipError_t e;
    if (type == REAL_BF16)
      e = head_dim == 64    ? launch_for<64, REAL_BF16>(A, cut, here, s)
          : head_dim == 128 ? launch_for<128, REAL_BF16>(A, cut, here, s)
                            : launch_for<256, REAL_BF16>(A, cut, here, s);
    else
      e = head_dim == 64    ? launch_for<64, REAL_F16>(A, cut, here, s)
          : head_dim == 128 ? launch_for<128, REAL_F16>(A, cut, here, s)
                            : launch_for<256, REAL_F16>(A, cut, here, s);
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}

}  // namespace mip
