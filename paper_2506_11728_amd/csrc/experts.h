// What the kernels of the experts' products share: which rows of which expert a workgroup has, and the write-back.
#pragma once
#include "layer_internal.h"
#include "linear.h"

namespace mip {

// The kernels, each with what it can take: any call (kernel_experts.hip), 16 rows to a workgroup, tiles of many rows (large: 192 x 256).
int64_t experts_slim_tiles(const ExpertsArgs &X);
bool experts_slim_eligible(const ExpertsArgs &X);
hipError_t launch_experts_slim(const ExpertsArgs &X, hipStream_t s);
bool experts_tile_eligible(const ExpertsArgs &X);
hipError_t launch_experts_tile(const ExpertsArgs &X, bool large, hipStream_t s);

// Rows `first` .. first + count - 1 (count up to BM) of expert e.
struct ExpertTile {
  int e, count;
  int64_t first;
};

// Tile `slot` of the experts' rows cut into pieces of BM, expert by expert; count 0: there are not so many.  The whole wave
// calls it, every lane with the same arguments.  A lane takes up to 16 neighbouring experts: one round of loads, a
// scan over the lanes, a ballot.
__device__ __forceinline__ ExpertTile expert_tile(const int32_t *starts, int experts, int64_t rows, int BM, int64_t slot, int lane) {
  const int each = (experts + 63) / 64, e0 = lane * each;
  auto start = [&](int e) -> int64_t {
    const int64_t s = starts[e < experts ? e : experts];
    return s < 0 ? 0 : (s > rows ? rows : s);
  };
  auto pieces = [&](int64_t from, int64_t to) { return to > from ? (int)((to - from + BM - 1) / BM) : 0; };
  int mine = 0;
  int64_t from = start(e0);
  for (int i = 0; i < each; ++i) {
    const int64_t to = start(e0 + i + 1);
    if (e0 + i < experts) mine += pieces(from, to);
    from = to;
  }
  int sum = mine;
#pragma unroll
  for (int d = 1; d < 64; d *= 2) {
    const int o = __shfl_up(sum, d);
    if (lane >= d) sum += o;
  }
  const uint64_t beyond = __ballot((int64_t)sum > slot);
  if (!beyond) return {0, 0, 0};
  const int owner = __builtin_ctzll(beyond);
  int64_t left = slot - (__builtin_amdgcn_readlane(sum, owner) - __builtin_amdgcn_readlane(mine, owner));
  if (left < 0) return {0, 0, 0};  // (starts that fall)
  int64_t at = start(owner * each);
  for (int i = 0; i < each; ++i) {
    const int e = owner * each + i;
    const int64_t to = start(e + 1);
    const int n = pieces(at, to);
    if (left < n) {
      const int64_t first = at + left * BM, rest = to - first;
      return {e, (int)(rest < BM ? rest : BM), first};
    }
    left -= n;
    at = to;
  }
  return {0, 0, 0};
}

// The same for tiles of `columns` columns as well, workgroup `id` of a grid: the tiles of an XCD, which every eighth workgroup
// goes to, are neighbours, and of neighbours the rows change first: they share an expert's weights in its L2.
__device__ __forceinline__ ExpertTile expert_tile_of(const int32_t *starts, int experts, int64_t rows, int BM, int columns, unsigned id, int lane,
                                                     int *column) {
  const int each = (experts + 63) / 64, e0 = lane * each;
  auto start = [&](int e) -> int64_t {
    const int64_t s = starts[e < experts ? e : experts];
    return s < 0 ? 0 : (s > rows ? rows : s);
  };
  auto pieces = [&](int64_t from, int64_t to) { return to > from ? (int)((to - from + BM - 1) / BM) : 0; };
  int mine = 0;
  int64_t from = start(e0);
  for (int i = 0; i < each; ++i) {
    const int64_t to = start(e0 + i + 1);
    if (e0 + i < experts) mine += pieces(from, to);
    from = to;
  }
  int sum = mine;
#pragma unroll
  for (int d = 1; d < 64; d *= 2) {
    const int o = __shfl_up(sum, d);
    if (lane >= d) sum += o;
  }
  const int64_t total = (int64_t)__builtin_amdgcn_readlane(sum, 63) * columns, share = (total + 7) / 8;
  const int64_t at = id / 8, slot = (id % 8) * share + at;
  if (at >= share || slot >= total) return {0, 0, 0};
  const uint64_t beyond = __ballot((int64_t)sum * columns > slot);
  if (!beyond) return {0, 0, 0};
  const int owner = __builtin_ctzll(beyond);
  int64_t left = slot - (int64_t)(__builtin_amdgcn_readlane(sum, owner) - __builtin_amdgcn_readlane(mine, owner)) * columns;
  if (left < 0) return {0, 0, 0};  // (starts that fall)
  int64_t row = start(owner * each);
  for (int i = 0; i < each; ++i) {
    const int e = owner * each + i;
    const int64_t to = start(e + 1);
    const int n = pieces(row, to);
    if (left < (int64_t)n * columns) {
      const int c = (int)((unsigned)left / (unsigned)n), r = (int)left - c * n;
      const int64_t first = row + (int64_t)r * BM, rest = to - first;
      *column = c;
      return {e, (int)(rest < BM ? rest : BM), first};
    }
    left -= (int64_t)n * columns;
    row = to;
  }
  return {0, 0, 0};
}

// The row of A behind sorted row p (below `rows`), and its scale; a row that A does not have: row 0 with a scale of 0, which
// makes zeros of its sums.
struct ExpertRow {
  int64_t at;
  float scale;
};
__device__ __forceinline__ ExpertRow expert_row(const ExpertsArgs &P, int64_t p) {
  int64_t at = p;
  if (P.order) {
    const int32_t o = P.order[p];
    at = o < 0 ? -1 : (int64_t)(P.top.inv ? __umulhi((unsigned)o, P.top.inv) : (unsigned)o / P.top.d);
  }
  const bool there = at >= 0 && at < P.a_rows;
  return {there ? at : 0, there ? (P.a_scales ? P.a_scales[at] : 1.0f) : 0.0f};
}

}  // namespace mip
