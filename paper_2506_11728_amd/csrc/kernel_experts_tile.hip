// The experts' products where an expert has many rows: tiles of BM rows of one expert by BN rows of its weights (with a gate
// BN / 2 pairs of a gate's and the other), operands global -> LDS directly, the rows of A from where `order` says they are.
//
// The main loop is that of the kernel for large products (dma_k128.h says why it is as it is): k blocks of 128, two LDS stages for A
// and three for B, the four waves 2 x 2 over the tile, v_mfma_i32_16x16x64_i8 with direct loads and fragment reads between
// them.  A direct load takes its address by lane, so that gathered rows cost nothing over neighbouring ones.
//
// 64 experts, 512 rows each on average, 1024 pairs of columns of 2048: 196 us, matrix units busy for 34 % of the time; 8 experts, 512 rows each, 4096
// columns of 11008: 216 us, 45 % (62 % of the time in which a compute unit has a tile: two rounds that fill one and a half).
//
// With a gate, blocks of 16 of its columns and 16 of the others take turns in LDS, so that a lane has the sums of a pair in
// two of its accumulators.
#include "dma_k128.h"
#include "experts.h"
#include "experts_store.h"

namespace mip {

namespace {

struct TileParams {
  ExpertsArgs X;
  int columns;  // column tiles
};

template <int BM, int BN>
struct ExpertsTile {
  using TS = Tile16<BM, BN>;
  using SA = Stage16<BM, true>;
  using SB = Stage16<BN, true>;
  static constexpr int FM = TS::FM, FN = TS::FN, WM = BM / 2, WN = BN / 2;
  static constexpr int A_BYTES = TS::A_STAGE_BYTES, B_BYTES = TS::B_STAGE_BYTES, B_BASE = TS::B_BASE;

  uint8_t *smem;
  int lane, wave, wm, wn;
  uint32_t lds0;
  int baseA[FM], baseB[FN];

  __device__ __forceinline__ void read(int sa, int sb, int ks, int r, v4i (&a)[FM], v4i (&b)[FN]) const {
    if (r < FN) b[r] = SB::fragment(smem + B_BASE + sb * B_BYTES, baseB[r], ks, lane);
    else a[r - FN] = SA::fragment(smem + sa * A_BYTES, baseA[r - FN], ks, lane);
  }
};

// Where the matrix instructions of 64 k leave room: loads between the first, reads between the later ones (Tile16's slots).
template <int BM, int BN, int LOADS, int LOADS_MAX, typename Reader>
__device__ __forceinline__ void multiply_64(v4i (&acc)[BM / 32][BN / 32], const v4i (&a)[BM / 32], const v4i (&b)[BN / 32], Reader reader,
                                            uint32_t lds, const uint32_t (&off)[LOADS_MAX], const uint8_t *from) {
  using TS = Tile16<BM, BN>;
#pragma unroll
  for (int s = 0; s < TS::NMFMA; ++s) {
    const int i = s / TS::FN, j = (i & 1) ? TS::FN - 1 - (s % TS::FN) : (s % TS::FN);
    if (s % TS::LOAD_EVERY == 0 && s / TS::LOAD_EVERY < LOADS) {
      asm volatile(
          "s_add_u32 m0, %3, %4\n\t"
          "v_mfma_i32_16x16x64_i8 %0, %1, %2, %0\n\t"
          "global_load_lds_dwordx4 %5, %6"
          : "+a"(acc[i][j])
          : "v"(b[j]), "v"(a[i]), "s"(lds), "i"((s / TS::LOAD_EVERY) * 4096), "v"(off[s / TS::LOAD_EVERY]), "s"(from)
          : "scc");
    } else {
      asm volatile("v_mfma_i32_16x16x64_i8 %0, %1, %2, %0" : "+a"(acc[i][j]) : "v"(b[j]), "v"(a[i]));
    }
    if (s >= TS::READ_FROM && (s - TS::READ_FROM) % TS::READ_EVERY == 0) {
      const int r = (s - TS::READ_FROM) / TS::READ_EVERY;
      if (r < TS::NREADS) reader(r);
    }
    __builtin_amdgcn_sched_barrier(0);
  }
}

template <int BM, int BN, int GATED>
__global__ __launch_bounds__(NTHREADS) void experts_tile_kernel(TileParams P) {
  using ET = ExpertsTile<BM, BN>;
  using TS = Tile16<BM, BN>;
  using SA = typename ET::SA;
  using SB = typename ET::SB;
  constexpr int FM = TS::FM, FN = TS::FN, LOADS_A = TS::LOADS_A, LOADS_B = TS::LOADS_B, LOADS_MAX = TS::LOADS_MAX;
  constexpr int OUT = GATED ? BN / 2 : BN;
  extern __shared__ __attribute__((aligned(16))) uint8_t smem[];
  const ExpertsArgs &X = P.X;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);

  int column;
  const ExpertTile tile = expert_tile_of(X.starts, X.experts, X.rows, BM, P.columns, blockIdx.x, lane, &column);
  if (tile.count == 0) return;
  const int64_t n0 = (int64_t)column * OUT;

  uint32_t offA[LOADS_MAX], offB[LOADS_MAX];
#pragma unroll
  for (int i = 0; i < LOADS_MAX; ++i) {
    int a, c;
    if (i < LOADS_A) {
      SA::chunk_of(i, tid, a, c);
      const int64_t at = expert_row(X, tile.first + (a < tile.count ? a : tile.count - 1)).at;
      offA[i] = (uint32_t)(at * X.lda + ((c ^ SA::kswz(a)) << 4));
    } else {
      offA[i] = 0;
    }
    if (i < LOADS_B) {
      SB::chunk_of(i, tid, a, c);
      int64_t to = n0 + (GATED ? a / 32 * 16 + a % 16 : a);
      to = to < X.n ? to : X.n - 1;
      if (GATED && (a / 16) % 2) to += X.n;
      offB[i] = (uint32_t)(to * X.ldb + ((c ^ SB::kswz(a)) << 4));
    } else {
      offB[i] = 0;
    }
  }
  // the scale of row `tid` of the tile, which goes to LDS when the stages are done with
  const float row_scale = tid < BM ? expert_row(X, tile.first + (tid < tile.count ? tid : 0)).scale : 0.0f;
  const uint8_t *gA = X.A, *gB = wave_uniform(X.B + tile.e * X.strideB);

  ET T;
  T.smem = smem; T.lane = lane; T.wave = wave; T.wm = wave >> 1; T.wn = wave & 1;
  T.lds0 = lds_address(smem) + wave * 1024;
#pragma unroll
  for (int f = 0; f < FM; ++f) T.baseA[f] = SA::lane_base(T.wm * ET::WM + f * 16, lane);
#pragma unroll
  for (int f = 0; f < FN; ++f) T.baseB[f] = SB::lane_base(T.wn * ET::WN + f * 16, lane);

  v4i acc[FM][FN];
#pragma unroll
  for (int i = 0; i < FM; ++i)
#pragma unroll
    for (int j = 0; j < FN; ++j) acc[i][j] = v4i{0, 0, 0, 0};
  v4i fa[2][FM], fb[2][FN];

  const uint32_t ldsB = T.lds0 + ET::B_BASE;
  auto issue_a = [&](int stage, int q) { dma16(offA[q], gA, T.lds0 + stage * ET::A_BYTES + q * 4096); };
  auto issue_b = [&](int stage, int q) { dma16(offB[q], gB, ldsB + stage * ET::B_BYTES + q * 4096); };
  using std::integral_constant;
  const int nkt = (int)(X.k / KD2);
  if (nkt > 0) {
#pragma unroll
    for (int q = 0; q < LOADS_A; ++q) issue_a(0, q);
#pragma unroll
    for (int q = 0; q < LOADS_B; ++q) issue_b(0, q);
    gA += KD2;
    gB += KD2;
    publish_barrier<0>();
#pragma unroll
    for (int r = 0; r < TS::NREADS; ++r) T.read(0, 0, 0, r, fa[0], fb[0]);
    if (nkt > 1) {
#pragma unroll
      for (int q = 0; q < LOADS_A; ++q) issue_a(1, q);
#pragma unroll
      for (int q = 0; q < LOADS_B; ++q) issue_b(1, q);
      gA += KD2;
      gB += KD2;
    }
    // Step t multiplies block t (A in stage t % 2, B in stage t % 3).  On entry A and B of block t + 1 are on their way.
    int bcur = 0;
    auto step = [&](int t, auto next_tag, auto next2_tag) {
      constexpr bool NEXT = decltype(next_tag)::value, NEXT2 = decltype(next2_tag)::value;
      const int cur = t & 1, oth = cur ^ 1;
      const int bnext = bcur == B_STAGES - 1 ? 0 : bcur + 1;
      const int bfill = bnext == B_STAGES - 1 ? 0 : bnext + 1;  // held block t - 1: free since the last barrier
      multiply_64<BM, BN, NEXT2 ? LOADS_B : 0, LOADS_MAX>(acc, fa[0], fb[0], [&](int r) { T.read(cur, bcur, 1, r, fa[1], fb[1]); },
                                                          ldsB + bfill * ET::B_BYTES, offB, gB);
      if (NEXT2) gB += KD2;
      // block t + 1 visible (only the B loads of block t + 2 may still fly); the A stage of block t may be refilled
      if (NEXT) {
        if (NEXT2) publish_barrier<LOADS_B>();
        else publish_barrier<0>();
      }
      multiply_64<BM, BN, NEXT2 ? LOADS_A : 0, LOADS_MAX>(acc, fa[1], fb[1], [&](int r) { if (NEXT) T.read(oth, bnext, 0, r, fa[0], fb[0]); },
                                                          T.lds0 + cur * ET::A_BYTES, offA, gA);
      if (NEXT2) gA += KD2;
      bcur = bnext;
    };
    using Y = integral_constant<bool, true>;
    using N = integral_constant<bool, false>;
    int t = 0;
    for (; t + 2 < nkt; ++t) step(t, Y{}, Y{});
    if (t + 1 < nkt) { step(t, Y{}, N{}); ++t; }
    step(t, N{}, N{});
  }
  // What is left of k, whole pieces of 16 bytes: a block whose other pieces come from a place that holds zeros.  (The last matrix
  // instructions have to have left the pipe before anything else may touch their accumulators, and no wave may still read
  // the stages.)
  asm volatile("s_nop 15\n\ts_nop 15\n\ts_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
  const int rest = (int)(X.k % KD2);
  if (rest > 0) {
#pragma unroll
    for (int q = 0; q < LOADS_A; ++q) {
      int a, c;
      SA::chunk_of(q, tid, a, c);
      dma16_at((c ^ SA::kswz(a)) * 16 < rest ? gA + offA[q] : outside_image, T.lds0 + q * 4096);
    }
#pragma unroll
    for (int q = 0; q < LOADS_B; ++q) {
      int a, c;
      SB::chunk_of(q, tid, a, c);
      dma16_at((c ^ SB::kswz(a)) * 16 < rest ? gB + offB[q] : outside_image, ldsB + q * 4096);
    }
    publish_barrier<0>();
#pragma unroll
    for (int ks = 0; ks < 2; ++ks) {
#pragma unroll
      for (int r = 0; r < TS::NREADS; ++r) T.read(0, 0, ks, r, fa[0], fb[0]);
      asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
      multiply_64<BM, BN, 0, LOADS_MAX>(acc, fa[0], fb[0], [](int) {}, 0, offA, gA);
    }
    asm volatile("s_nop 15\n\ts_nop 15\n\ts_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
  }

  int32_t *patch = reinterpret_cast<int32_t *>(smem) + wave * Patch16<FN>::WORDS;
  float *scales = reinterpret_cast<float *>(smem) + 4 * Patch16<FN>::WORDS;
  if (tid < BM) scales[tid] = row_scale;
  __syncthreads();
  const int64_t row0 = tile.first + T.wm * ET::WM, rows = tile.count - T.wm * ET::WM;
  const int64_t col0 = n0 + T.wn * (OUT / 2);
  if (rows <= 0 || col0 >= X.n) return;
  scales += T.wm * ET::WM;
  store_experts<FM, FN, GATED>(acc, X, tile.e, row0, rows, col0, lane, patch, scales);
}

template <int BM, int BN>
hipError_t launch_tile(const ExpertsArgs &X, hipStream_t s) {
  const int64_t out = X.gated ? BN / 2 : BN;
  const int64_t columns = (X.n + out - 1) / out, slots = X.rows / BM + (X.experts < X.rows ? X.experts : X.rows);
  const TileParams P{X, (int)columns};
  const void *kernel = X.gated ? reinterpret_cast<const void *>(experts_tile_kernel<BM, BN, 1>)
                               : reinterpret_cast<const void *>(experts_tile_kernel<BM, BN, 0>);
  const size_t lds = (size_t)Tile16<BM, BN>::LDS_BYTES;
  const hipError_t e = allow_dynamic_lds(kernel, lds);
  if (e != hipSuccess) return e;
  return launch_with(kernel, dim3((unsigned)((slots * columns + 7) / 8 * 8)), NTHREADS, lds, s, &P);
}

}  // namespace

// Pieces of 16 bytes, offsets of 32 bits, and a grid whose threads they hold.
bool experts_tile_eligible(const ExpertsArgs &X) {
  auto aligned = [](const void *p, int64_t ld) { return reinterpret_cast<uintptr_t>(p) % 16 == 0 && ld % 16 == 0; };
  const int64_t outputs = X.gated ? 2 * X.n : X.n;
  return X.k > 0 && X.k % 16 == 0 && aligned(X.A, X.lda) && aligned(X.B, X.ldb) && X.strideB % 16 == 0 && X.a_rows * X.lda < (int64_t)1 << 32 &&
         outputs * X.ldb < (int64_t)1 << 32 && (X.rows / 128 + X.experts + 1) * ((X.n + 63) / 64) < (int64_t)1 << 23;
}

hipError_t launch_experts_tile(const ExpertsArgs &X, bool large, hipStream_t s) {
  return large ? launch_tile<192, 256>(X, s) : launch_tile<128, 128>(X, s);
}

}  // namespace mip
