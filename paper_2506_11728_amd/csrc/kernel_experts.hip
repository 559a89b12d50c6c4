// The experts' products of rows sorted by expert, for operands of any alignment and any k:
//     C(p, j) = act(float(A(p) . B(e, j)) a_scale b_scale + bias)
// 64 MB rows of one expert by 128 rows of its weights (with a gate 64 of the gate's and 64 of the others) to a workgroup, k in blocks of 64
// through registers into LDS, two stages, v_mfma_i32_32x32x32_i8.  64 experts, 512 rows each on average, 1024 pairs of columns of 2048: 400 us, where rows that
// are aligned take 196 by direct loads.  A wave waits for 76 % of its life, the matrix units are busy for 16 % of the time: the loads bound it, 11 bytes
// a clock to a compute unit in unaligned pieces of 16; where k is no multiple of 16 the last piece of a row comes byte by byte.
#include "experts.h"
#include "dma_common.h"

namespace mip {

namespace {

constexpr int TN = 128, TK = 64;  // rows of B, k of a block

struct Params {
  ExpertsArgs X;
  int64_t slot0, column0;
};

template <int GATED, int MB>
__global__ __launch_bounds__(256) void experts_kernel(Params P) {
  constexpr int TM = 64 * MB;
  constexpr int OUT = GATED ? TN / 2 : TN, STAGE = (TM + TN) * TK;
  __shared__ __attribute__((aligned(16))) uint8_t lds[2 * STAGE];
  __shared__ float scales[TM];
  const ExpertsArgs &X = P.X;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const ExpertTile tile = expert_tile(X.starts, X.experts, X.rows, TM, P.slot0 + blockIdx.y, lane);
  if (tile.count == 0) return;
  const int64_t n0 = P.column0 + (int64_t)blockIdx.x * OUT;
  const int64_t outputs = GATED ? 2 * X.n : X.n;
  using SA = Stage<TM, true, TK>;
  using SB = Stage<TN, true, TK>;
  // this thread's pieces of A and of B
  constexpr int PIECES = SA::PER_THREAD + SB::PER_THREAD;
  const uint8_t *from[PIECES];
  int to[PIECES], deep[PIECES];
#pragma unroll
  for (int i = 0; i < SA::PER_THREAD; ++i) {
    int a, c;
    SA::chunk_of(i, tid, a, c);
    const ExpertRow r = expert_row(X, tile.first + (a < tile.count ? a : 0));
    if (c == 0) scales[a] = r.scale;
    from[i] = X.A + r.at * X.lda + 16 * c;
    to[i] = SA::lds_offset(a, c);
    deep[i] = 16 * c;
  }
#pragma unroll
  for (int i = 0; i < SB::PER_THREAD; ++i) {
    int a, c;
    SB::chunk_of(i, tid, a, c);
    // (with a gate, blocks of 32 of its columns and of the others in turn: a wave has both of a pair)
    int64_t column = n0 + (GATED ? a / 64 * 32 + a % 32 : a);
    if (column > X.n - 1) column = X.n - 1;
    if (GATED && (a / 32) % 2) column += X.n;
    from[SA::PER_THREAD + i] = X.B + tile.e * X.strideB + column * X.ldb + 16 * c;
    to[SA::PER_THREAD + i] = TM * TK + SB::lds_offset(a, c);
    deep[SA::PER_THREAD + i] = 16 * c;
  }
  v4i held[PIECES];
  auto load = [&](int64_t k0) {
#pragma unroll
    for (int i = 0; i < PIECES; ++i) {
      const int64_t left = X.k - k0 - deep[i];
      held[i] = left >= 16 ? load16(from[i] + k0) : load16_partial(from[i] + k0, left > 0 ? (int)left : 0);
    }
  };
  auto store = [&](int stage) {
#pragma unroll
    for (int i = 0; i < PIECES; ++i) *reinterpret_cast<v4i *>(lds + stage * STAGE + to[i]) = held[i];
  };
  const int wm = wave >> 1, wn = wave & 1;
  v16i acc[MB][2] = {};
  const int64_t blocks = (X.k + TK - 1) / TK;
  if (blocks > 0) {
    load(0);
    store(0);
  }
  __syncthreads();
  for (int64_t t = 0; t < blocks; ++t) {
    const bool more = t + 1 < blocks;
    if (more) load((t + 1) * TK);
    const uint8_t *sa = lds + (t & 1) * STAGE, *sb = sa + TM * TK;
#pragma unroll
    for (int ks = 0; ks < TK / 32; ++ks) {
      v4i a[MB], b[2];
#pragma unroll
      for (int i = 0; i < MB; ++i) a[i] = SA::fragment(sa, wm * (TM / 2) + 32 * i, ks, lane);
#pragma unroll
      for (int j = 0; j < 2; ++j) b[j] = SB::fragment(sb, wn * 64 + 32 * j, ks, lane);
#pragma unroll
      for (int i = 0; i < MB; ++i)
#pragma unroll
        for (int j = 0; j < 2; ++j) acc[i][j] = __builtin_amdgcn_mfma_i32_32x32x32_i8(b[j], a[i], acc[i][j], 0, 0, 0);
    }
    if (more) store((t + 1) & 1);
    __syncthreads();
  }
  // lane l has row l % 32 of a block and, of its quarter q, columns 8 q + 4 (l / 32) .. + 3
  const LinearArgs L{X.C, nullptr, X.ldc, 0, nullptr, X.b_scales ? X.b_scales + tile.e * outputs : nullptr,
                     X.bias ? X.bias + tile.e * outputs : nullptr, X.act, X.type};
  auto put = [&](auto act) {
#pragma unroll
    for (int i = 0; i < MB; ++i) {
      const int row = wm * (TM / 2) + 32 * i + (lane & 31);
      if (row >= tile.count) continue;
      const float row_scale = scales[row];
#pragma unroll
      for (int j = 0; j < (GATED ? 1 : 2); ++j) {
#pragma unroll
        for (int q = 0; q < 4; ++q) {
          const int64_t col = n0 + wn * (OUT / 2) + 32 * j + 8 * q + 4 * (lane >> 5), count = X.n - col;
          if (count <= 0) continue;
          const LinearColumns c = linear_columns(L, col, count);
          v4f y;
#pragma unroll
          for (int e = 0; e < 4; ++e) y[e] = act(linear_value(acc[i][j][4 * q + e], row_scale, c.scale[e], c.bias[e]));
          if (GATED) {
            const LinearColumns up = linear_columns(L, X.n + col, count);
#pragma unroll
            for (int e = 0; e < 4; ++e) y[e] *= linear_value(acc[i][1][4 * q + e], row_scale, up.scale[e], up.bias[e]);
          }
          const int64_t at = (tile.first + row) * X.ldc + col;
          if (count >= 4) {
            store_real4<false>(X.C, at, X.type, y);
          } else {
#pragma unroll
            for (int e = 0; e < 3; ++e)
              if (e < count) store_real(X.C, at + e, X.type, y[e]);
          }
        }
      }
    }
  };
  switch (activation_kind(X.act)) {  // wave-uniform
    case 0: put(Activate<0>::of(X.act)); break;
    case 1: put(Activate<1>::of(X.act)); break;
    default: put(Activate<2>::of(X.act)); break;
  }
}

template <int MB>
hipError_t launch_unaligned(const ExpertsArgs &X, hipStream_t s) {
  constexpr int TM = 64 * MB;
  // as many pieces as the experts' rows can be cut into; a grid has at most 65535 rows, and 2^32 - 1 threads a dimension
  const int64_t slots = X.rows / TM + (X.experts < X.rows ? X.experts : X.rows);
  const int64_t out = X.gated ? TN / 2 : TN, columns = (X.n + out - 1) / out;
  constexpr int64_t MOST_X = 1 << 20, MOST_Y = 65535;
  for (int64_t c = 0; c < columns; c += MOST_X)
    for (int64_t slot = 0; slot < slots; slot += MOST_Y) {
      Params P{X, slot, c * out};
      const dim3 grid((unsigned)(columns - c < MOST_X ? columns - c : MOST_X), (unsigned)(slots - slot < MOST_Y ? slots - slot : MOST_Y));
      const hipError_t e = launch_with(X.gated ? reinterpret_cast<const void *>(experts_kernel<1, MB>) : reinterpret_cast<const void *>(experts_kernel<0, MB>),
                                       grid, 256, 0, s, &P);
      if (e != hipSuccess) return e;
    }
  return hipSuccess;
}

}  // namespace

// The host knows the rows of all experts together and no expert's.  16 rows to a workgroup where an expert has few on average, or where so few
// workgroups result that the device would not be full with larger ones: each reads its weights once, by itself (64 experts' 1024
// pairs of columns of 2048, 8 rows each on average 57.3 us, with tiles 63.2; 12 rows 61.9 and 60.0; 16 rows 69.7 and 63.5; 8 experts' 4096 columns of 4096,
// 16 rows each 36.7 and 39.2, 32 rows 49.7 and 40.0).  Else tiles of rows that can be streamed: 128 x 128, two workgroups to a compute
// unit, so that one's first loads and write-back go on beside the other's products; under a long k of many rows 192 x 256, which load less for a product (8 experts,
// 512 rows each on average, 4096 columns of 11008: 216 us against 243; 5504: 124 and 126; 4096: 100 and 98; 2048: 62 and 54; 64 experts, 512 rows each,
// 1024 pairs of columns of 2048: 222 and 201).  The rule counts neither the columns nor the rounds of workgroups on the compute units, which decide
// where there are few: 384 rows each under 11008 take 216 with the large tiles and 190 with the small ones, 256 rows 128 and 165; 512 rows and 1024
// columns 98 and 82, under 4096 42 and 31.
hipError_t launch_experts(const ExpertsArgs &X, hipStream_t s) {
  const bool tiles = experts_tile_eligible(X);
  if ((X.rows <= 12 * (int64_t)X.experts || experts_slim_tiles(X) <= 1024) && experts_slim_eligible(X)) return launch_experts_slim(X, s);
  if (tiles) return launch_experts_tile(X, X.k >= 4096 && X.rows >= 384 * (int64_t)X.experts, s);
  return X.rows <= 64 * (int64_t)X.experts ? launch_unaligned<1>(X, s) : launch_unaligned<2>(X, s);
}

}  // namespace mip
