// The experts' products where there is little to do: 16 rows of one expert by 64 rows of its weights to a workgroup (with a gate 32 of the
// gate's and 32 of the others), its four waves taking k blocks of 128 in turn.
//
// The time is that of reading the weights, so what counts is how many loads are on their way: both operands go from memory into
// registers as v_mfma_i32_16x16x64_i8 takes them (16 rows x 64 bytes to a load), a block ahead, with no barrier before the four
// sums are added up.  Rows of any alignment, any k.  One token, eight experts' 1024 pairs of columns of 2048 (34 MB): 9.4 us, where 256
// rows of weights to a workgroup took 20; 256 rows over 64 experts' 2048 columns of 1024 (136 MB) 29.7 us, 4.6 TB/s.
#include "dma_common.h"
#include "epilogue16.h"
#include "experts.h"

namespace mip {

namespace {

struct SlimParams {
  ExpertsArgs X;
  int columns;  // column tiles
};

typedef __attribute__((address_space(1))) const uint8_t *global_bytes;
__device__ __forceinline__ v4i load16_at(const uint8_t *p) {
  return reinterpret_cast<const __attribute__((address_space(1))) unaligned_v4i *>((global_bytes)p)->v;
}

constexpr int SLIM_K = 128, FN = 4, PITCH = Patch16<FN>::PITCH;

template <int GATED>
__global__ __launch_bounds__(256) void experts_slim_kernel(SlimParams P) {
  constexpr int OUT = GATED ? 32 : 64;
  __shared__ __attribute__((aligned(16))) int32_t patch[4][16 * PITCH];
  const ExpertsArgs &X = P.X;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  int column = 0;
  const ExpertTile tile = expert_tile_of(X.starts, X.experts, X.rows, 16, P.columns, blockIdx.x, lane, &column);
  if (tile.count == 0) return;
  const int64_t n0 = (int64_t)column * OUT;
  const int mine = lane & 15, chunk = 16 * (lane >> 4);
  const uint8_t *a = X.A + expert_row(X, tile.first + (mine < tile.count ? mine : tile.count - 1)).at * X.lda;
  const uint8_t *b[FN];
#pragma unroll
  for (int f = 0; f < FN; ++f) {
    int64_t to = n0 + (GATED ? 16 * (f / 2) : 16 * f) + mine;
    to = to < X.n ? to : X.n - 1;
    b[f] = X.B + tile.e * X.strideB + (GATED && (f & 1) ? X.n + to : to) * X.ldb;
  }
  // the row whose sums this thread writes, four columns of it
  constexpr int QUADS = OUT / 4;
  const int row = tid / QUADS, quad = tid % QUADS;
  const float row_scale = row < tile.count ? expert_row(X, tile.first + (row < tile.count ? row : 0)).scale : 0.0f;

  struct Block {
    v4i a[2], b[2][FN];
  };
  const int64_t whole = X.k / SLIM_K;
  auto load = [&](int64_t t, Block &to) {
#pragma unroll
    for (int ks = 0; ks < 2; ++ks) {
      const int64_t at = t * SLIM_K + 64 * ks + chunk;
      to.a[ks] = load16_at(a + at);
#pragma unroll
      for (int f = 0; f < FN; ++f) to.b[ks][f] = load16_at(b[f] + at);
    }
  };
  v4i acc[FN] = {};
  auto multiply = [&](const Block &x) {
#pragma unroll
    for (int ks = 0; ks < 2; ++ks)
#pragma unroll
      for (int f = 0; f < FN; ++f) acc[f] = __builtin_amdgcn_mfma_i32_16x16x64_i8(x.b[ks][f], x.a[ks], acc[f], 0, 0, 0);
  };
  Block set[2];
  if (wave < whole) load(wave, set[0]);
  for (int64_t t = wave; t < whole; t += 8) {
    if (t + 4 < whole) load(t + 4, set[1]);
    __builtin_amdgcn_sched_barrier(0);
    multiply(set[0]);
    __builtin_amdgcn_sched_barrier(0);
    if (t + 8 < whole) load(t + 8, set[0]);
    __builtin_amdgcn_sched_barrier(0);
    if (t + 4 < whole) multiply(set[1]);
    __builtin_amdgcn_sched_barrier(0);
  }
  if (whole % 4 == wave && X.k % SLIM_K != 0) {  // what is left of k, as far as it goes
    Block rest;
#pragma unroll
    for (int ks = 0; ks < 2; ++ks) {
      const int64_t at = whole * SLIM_K + 64 * ks + chunk, left = X.k - at;
      const int64_t from = left > 0 ? at : 0;
      const int n = left > 16 ? 16 : (left > 0 ? (int)left : 0);
      rest.a[ks] = n == 16 ? load16_at(a + from) : load16_partial(a + from, n);
#pragma unroll
      for (int f = 0; f < FN; ++f) rest.b[ks][f] = n == 16 ? load16_at(b[f] + from) : load16_partial(b[f] + from, n);
    }
    multiply(rest);
  }
#pragma unroll
  for (int f = 0; f < FN; ++f) *reinterpret_cast<v4i *>(&patch[wave][mine * PITCH + 16 * f + 4 * (lane >> 4)]) = acc[f];
  __syncthreads();
  if (row >= 16 || row >= tile.count) return;
  const int at = row * PITCH + (GATED ? 32 * (quad / 4) + 4 * (quad % 4) : 4 * quad);
  auto sum = [&](int from) {
    v4i s = *reinterpret_cast<const v4i *>(&patch[0][from]);
#pragma unroll
    for (int w = 1; w < 4; ++w) s += *reinterpret_cast<const v4i *>(&patch[w][from]);
    return s;
  };
  const int64_t outputs = GATED ? 2 * X.n : X.n, col = n0 + 4 * quad, count = X.n - col;
  if (count <= 0) return;
  const LinearArgs L{X.C, nullptr, X.ldc, 0, nullptr, X.b_scales ? X.b_scales + tile.e * outputs : nullptr,
                     X.bias ? X.bias + tile.e * outputs : nullptr, X.act, X.type};
  const LinearColumns c = linear_columns(L, col, count);
  const v4i s = sum(at);
  v4f y;
#pragma unroll
  for (int e = 0; e < 4; ++e) y[e] = linear_value(s[e], row_scale, c.scale[e], c.bias[e]);
  switch (activation_kind(X.act)) {  // wave-uniform
    case 0: {
      const Activate<0> act = Activate<0>::of(X.act);
#pragma unroll
      for (int e = 0; e < 4; ++e) y[e] = act(y[e]);
      break;
    }
    case 1: {
      const Activate<1> act = Activate<1>::of(X.act);
#pragma unroll
      for (int e = 0; e < 4; ++e) y[e] = act(y[e]);
      break;
    }
    default: {
      const Activate<2> act = Activate<2>::of(X.act);
#pragma unroll
      for (int e = 0; e < 4; ++e) y[e] = act(y[e]);
    }
  }
  if (GATED) {
    const LinearColumns up = linear_columns(L, X.n + col, count);
    const v4i u = sum(at + 16);
#pragma unroll
    for (int e = 0; e < 4; ++e) y[e] *= linear_value(u[e], row_scale, up.scale[e], up.bias[e]);
  }
  const int64_t to = (tile.first + row) * X.ldc + col;
  if (count >= 4) {
    store_real4<false>(X.C, to, X.type, y);
  } else {
#pragma unroll
    for (int e = 0; e < 3; ++e)
      if (e < count) store_real(X.C, to + e, X.type, y[e]);
  }
}

}  // namespace

int64_t experts_slim_tiles(const ExpertsArgs &X) {
  const int64_t out = X.gated ? 32 : 64;
  return (X.rows / 16 + (X.experts < X.rows ? X.experts : X.rows)) * ((X.n + out - 1) / out);
}

// (a grid whose threads 32 bits hold)
bool experts_slim_eligible(const ExpertsArgs &X) {
  return (X.rows / 16 + X.experts + 1) < (int64_t)1 << 31 && (X.n + 31) / 32 < (int64_t)1 << 31 && experts_slim_tiles(X) < (int64_t)1 << 23;
}

hipError_t launch_experts_slim(const ExpertsArgs &X, hipStream_t s) {
  const int64_t out = X.gated ? 32 : 64;
  const SlimParams P{X, (int)((X.n + out - 1) / out)};
  const void *kernel = X.gated ? reinterpret_cast<const void *>(experts_slim_kernel<1>) : reinterpret_cast<const void *>(experts_slim_kernel<0>);
  return launch_with(kernel, dim3((unsigned)((experts_slim_tiles(X) + 7) / 8 * 8)), 256, 0, s, &P);
}

}  // namespace mip
