// Routing of tokens to experts, and the tokens' rows sorted by expert.
//
// A wave takes a token, its lanes the experts 64 i + lane.  What is compared:
//   the logits themselves where nothing is added to the scores and no sum of two of them is asked for: softmax and the
//   sigmoid rise with the logit, so the order of the exact scores is that of the logits, and it is exact;
//   else c = score + bias in float32.  Each is off by at most `wrong`; where two that are compared, of neighbours in
//   the order, or of the last group that stays and the first that does not, are nearer than twice that (and where they are
//   equal), the wave does the token again in float64.
// The largest of 64 lanes in six steps of data-parallel primitives, the expert by a ballot: the lowest index of equal ones.
//
// The rows by expert: 32 tokens to a workgroup, a word of 32 bits for each expert with a bit for each token that has it.
// A row's place among the workgroup's rows of its expert is the number of bits below its own, and the number of bits is
// what the workgroup adds to the expert: no atomic whose order shows.  A second kernel adds the workgroups' counts up and puts
// each row in its place; 32 tokens or fewer need no second one.
#include "layer_internal.h"
#include "real.h"

namespace mip {

namespace {

constexpr int TOKENS = 32;         // of a workgroup: the bits of a word
constexpr int THREADS = 1024;      // of both kernels
constexpr int WAVES = THREADS / 64;

template <int CTRL, int ROWS>
__device__ __forceinline__ float moved(float x, float other) {
  return __int_as_float(__builtin_amdgcn_update_dpp(__float_as_int(other), __float_as_int(x), CTRL, ROWS, 0xf, false));
}
constexpr int SHR_1 = 0x111, SHR_2 = 0x112, SHR_4 = 0x114, SHR_8 = 0x118, BROADCAST_15 = 0x142, BROADCAST_31 = 0x143;

__device__ __forceinline__ float last_lane(float x) { return __int_as_float(__builtin_amdgcn_readlane(__float_as_int(x), 63)); }
__device__ __forceinline__ float wave_most(float v) {
  v = __builtin_fmaxf(v, moved<SHR_1, 0xf>(v, v));
  v = __builtin_fmaxf(v, moved<SHR_2, 0xf>(v, v));
  v = __builtin_fmaxf(v, moved<SHR_4, 0xf>(v, v));
  v = __builtin_fmaxf(v, moved<SHR_8, 0xf>(v, v));
  v = __builtin_fmaxf(v, moved<BROADCAST_15, 0xa>(v, v));
  v = __builtin_fmaxf(v, moved<BROADCAST_31, 0xc>(v, v));
  return last_lane(v);
}
__device__ __forceinline__ float wave_sum(float v) {
  v += moved<SHR_1, 0xf>(v, 0.0f);
  v += moved<SHR_2, 0xf>(v, 0.0f);
  v += moved<SHR_4, 0xf>(v, 0.0f);
  v += moved<SHR_8, 0xf>(v, 0.0f);
  v += moved<BROADCAST_15, 0xa>(v, 0.0f);
  v += moved<BROADCAST_31, 0xc>(v, 0.0f);
  return last_lane(v);
}
__device__ __forceinline__ double wave_most(double v) {
#pragma unroll
  for (int d = 1; d < 64; d *= 2) {
    const double o = __shfl_xor(v, d);
    v = o > v ? o : v;
  }
  return v;
}
__device__ __forceinline__ double wave_sum(double v) {
#pragma unroll
  for (int d = 1; d < 64; d *= 2) v += __shfl_xor(v, d);
  return v;
}

constexpr float NONE = -__builtin_inff();

// What a wave knows of its token's choice: lane j holds the j-th.
struct Chosen {
  int id, count;  // count: how many there are (the same in every lane)
  float logit;
};

// The choice among c (-infinity: not to be chosen), which it uses up.  x: the logits.  near: what two numbers must be apart to be
// told apart, below 0: they are exact.  Returns whether they could not be.
template <typename K, int PER>
__device__ __forceinline__ bool choose(const RouteArgs &P, K (&c)[PER], const float (&x)[PER], K near, int lane, Chosen *chosen) {
  bool doubt = false;
  if (P.groups > 1) {
    K score = (K)NONE;  // of group `lane`
    for (int g = 0; g < P.groups; ++g) {
      const int first = g * (int)P.each.d, last = first + (int)P.each.d;
      K one = (K)NONE, two = (K)NONE;  // the lane's two largest of the group
#pragma unroll
      for (int i = 0; i < PER; ++i) {
        const int e = 64 * i + lane;
        const K v = e >= first && e < last ? c[i] : (K)NONE;
        two = v > one ? one : (v > two ? v : two);
        one = v > one ? v : one;
      }
      K sum = wave_most(one);
      if (P.best == 2 && sum > (K)NONE) {
        const uint64_t has = __ballot(one == sum);
        const K second = wave_most(lane == __builtin_ctzll(has) ? two : one);
        if (second > (K)NONE) sum += second;
      }
      score = lane == g ? sum : score;
    }
    uint64_t kept = 0;
    K least = (K)NONE;
    for (int r = 0; r < P.top_groups; ++r) {
      const K most = wave_most(score);
      if (!(most > (K)NONE)) break;
      const int g = __builtin_ctzll(__ballot(score == most));
      kept |= 1ull << g;
      score = lane == g ? (K)NONE : score;
      least = most;
    }
    const K next = wave_most(score);
    if (next > (K)NONE && least - next <= 4 * near) doubt = true;
#pragma unroll
    for (int i = 0; i < PER; ++i) {
      const unsigned e = 64 * i + lane, g = P.each.inv ? __umulhi(e, P.each.inv) : e / P.each.d;
      c[i] = (kept >> (g & 63)) & 1 ? c[i] : (K)NONE;
    }
  }
  K before = (K)NONE;
  int j = 0;
  for (; j <= P.top; ++j) {
    K own = c[0];
#pragma unroll
    for (int i = 1; i < PER; ++i) own = c[i] > own ? c[i] : own;
    const K most = wave_most(own);
    if (!(most > (K)NONE)) break;
    if (j > 0 && before - most <= near) doubt = true;
    if (j == P.top) break;
    before = most;
    bool found = false;
#pragma unroll
    for (int i = 0; i < PER; ++i) {
      if (found) continue;
      const uint64_t has = __ballot(c[i] == most);
      if (!has) continue;
      found = true;
      const int of = __builtin_ctzll(has);
      const float logit = __int_as_float(__builtin_amdgcn_readlane(__float_as_int(x[i]), of));
      if (lane == j) {
        chosen->id = 64 * i + of;
        chosen->logit = logit;
      }
      c[i] = lane == of ? (K)NONE : c[i];
    }
  }
  chosen->count = j;
  return doubt;
}

// One token: lane j < top gets its j-th expert (-1: none) and its weight.
template <int PER>
__device__ __forceinline__ void route_token(const RouteArgs &P, int type, int64_t token, int lane, int *id, float *weight) {
  float x[PER];
  float largest = NONE;
  bool lost = false;
#pragma unroll
  for (int i = 0; i < PER; ++i) {
    const int e = 64 * i + lane;
    x[i] = e < P.experts ? load_real(P.logits, token * P.ldl + e, type) : NONE;
    lost |= x[i] != x[i];
    largest = __builtin_fmaxf(largest, x[i]);
  }
  largest = wave_most(largest);
  if (!P.sigmoid) lost |= largest == __builtin_inff();
  Chosen chosen{-1, 0, 0.0f};
  const bool summed = P.groups > 1 && P.best == 2;
  float all = 0.0f;  // softmax: the sum of all exponentials
  if (!P.sigmoid && (!P.normalise || P.bias || summed)) {
    float sum = 0.0f;
#pragma unroll
    for (int i = 0; i < PER; ++i) sum += x[i] > NONE ? expf(x[i] - largest) : 0.0f;
    all = wave_sum(sum);
  }
  if (!P.bias && !summed) {
    if (!__ballot(lost)) {
      float c[PER];
#pragma unroll
      for (int i = 0; i < PER; ++i) c[i] = x[i];
      choose<float, PER>(P, c, x, -1.0f, lane, &chosen);
    }
  } else {
    float c[PER], size = 0.0f;
#pragma unroll
    for (int i = 0; i < PER; ++i) {
      const int e = 64 * i + lane;
      const float b = P.bias && e < P.experts ? P.bias[e] : 0.0f;
      lost |= b != b;
      if (P.sigmoid) c[i] = __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(-1.4426950408889634f * x[i]));
      else c[i] = __builtin_amdgcn_exp2f(1.4426950408889634f * (x[i] - largest)) * __builtin_amdgcn_rcpf(all);
      c[i] += b;
      c[i] = x[i] > NONE ? c[i] : NONE;
      size = c[i] > NONE ? __builtin_fmaxf(size, __builtin_fabsf(c[i])) : size;
    }
    if (!__ballot(lost)) {
      // Sigmoid: s (1 - s) |x| 2^-23 of the exponential's argument (below 2^-25), two units of the sum's and the reciprocal's last place
      // of a number of at most 1.  Softmax: the largest score times what the argument (|t| e^t 2^-23), the sum (a chain of at most 22
      // additions, and its terms' arguments, 7 2^-23 of it) and the reciprocal are off, below 2^-18 of it together.  The addition of the bias.
      const float most = wave_most(size);
      const float wrong = (P.sigmoid ? 0x1p-22f : 0x1p-18f * __builtin_amdgcn_rcpf(all)) + most * 0x1p-24f;
      if (choose<float, PER>(P, c, x, 2.0f * wrong, lane, &chosen)) {
        double d[PER], sum = 0.0;
#pragma unroll
        for (int i = 0; i < PER; ++i) {
          d[i] = P.sigmoid ? 1.0 / (1.0 + exp(-(double)x[i])) : (x[i] > NONE ? exp((double)x[i] - (double)largest) : 0.0);
          sum += d[i];
        }
        if (!P.sigmoid) sum = wave_sum(sum);
#pragma unroll
        for (int i = 0; i < PER; ++i) {
          const int e = 64 * i + lane;
          const float b = P.bias && e < P.experts ? P.bias[e] : 0.0f;
          if (!P.sigmoid) d[i] /= sum;
          d[i] = x[i] > NONE && b > NONE ? d[i] + (double)b : (double)NONE;
        }
        chosen = Chosen{-1, 0, 0.0f};
        choose<double, PER>(P, d, x, -1.0, lane, &chosen);
      }
    }
  }
  // the weights, of lane j the j-th
  const bool any = lane < chosen.count;
  float w = 0.0f;
  if (__ballot(lost)) {
    w = __builtin_nanf("");
  } else if (chosen.count > 0) {
    const float top = wave_most(any ? chosen.logit : NONE);
    // (far below zero the sigmoid is its exponential to the last bit of a float64, and may pass float32)
    const bool ratio = P.normalise && (!P.sigmoid || top < -40.0f);
    float s;
    if (P.sigmoid && !ratio) s = chosen.logit < -40.0f ? expf(chosen.logit) : __fdiv_rn(1.0f, 1.0f + expf(-chosen.logit));
    else s = expf(chosen.logit - (ratio ? top : largest));
    if (!any) s = 0.0f;
    const float over = P.normalise ? wave_sum(s) : (P.sigmoid ? 1.0f : all);
    w = any ? P.scale * __fdiv_rn(s, over) : 0.0f;
  }
  *id = any ? chosen.id : -1;
  *weight = w;
}

// Sums of what lies before this thread's number among those of the workgroup.  All threads call it.
__device__ __forceinline__ int before_in_group(int n, int *waves, int tid) {
  const int lane = tid & 63, wave = tid >> 6;
  int sum = n;
#pragma unroll
  for (int d = 1; d < 64; d *= 2) {
    const int o = __shfl_up(sum, d);
    if (lane >= d) sum += o;
  }
  if (lane == 63) waves[wave] = sum;
  __syncthreads();
  int first = 0;
#pragma unroll
  for (int w = 0; w < WAVES; ++w) first += w < wave ? waves[w] : 0;
  __syncthreads();
  return first + sum - n;
}

template <int PER>
__global__ __launch_bounds__(THREADS) void route_kernel(RouteArgs P, int type) {
  __shared__ uint32_t has[64 * PER];
  __shared__ int ids[TOKENS * MOST_CHOSEN];
  __shared__ int waves[WAVES], first[64 * PER];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int64_t token0 = (int64_t)blockIdx.x * TOKENS;
  const int tokens = (int)(P.tokens - token0 < TOKENS ? P.tokens - token0 : TOKENS);
  if (P.starts) {
    for (int e = tid; e < 64 * PER; e += THREADS) has[e] = 0;
    __syncthreads();
  }
  for (int t = wave; t < tokens; t += WAVES) {
    int id;
    float w;
    route_token<PER>(P, type, token0 + t, lane, &id, &w);
    if (lane < P.top) {
      P.ids[(token0 + t) * P.top + lane] = id;
      P.weights[(token0 + t) * P.top + lane] = w;
      ids[t * P.top + lane] = id;
      if (P.starts && id >= 0) atomicOr(&has[id], 1u << t);
    }
  }
  if (!P.starts) return;
  __syncthreads();
  const int rows = tokens * P.top;
  if (P.counts) {  // for the second kernel
    const int padded = (P.experts + 3) & ~3;
    for (int e = tid; e < padded; e += THREADS)
      P.counts[(int64_t)blockIdx.x * padded + e] = e < P.experts ? (uint8_t)__popc(has[e]) : 0;
    for (int i = tid; i < rows; i += THREADS) {
      const int id = ids[i];
      if (id >= 0) P.ranks[token0 * P.top + i] = (uint8_t)__popc(has[id] & ((1u << (i / P.top)) - 1));
    }
    return;
  }
  const int mine = tid < P.experts ? __popc(has[tid]) : 0;
  const int from = before_in_group(mine, waves, tid);
  if (tid < P.experts) {
    first[tid] = from;
    P.starts[tid] = from;
    if (tid == P.experts - 1) P.starts[P.experts] = from + mine;
  }
  __syncthreads();
  for (int i = tid; i < rows; i += THREADS) {
    const int id = ids[i];
    const int at = id < 0 ? -1 : first[id] + __popc(has[id] & ((1u << (i / P.top)) - 1));
    if (P.places) P.places[i] = at;
    if (P.order && at >= 0) P.order[at] = i;
  }
}

// The second kernel: workgroup b puts the rows of the `blocks` blocks of tokens from b * blocks on in their places.
constexpr int AT_ONCE = 8;  // blocks whose first places are in LDS together
__global__ __launch_bounds__(THREADS) void place_kernel(RouteArgs P, int64_t all_blocks, int blocks) {
  __shared__ int total[MOST_EXPERTS], before[MOST_EXPERTS], waves[WAVES];
  __shared__ int first[AT_ONCE][MOST_EXPERTS];
  const int tid = threadIdx.x, padded = (P.experts + 3) & ~3, words = padded / 4;
  const int64_t block0 = (int64_t)blockIdx.x * blocks;
  const int64_t block1 = block0 + blocks < all_blocks ? block0 + blocks : all_blocks;
  total[tid] = before[tid] = 0;
  __syncthreads();
  // four experts to a thread, the blocks among as many threads as there are for it
  int wide = 1;
  while (wide < words) wide *= 2;
  const int word = tid & (wide - 1), part = tid / wide, parts = THREADS / wide;
  if (word < words) {
    const uint32_t *counts = reinterpret_cast<const uint32_t *>(P.counts);
    int sum[4] = {0, 0, 0, 0}, sum_before[4] = {0, 0, 0, 0};
#pragma unroll 8
    for (int64_t b = part; b < all_blocks; b += parts) {
      const uint32_t four = counts[b * words + word];
      const uint32_t mask = b < block0 ? ~0u : 0u;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        sum[i] += (four >> (8 * i)) & 0xff;
        sum_before[i] += ((four & mask) >> (8 * i)) & 0xff;
      }
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      atomicAdd(&total[4 * word + i], sum[i]);
      atomicAdd(&before[4 * word + i], sum_before[i]);
    }
  }
  __syncthreads();
  const int mine = tid < P.experts ? total[tid] : 0;
  const int from = before_in_group(mine, waves, tid);
  if (blockIdx.x == 0 && tid < P.experts) {
    P.starts[tid] = from;
    if (tid == P.experts - 1) P.starts[P.experts] = from + mine;
  }
  int next = from + before[tid];  // the first place of expert tid's rows in the next block
  for (int64_t b0 = block0; b0 < block1; b0 += AT_ONCE) {
    const int count = (int)(block1 - b0 < AT_ONCE ? block1 - b0 : AT_ONCE);
    if (tid < P.experts) {
#pragma unroll
      for (int b = 0; b < AT_ONCE; ++b) {
        if (b >= count) break;
        first[b][tid] = next;
        next += P.counts[(b0 + b) * padded + tid];
      }
    }
    __syncthreads();
    const int64_t row0 = b0 * TOKENS * P.top, end = (b0 + count) * TOKENS < P.tokens ? (b0 + count) * TOKENS * P.top : P.tokens * P.top;
    for (int64_t i = row0 + tid; i < end; i += THREADS) {
      const int id = P.ids[i];
      const int at = id < 0 ? -1 : first[(int)(i - row0) / (TOKENS * P.top)][id] + P.ranks[i];
      if (P.places) P.places[i] = at;
      if (P.order && at >= 0) P.order[at] = (int)i;
    }
    __syncthreads();
  }
}

size_t counts_bytes(int64_t tokens, int64_t experts) {
  return (size_t)((((tokens + TOKENS - 1) / TOKENS) * ((experts + 3) & ~3) + 15) & ~(int64_t)15);
}


}  // namespace

size_t route_scratch(int64_t tokens, int64_t experts, int64_t top) {
  return tokens <= TOKENS ? 0 : counts_bytes(tokens, experts) + (size_t)(tokens * top);
}

hipError_t launch_route(RouteArgs P, int type, void *ws, hipStream_t s) {
  const int64_t blocks = P.tokens > TOKENS ? (P.tokens + TOKENS - 1) / TOKENS : 1;
  if (P.starts && blocks > 1) {
    P.counts = static_cast<uint8_t *>(ws);
    P.ranks = P.counts + counts_bytes(P.tokens, P.experts);
  }
  void (*kernel)(RouteArgs, int) = P.experts <= 64 ? route_kernel<1> : P.experts <= 128 ? route_kernel<2> : P.experts <= 256 ? route_kernel<4>
                                   : P.experts <= 512 ? route_kernel<8> : route_kernel<16>;
  void *list[] = {&P, &type};
  hipError_t e = hipLaunchKernel(reinterpret_cast<const void *>(kernel), dim3((unsigned)blocks), dim3(THREADS), list, 0, s);
  if (e == hipSuccess && P.counts) {
    const int64_t groups = blocks / AT_ONCE < 256 ? (blocks + AT_ONCE - 1) / AT_ONCE : 256;
    int64_t all = blocks;
    int each = (int)((blocks + groups - 1) / groups);
    void *more[] = {&P, &all, &each};
    e = hipLaunchKernel(reinterpret_cast<const void *>(place_kernel), dim3((unsigned)((blocks + each - 1) / each)), dim3(THREADS), more, 0, s);
  }
  if (e != hipSuccess) (void)hipGetLastError();  // (the caller gets it; the next check of theirs must not find it again)
  return e;
}

}  // namespace mip
