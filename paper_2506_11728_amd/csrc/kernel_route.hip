// Routing of tokens to experts, and the tokens' rows sorted by expert.
//
// Up to 32 tokens a wave takes a token, its lanes the experts 64 i + lane (route_token); of more a row of 16 lanes takes one, four to a wave, where
// 16 lanes hold the groups, of up to 512 experts with up to 15 chosen (route_row).  What is compared:
//   the logits themselves where nothing is added to the scores and no sum of two of them is asked for: softmax and the
//   sigmoid rise with the logit, so the order of the exact scores is that of the logits, and it is exact;
//   else c = score + bias in float32.  Each is off by at most `wrong`; where two that are compared, of neighbours in
//   the order, or of the last group that stays and the first that does not, are nearer than twice that (and where they are
//   equal), float64 decides: a wave does its token again, a row of 16 lanes puts those chosen and the next one in order, one to a lane, and
//   leaves to the wave a token with a group, or one more expert, in doubt.
// The largest of 64 lanes in six steps of data-parallel primitives, the expert by a ballot (of 16 in four steps each): the lowest index of equal ones.
//
// 8192 tokens, 8 of 256 experts, sigmoid, bias, 4 of 8 groups: 12.2 us and 6.7 for the places; vector instructions issue in 56 and 58 % of the
// clocks in which a compute unit has waves, the rest is waiting (a wave waits for half its life).
//
// The rows by expert: 32 tokens to a workgroup, a word of 32 bits for each expert with a bit for each token that has it.
// A row's place among the workgroup's rows of its expert is the number of bits below its own, and the number of bits is
// what the workgroup adds to the expert: no atomic whose order shows.  A second kernel adds the workgroups' counts up and puts
// each row in its place; 32 tokens or fewer need no second one.
#include "layer_internal.h"
#include "real.h"
#include "wave.h"

namespace mip {

namespace {

constexpr int TOKENS = 32;         // of a workgroup: the bits of a word
constexpr int THREADS = 1024;      // of both kernels
constexpr int WAVES = THREADS / 64;

template <int CTRL, int ROWS>
__device__ __forceinline__ double moved(double x, double other) {
  const long long v = __double_as_longlong(x), o = __double_as_longlong(other);
  const int lo = __builtin_amdgcn_update_dpp((int)o, (int)v, CTRL, ROWS, 0xf, false);
  const int hi = __builtin_amdgcn_update_dpp((int)(o >> 32), (int)(v >> 32), CTRL, ROWS, 0xf, false);
  return __longlong_as_double((long long)hi << 32 | (unsigned)lo);
}
__device__ __forceinline__ double last_lane(double x) {
  const long long v = __double_as_longlong(x);
  const int lo = __builtin_amdgcn_readlane((int)v, 63), hi = __builtin_amdgcn_readlane((int)(v >> 32), 63);
  return __longlong_as_double((long long)hi << 32 | (unsigned)lo);
}
__device__ __forceinline__ double wave_most(double v) {
  auto larger = [](double a, double b) { return a > b ? a : b; };
  v = larger(v, moved<SHR_1, 0xf>(v, v));
  v = larger(v, moved<SHR_2, 0xf>(v, v));
  v = larger(v, moved<SHR_4, 0xf>(v, v));
  v = larger(v, moved<SHR_8, 0xf>(v, v));
  v = larger(v, moved<BROADCAST_15, 0xa>(v, v));
  return last_lane(larger(v, moved<BROADCAST_31, 0xc>(v, v)));
}
__device__ __forceinline__ double wave_sum(double v) {
  v += moved<SHR_1, 0xf>(v, 0.0);
  v += moved<SHR_2, 0xf>(v, 0.0);
  v += moved<SHR_4, 0xf>(v, 0.0);
  v += moved<SHR_8, 0xf>(v, 0.0);
  v += moved<BROADCAST_15, 0xa>(v, 0.0);
  return last_lane(v + moved<BROADCAST_31, 0xc>(v, 0.0));
}

constexpr float NONE = -__builtin_inff();

// The score of a chosen expert that is divided by the sum of them all or, where the chosen are, of theirs: softmax without its denominator, and for
// weights that add up to one times a power of e, the same for the whole token, that leaves the largest of the chosen (of logit `top`) at 1 / 2 or more.
// So float32 holds, of shares of 2^-126 and more, all bits: a sigmoid is e^l / (1 + e^l) below zero, and times e^-top there e^(l - top) / (1 + e^l).
__device__ __forceinline__ float to_weigh(const RouteArgs &P, float logit, float top, float largest) {
  if (!P.sigmoid) return expf(logit - (P.normalise ? top : largest));
  const float from = P.normalise ? __builtin_fminf(top, 0.0f) : 0.0f;
  return __fdiv_rn(logit < 0.0f ? expf(logit - from) : 1.0f, 1.0f + expf(-__builtin_fabsf(logit)));
}

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

// One token: lane j < top gets its j-th expert (-1: none) and its weight.  doubted: float32 has been tried.
template <int PER>
__device__ __forceinline__ void route_token(const RouteArgs &P, int type, int64_t token, int lane, bool doubted, int *id, float *weight) {
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
      if (doubted || choose<float, PER>(P, c, x, 2.0f * wrong, lane, &chosen)) {
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
    const float s = any ? to_weigh(P, chosen.logit, top, largest) : 0.0f;
    const float over = P.normalise ? wave_sum(s) : (P.sigmoid ? 1.0f : all);
    w = any ? P.scale * __fdiv_rn(s, over) : 0.0f;
  }
  *id = any ? chosen.id : -1;
  *weight = w;
}

// ---- four tokens to a wave ----
// A row of 16 lanes takes a token, a lane PER of its experts: what is done once for a token, the steps of a
// maximum above all, is done for four at a time.

template <int BY>
__device__ __forceinline__ float turned(float x) { return __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(x), 0x120 + BY, 0xf, 0xf, true)); }
template <int BY>
__device__ __forceinline__ int turned(int x) { return __builtin_amdgcn_update_dpp(0, x, 0x120 + BY, 0xf, 0xf, true); }
__device__ __forceinline__ float row_most(float v) {
  v = __builtin_fmaxf(v, turned<8>(v));
  v = __builtin_fmaxf(v, turned<4>(v));
  v = __builtin_fmaxf(v, turned<2>(v));
  return __builtin_fmaxf(v, turned<1>(v));
}
__device__ __forceinline__ int row_least(int v) {
  v = min(v, turned<8>(v));
  v = min(v, turned<4>(v));
  v = min(v, turned<2>(v));
  return min(v, turned<1>(v));
}
__device__ __forceinline__ float row_sum(float v) {
  v += turned<8>(v);
  v += turned<4>(v);
  v += turned<2>(v);
  return v + turned<1>(v);
}
__device__ __forceinline__ bool any_of_row(bool b, int lane) { return ((__ballot(b) >> (lane & 48)) & 0xffff) != 0; }

// How many of the row's other lanes have a larger v, or the same and a smaller number.
template <int D = 1>
__device__ __forceinline__ int larger_in_row(float v, int number) {
  if constexpr (D > 15) {
    return 0;
  } else {
    const float o = turned<D>(v);
    const int n = turned<D>(number);
    return (o > v || (o == v && n < number) ? 1 : 0) + larger_in_row<D + 1>(v, number);
  }
}

template <int BY>
__device__ __forceinline__ double turned(double x) {
  return moved<0x120 + BY, 0xf>(x, x);
}
template <int D = 1>
__device__ __forceinline__ int larger_in_row(double v, int number) {
  if constexpr (D > 15) {
    return 0;
  } else {
    const double o = turned<D>(v);
    const int n = turned<D>(number);
    return (o > v || (o == v && n < number) ? 1 : 0) + larger_in_row<D + 1>(v, number);
  }
}

// Lane q < top (at most 15) gets its token's q-th expert (-1: none) and its weight; returns whether the token has to be done again, in float64.
// P.span lanes to a group, a power of two; their experts are neighbours, and the last of a group's lanes may have fewer or none.
template <int PER>
__device__ __forceinline__ bool route_row(const RouteArgs &P, int type, int64_t token, int lane, int *id, float *weight) {
  const int q = lane & 15, span = P.span, group = q / span, part = q % span * PER;
  const int each = (int)P.each.d, first = group * each + part;
  const int own_experts = group < P.groups ? (each - part < PER ? each - part : PER) : 0;  // (none, or below)
  const int64_t at = token * P.ldl + first;
  float x[PER], bias[PER];
  bool lost = false;
  float largest = NONE;
#pragma unroll
  for (int i = 0; i < PER; i += 4) {
    if (i + 4 <= own_experts) {
      const v4f four = load_real4(P.logits, at + i, type);
      const v4f more = P.bias ? load_real4(P.bias, first + i, REAL_F32) : v4f{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        x[i + k] = four[k];
        bias[i + k] = more[k];
      }
    } else {
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        const bool here = i + k < own_experts;
        x[i + k] = here ? load_real(P.logits, at + i + k, type) : NONE;
        bias[i + k] = here && P.bias ? P.bias[first + i + k] : 0.0f;
      }
    }
  }
#pragma unroll
  for (int i = 0; i < PER; ++i) {
    lost |= x[i] != x[i];
    largest = __builtin_fmaxf(largest, x[i]);
  }
  largest = row_most(largest);
  if (!P.sigmoid) lost |= largest == __builtin_inff();
  const bool summed = P.groups > 1 && P.best == 2, scored = P.bias || summed;
  float all = 1.0f;  // softmax: the sum of all exponentials
  if (!P.sigmoid && (!P.normalise || scored)) {
    float sum = 0.0f;
#pragma unroll
    for (int i = 0; i < PER; ++i) sum += x[i] > NONE ? expf(x[i] - largest) : 0.0f;
    all = row_sum(sum);
  }
  float c[PER], near = -1.0f;
  if (!scored) {
#pragma unroll
    for (int i = 0; i < PER; ++i) c[i] = x[i];
  } else {
    const float over = P.sigmoid ? 1.0f : __builtin_amdgcn_rcpf(all);
    float size = 0.0f;
#pragma unroll
    for (int i = 0; i < PER; ++i) {
      lost |= bias[i] != bias[i];
      if (P.sigmoid) c[i] = __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(-1.4426950408889634f * x[i]));
      else c[i] = __builtin_amdgcn_exp2f(1.4426950408889634f * (x[i] - largest)) * over;
      c[i] += bias[i];
      c[i] = x[i] > NONE ? c[i] : NONE;
      size = c[i] > NONE ? __builtin_fmaxf(size, __builtin_fabsf(c[i])) : size;
    }
    // As in route_token, but for the chain of softmax's sum: up to 31 additions in a lane and 4 over the row, 35 2^-24; the terms and their arguments
    // 14 2^-24, the score's own argument, exponential, reciprocal and product below 6: 55 of the 64 2^-24 that 2^-18 are.
    near = 2.0f * ((P.sigmoid ? 0x1p-22f : 0x1p-18f * over) + row_most(size) * 0x1p-24f);
  }
  lost = any_of_row(lost, lane);
  bool doubt = false;
  if (P.groups > 1) {
    float one = c[0], two = NONE;
#pragma unroll
    for (int i = 1; i < PER; ++i) {
      two = __builtin_fmaxf(two, __builtin_fminf(one, c[i]));
      one = __builtin_fmaxf(one, c[i]);
    }
    auto join = [&](float o1, float o2) {
      two = __builtin_fmaxf(__builtin_fmaxf(two, o2), __builtin_fminf(one, o1));
      one = __builtin_fmaxf(one, o1);
    };
    // (lane ^ 1, ^ 2; then the other half of eight lanes, whose quarters have the same by now: of more than one group none has 16 lanes)
    if (span > 1) join(moved<0xb1, 0xf>(one, one), moved<0xb1, 0xf>(two, two));
    if (span > 2) join(moved<0x4e, 0xf>(one, one), moved<0x4e, 0xf>(two, two));
    if (span > 4) join(moved<0x141, 0xf>(one, one), moved<0x141, 0xf>(two, two));
    const float score = one > NONE ? (P.best == 2 && two > NONE ? one + two : one) : NONE;
    const int ahead = larger_in_row(score, group);  // (by all lanes: one that is switched off has nothing to give)
    const bool kept = score > NONE && ahead < P.top_groups * span;
    const float least = -row_most(kept ? -score : NONE), next = row_most(kept ? NONE : score);
    doubt = next > NONE && least - next <= 4.0f * near;
#pragma unroll
    for (int i = 0; i < PER; ++i) c[i] = kept ? c[i] : NONE;
  }
  int mine = -1;
  float before = NONE;
  bool unsure = false;  // of the order of those that are chosen, and of the next one
  auto most_left = [&]() {
    float own = c[0];
#pragma unroll
    for (int i = 1; i < PER; ++i) own = __builtin_fmaxf(own, c[i]);
    return row_most(own);
  };
  const int turns = P.top + (scored ? 1 : 0);
  for (int j = 0; j < turns; ++j) {
    const float most = most_left();
    const bool found = most > NONE;
    unsure |= j > 0 && found && before - most <= near;
    before = most;
    int key = PER;
#pragma unroll
    for (int i = PER - 1; i >= 0; --i) key = c[i] == most ? i : key;
    const int winner = row_least(key < PER ? first + key : 1 << 20);
    if (q == j && found) mine = winner;
    const int local = winner - first;
#pragma unroll
    for (int i = 0; i < PER; ++i) c[i] = local == i ? NONE : c[i];
  }
  unsure = unsure && !lost;
  if (__ballot(unsure)) {
    // Those that were chosen and the next one, in the order of their exact c: one to a lane.  (Where one more is as near, it is all done again.)
    const float most = most_left();
    doubt |= unsure && most > NONE && before - most <= near;
    double sum = 1.0;
    if (!P.sigmoid) {
      sum = 0.0;
#pragma unroll
      for (int i = 0; i < PER; ++i) sum += x[i] > NONE ? exp((double)x[i] - (double)largest) : 0.0;
      sum += turned<8>(sum);
      sum += turned<4>(sum);
      sum += turned<2>(sum);
      sum += turned<1>(sum);
    }
    double exact = (double)NONE;
    const int number = mine >= 0 ? mine : (1 << 20) + q;
    if (mine >= 0 && !lost) {
      const double l = load_real(P.logits, token * P.ldl + mine, type);
      exact = P.sigmoid ? 1.0 / (1.0 + exp(-l)) : exp(l - (double)largest) / sum;
      if (P.bias) exact += (double)P.bias[mine];
    }
    const int rank = larger_in_row(exact, number);
    const int sorted = __builtin_amdgcn_ds_permute(((lane & 48) + rank) * 4, number);
    if (unsure) mine = sorted < (1 << 20) ? sorted : -1;
  }
  if (q >= P.top) mine = -1;
  if (lost) {
    mine = -1;
    doubt = false;
  }
  const bool any = mine >= 0;
  const float logit = any ? load_real(P.logits, token * P.ldl + mine, type) : NONE;
  const float top = row_most(logit);
  const float s = any ? to_weigh(P, logit, top, largest) : 0.0f;
  const float over = P.normalise ? row_sum(s) : (P.sigmoid ? 1.0f : all);
  *id = mine;
  *weight = lost ? __builtin_nanf("") : (any ? P.scale * __fdiv_rn(s, over) : 0.0f);
  return doubt;
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

// FOUR: four tokens to a wave, for more than 32 tokens.
template <int PER, bool FOUR>
__global__ __launch_bounds__(FOUR ? 512 : THREADS) void route_kernel(RouteArgs P, int type) {
  constexpr int OWN = FOUR ? 512 : THREADS;  // threads
  __shared__ uint32_t has[64 * PER];
  __shared__ int ids[TOKENS * MOST_CHOSEN];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int64_t token0 = (int64_t)blockIdx.x * TOKENS;
  const int tokens = (int)(P.tokens - token0 < TOKENS ? P.tokens - token0 : TOKENS);
  if (P.starts) {
    for (int e = tid; e < 64 * PER; e += OWN) has[e] = 0;
    __syncthreads();
  }
  // lane j has the j-th choice of token t of the workgroup
  auto put = [&](int t, int j, int id, float w) {
    P.ids[(token0 + t) * P.top + j] = id;
    P.weights[(token0 + t) * P.top + j] = w;
    ids[t * P.top + j] = id;
    if (P.starts && id >= 0) atomicOr(&has[id], 1u << t);
  };
  int id;
  float w;
  if constexpr (FOUR) {
    const int t0 = 4 * wave, t = t0 + (lane >> 4);
    if (t0 < tokens) {
      const bool again = route_row<4 * PER>(P, type, token0 + (t < tokens ? t : tokens - 1), lane, &id, &w);
      const uint64_t rows = __ballot(again && t < tokens);
      if (t < tokens && !again && (lane & 15) < P.top) put(t, lane & 15, id, w);
      for (int r = 0; r < 4; ++r) {
        if (!((rows >> (16 * r)) & 1)) continue;
        route_token<PER>(P, type, token0 + t0 + r, lane, true, &id, &w);
        if (lane < P.top) put(t0 + r, lane, id, w);
      }
    }
  } else {
    for (int t = wave; t < tokens; t += WAVES) {
      route_token<PER>(P, type, token0 + t, lane, false, &id, &w);
      if (lane < P.top) put(t, lane, id, w);
    }
  }
  if (!P.starts) return;
  __syncthreads();
  const int rows = tokens * P.top;
  if (P.counts) {  // for the second kernel
    const int padded = (P.experts + 3) & ~3;
    for (int e = tid; e < padded; e += OWN)
      P.counts[(int64_t)blockIdx.x * padded + e] = e < P.experts ? (uint8_t)__popc(has[e]) : 0;
    for (int i = tid; i < rows; i += OWN) {
      const int id = ids[i];
      if (id >= 0) P.ranks[token0 * P.top + i] = (uint8_t)__popc(has[id] & ((1u << (i / P.top)) - 1));
    }
    return;
  }
  if constexpr (!FOUR) {
    __shared__ int waves[WAVES], first[64 * PER];
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
}

// The second kernel: workgroup b puts the rows of the `blocks` blocks of tokens from b * blocks on in their places.
__global__ __launch_bounds__(THREADS) void place_kernel(RouteArgs P, int64_t all_blocks, int blocks) {
  __shared__ int total[MOST_EXPERTS], before[MOST_EXPERTS], waves[WAVES];
  __shared__ int first[MOST_EXPERTS];
  const int tid = threadIdx.x, padded = (P.experts + 3) & ~3, words = padded / 4;
  const int64_t block0 = (int64_t)blockIdx.x * blocks;
  const int64_t block1 = block0 + blocks < all_blocks ? block0 + blocks : all_blocks;
  // what is needed of a block of tokens behind the sums, sent for before them: a row to a thread, and an expert's count
  static_assert(TOKENS * MOST_CHOSEN <= THREADS && MOST_EXPERTS <= THREADS, "one of each to a thread");
  const int rows = TOKENS * P.top;
  int id = -1, rank = 0, count = 0;
  auto fetch = [&](int64_t b) {
    const int64_t i = b * rows + tid;
    id = -1;
    if (tid < rows && i < P.tokens * P.top) {
      id = P.ids[i];
      rank = P.ranks[i];
    }
    count = tid < P.experts ? P.counts[b * padded + tid] : 0;
  };
  fetch(block0);
  total[tid] = before[tid] = 0;
  __syncthreads();
  // four experts to a thread, the blocks among as many threads as there are for it
  int wide = 1;
  while (wide < words) wide *= 2;
  const int word = tid & (wide - 1), part = tid / wide, parts = THREADS / wide;
  if (word < words) {
    const uint32_t *counts = reinterpret_cast<const uint32_t *>(P.counts);
    int sum[4] = {0, 0, 0, 0}, sum_before[4] = {0, 0, 0, 0};
    for (int64_t b0 = part; b0 < all_blocks; b0 += 16 * parts) {
      uint32_t four[16];  // (all on their way before the first is used)
#pragma unroll
      for (int u = 0; u < 16; ++u) four[u] = b0 + u * parts < all_blocks ? counts[(b0 + u * parts) * words + word] : 0u;
#pragma unroll
      for (int u = 0; u < 16; ++u) {
        const uint32_t earlier = b0 + u * parts < block0 ? four[u] : 0u;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          sum[i] += (four[u] >> (8 * i)) & 0xff;
          sum_before[i] += (earlier >> (8 * i)) & 0xff;
        }
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
  for (int64_t b = block0; b < block1; ++b) {
    first[tid] = next;
    next += count;
    __syncthreads();
    const int64_t i = b * rows + tid;
    const int at = id < 0 ? -1 : first[id] + rank;
    const bool here = tid < rows && i < P.tokens * P.top;
    if (b + 1 < block1) fetch(b + 1);
    if (here && P.places) P.places[i] = at;
    if (here && P.order && at >= 0) P.order[at] = (int)i;
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
  // Four tokens to a wave where the groups fit 16 lanes: without the places, 517 tokens, 4 of 60 experts, softmax 8.6 -> 3.9 us; 8192 tokens, 8 of
  // 256 experts, softmax 14.7 -> 7.2, sigmoid and bias 18.3 -> 9.6, by groups as well 39.7 -> 12.9.  Up to 32 tokens a token has a wave of its own,
  // and the rows by expert are put in place by the same launch, which the form of four leaves to a second one.  With the places, 8 of 128 experts,
  // softmax, tokens 8, 16, 32 and 33 (the first in two launches): 6.0, 7.8, 12.8, 9.8 us; 8 of 256, sigmoid, bias, 4 of 8 groups: 13.0, 18.8, 33.9,
  // 14.2.  So it is the sooner done up to some 20 tokens without groups and 8 with them; from there to 32 it is not, and the limit is what 32 bits hold.
  int per = P.experts <= 64 ? 1 : P.experts <= 128 ? 2 : P.experts <= 256 ? 4 : P.experts <= 512 ? 8 : 16;
  bool four = P.tokens > TOKENS && per <= 8 && P.top <= 15;
  if (four) {
    int in_rows = per;  // experts of a lane / 4
    for (; in_rows <= 8; in_rows *= 2) {
      P.span = P.groups == 1 ? 16 : 1;
      while ((int64_t)P.span * 4 * in_rows < (int64_t)P.each.d) P.span *= 2;
      if (P.span * P.groups <= 16) break;
    }
    four = in_rows <= 8;
    if (four) per = in_rows;
  }
  void (*kernel)(RouteArgs, int) = per == 1   ? (four ? route_kernel<1, true> : route_kernel<1, false>)
                                   : per == 2 ? (four ? route_kernel<2, true> : route_kernel<2, false>)
                                   : per == 4 ? (four ? route_kernel<4, true> : route_kernel<4, false>)
                                   : per == 8 ? (four ? route_kernel<8, true> : route_kernel<8, false>) : route_kernel<16, false>;
  void *list[] = {&P, &type};
  hipError_t e = hipLaunchKernel(reinterpret_cast<const void *>(kernel), dim3((unsigned)blocks), dim3(four ? 512 : THREADS), list, 0, s);
  if (e == hipSuccess && P.counts) {
    const int64_t groups = blocks < 256 ? blocks : 256;  // (each adds up all counts)
    int64_t all = blocks;
    int share = (int)((blocks + groups - 1) / groups);
    void *more[] = {&P, &all, &share};
    e = hipLaunchKernel(reinterpret_cast<const void *>(place_kernel), dim3((unsigned)((blocks + share - 1) / share)), dim3(THREADS), more, 0, s);
  }
  if (e != hipSuccess) (void)hipGetLastError();  // (the caller gets it; the next check of theirs must not find it again)
  return e;
}

}  // namespace mip
