// Routing to experts from the gate's logits: softmax or sigmoid scores, a bias that takes part in the choice only, groups
// of experts of which a token may use some, top-k, and weights that are renormalised and scaled (oled_route_scored; a
// layer's routing inside a step, oled_register_routing).
//
//   score  s_e = 1 / (1 + exp(-l_e)), or exp(l_e - max l) / sum exp(l - max l)
//   choice c_e = s_e + bias_e; without a bias c_e = l_e, the scores' own order
//   group  v_g = its largest choice, or the sum of its two largest s_e + bias_e; the top_groups largest stay
//   ids    the top_k largest choices in the groups that stay; weight = scale * s / (sum of the chosen s + 1e-20), or scale * s
// Equal values go to the lower index.  A NaN logit counts as -inf, and its choice as -inf; so does a choice that is NaN.
//
// The ids are those of the formulas in exact arithmetic as far as 64 bits tell: choices are compared in fp32 first, and a
// token two of whose compared values lie within the fp32 forms' error (near_choices() below) is decided again in fp64 by
// the same warp.  That is one token in about two thousand with a bias (256 experts in groups), none without one (logits are
// compared as they are).  With a bias it is every token, though, where nothing but -inf is left behind the last choice: as many experts wanted
// as the groups that stay have, or all others masked by their bias (32768 tokens, 32 of 256 experts out of one of eight groups: 84 us, 31 of them 55).
//
// A warp per token.  Its lanes are dealt to the groups (32 / G each, G rounded up to a power of two), a lane's experts are
// consecutive, so that lower lanes hold lower experts and a group never shares a lane with another.  Every lane
// sorts its keys once (a network of maxima and minima in registers); then each of the top_k rounds is one warp maximum
// over the lanes' heads, a vote for the lowest lane that has it, and a shift in that lane.
// Bound by the instructions of a token, 670 a warp at 256 experts in groups (32768 tokens: 34.9 us, 28 of them this kernel's; the bytes
// would take 6).
#include <algorithm>
#include <cmath>
#include <type_traits>

#include "kernels.h"
#include "route_math.h"
#include "row_args.h"
#include "sm100_ptx.h"

namespace oled {
namespace {

constexpr int kScoredWarps = 16;
constexpr int kScoredThreads = kScoredWarps * 32;
// Warps of a CTA that only routes, at most: one CTA an SM, of as many warps as its registers are enough for.
__host__ __device__ constexpr int route_warps(int per) { return per <= 8 ? 32 : 16; }
constexpr int kExactLanes = 32;  // experts that a warp decides in fp64 side by side

struct ScoredArgs {
  const float* logits;
  const float* bias;
  int64_t stride;
  int32_t* ids;
  float* gate;
  int T, E, K, G, top_groups, group_top, softmax, renormalise;
  float scale;
  int group_size, lanes_per_group, lanes_log2, per_lane, vec;
  // tokens of CTA c: segment c / parts, of seg_tokens tokens, and there the part c % parts, of part_tokens
  int parts, seg_tokens, part_tokens;
  // (nullptr: not wanted) per CTA and expert, [n_ctas][hist_stride]
  uint16_t* hist;
  int hist_stride;
  // (nullptr: not wanted) zeroed arrays of a step: counts [E], per-segment counts [n_segments][E], reuse-score numerators [E]
  int32_t* counts;
  int32_t* seg_counts;
  unsigned long long* scores;
  const float* conf;
};

__device__ __forceinline__ float warp_sum(float v) {
#pragma unroll
  for (int d = 16; d >= 1; d >>= 1) v += __shfl_xor_sync(0xffffffffu, v, d);
  return v;
}
__device__ __forceinline__ float no_nan(float v) { return v == v ? v : __int_as_float(0xff800000); }
// The warp's largest value (no NaN among them).
__device__ __forceinline__ float reduce_max(float v) {
  float r;
  asm volatile("redux.sync.max.f32 %0, %1, 0xffffffff;" : "=f"(r) : "f"(v));
  return r;
}
// Descending order of N values in registers (Batcher's odd-even merges: 19 exchanges for eight values).
template <int N>
__device__ __forceinline__ void sort_desc(float (&k)[N]) {
#pragma unroll
  for (int p = 1; p < N; p <<= 1)
#pragma unroll
    for (int d = p; d >= 1; d >>= 1)
#pragma unroll
      for (int i = 0; i < N; ++i) {
        const int at = i - d % p;  // pairs i, i + d lie in stretches of 2 d from d % p on, in their first halves
        if (at >= 0 && at % (2 * d) < d && i + d < N && i / (2 * p) == (i + d) / (2 * p)) {
          const float hi = fmaxf(k[i], k[i + d]), lo = fminf(k[i], k[i + d]);
          k[i] = hi;
          k[i + d] = lo;
        }
      }
}

__device__ __forceinline__ unsigned long long order_key64(double v) {  // v is not NaN and not -0
  const unsigned long long bits = (unsigned long long)__double_as_longlong(v);
  return (bits >> 63) ? ~bits : (bits | 0x8000000000000000ull);
}

// exp(x) in fp64, without a branch so that several run side by side: x = n ln 2 + r with ln 2 in two parts (Cody and Waite), the
// Taylor polynomial of degree 13 for |r| <= ln 2 / 2 (its remainder is below 2^-57 of the result), and 2^n in two factors, so that
// results down to the smallest subnormal number are rounded once, and zero and infinity beyond them come by themselves.  Off by a few
// units in the last place.
__device__ __forceinline__ double exp_double(double x) {
  x = fmin(fmax(x, -746.0), 710.0);  // (exp(-746) < 2^-1075, exp(710) > 2^1024)
  const double n = rint(x * 1.4426950408889634074);
  double r = fma(-n, 6.93147180369123816490e-01, x);  // ln 2 without its low 21 bits: n times it is exact
  r = fma(-n, 1.90821492927058770002e-10, r);
  double p = 1.0 / 6227020800.0;
  p = fma(p, r, 1.0 / 479001600.0);
  p = fma(p, r, 1.0 / 39916800.0);
  p = fma(p, r, 1.0 / 3628800.0);
  p = fma(p, r, 1.0 / 362880.0);
  p = fma(p, r, 1.0 / 40320.0);
  p = fma(p, r, 1.0 / 5040.0);
  p = fma(p, r, 1.0 / 720.0);
  p = fma(p, r, 1.0 / 120.0);
  p = fma(p, r, 1.0 / 24.0);
  p = fma(p, r, 1.0 / 6.0);
  p = fma(p, r, 0.5);
  p = fma(p, r, 1.0);
  p = fma(p, r, 1.0);
  const int whole = (int)n, half = whole / 2;
  return __longlong_as_double(__double_as_longlong(p) + ((long long)half << 52)) * __longlong_as_double((long long)(1023 + whole - half) << 52);
}
// 1 / x for x of 1 to 2^1000, by Newton's iteration from an approximation of 2^-20.
__device__ __forceinline__ double reciprocal_double(double x) {
  double y;
  asm("rcp.approx.ftz.f64 %0, %1;" : "=d"(y) : "d"(x));
  y = fma(y, fma(-x, y, 1.0), y);
  y = fma(y, fma(-x, y, 1.0), y);
  return y;
}

// The softmax's sum of a token in fp64.
__device__ __forceinline__ double sum_exact(const float* row, int first, int mine, float top) {
  double sum = 0.0;
#pragma unroll 1
  for (int i = 0; i < mine; ++i) {
    const float l = no_nan(row[first + i]);
    sum += exp_double(l == top ? 0.0 : (double)l - (double)top);
  }
  for (int d = 16; d >= 1; d >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, d);
  return sum;
}
// An expert's choice in fp64 (no NaN: -inf), and its score.
__device__ __forceinline__ double choice_exact(const ScoredArgs& a, const float* row, int e, float top, double sum, double& score) {
  const float l = row[e], x = no_nan(l);
  const double ex = exp_double(a.softmax ? (x == top ? 0.0 : (double)x - (double)top) : -(double)x);
  const double num = a.softmax ? ex : 1.0, den = a.softmax ? sum : 1.0 + ex;
  // (next to the smallest numbers the quotient is rounded once)
  score = num < 0x1p-900 || den > 0x1p900 ? num / den : num * reciprocal_double(den);
  const double c = a.bias == nullptr ? (double)l : score + (double)a.bias[e];
  return l == l && c == c ? c : -INFINITY;
}
// Deals the experts of the lanes' masks to the lanes, one each, by way of the warp's s_experts[kExactLanes]; their number (above 32: none dealt).
template <int PER>
__device__ __forceinline__ int deal(uint32_t mask, int lane, int first, int32_t* s_experts, int& expert) {
  int n = 0;
  __syncwarp();
#pragma unroll 1
  for (int i = 0; i < PER; ++i) {
    const bool in = (mask >> i) & 1u;
    const uint32_t lanes = __ballot_sync(0xffffffffu, in);
    const int at = n + __popc(lanes & ((1u << lane) - 1u));
    if (in && at < kExactLanes) s_experts[at] = first + i;
    n += __popc(lanes);
  }
  __syncwarp();
  expert = lane < n ? s_experts[lane] : 0;
  return n;
}

// Which groups stay, where the border between them lies between values that are too near to each other; sure: the lane's group stays in any
// case, question: it may (mask: those of its experts that can count for its value).  None of the values is NaN or -inf.
// False in `decided`: too many experts.
template <int PER>
__device__ __noinline__ bool groups_exact(const ScoredArgs& a, const float* row, int lane, int first, int mine, float top, bool sure, bool question,
                                          uint32_t mask, int32_t* s_experts, bool& decided) {
  int expert;
  const int n = deal<PER>(mask, lane, first, s_experts, expert);
  decided = n <= 32;
  if (!decided) return false;
  const double sum = a.softmax ? sum_exact(row, first, mine, top) : 1.0;
  double value, score;
  value = choice_exact(a, row, expert, top, sum, score);
  if (a.bias == nullptr && a.group_top == 2) value = score;
  const int group = expert / a.group_size, g = lane >> a.lanes_log2;
  double t1 = -INFINITY, t2 = -INFINITY;
#pragma unroll 4
  for (int o = 0; o < n; ++o) {
    const double v = __shfl_sync(0xffffffffu, value, o);
    if (__shfl_sync(0xffffffffu, group, o) == g) {
      t2 = fmax(t2, fmin(t1, v));
      t1 = fmax(t1, v);
    }
  }
  const double v = a.group_top == 1 ? t1 : t1 + t2;
  const uint32_t asked = __ballot_sync(0xffffffffu, question);
  const int places = a.top_groups - (__popc(__ballot_sync(0xffffffffu, sure)) >> a.lanes_log2);
  int before = 0;
#pragma unroll 1
  for (int o = 0; o < a.G; ++o) {
    const double w = __shfl_sync(0xffffffffu, v, o << a.lanes_log2);
    before += ((asked >> (o << a.lanes_log2)) & 1u) && (w > v || (w == v && o < g));
  }
  return sure || (question && before < places);
}

// The choice of one token in fp64, by the warp that holds its logits: lane r < K ends with the id of rank r.  mask: the lane's experts
// that can be among the K.  groups: the groups are chosen again too (all experts are in the masks then).
// Few tokens come here, but a CTA waits for the last of its own; what they cost is fp64 latency, so only those
// experts are computed that the fp32 forms leave in question, a lane each where there are lanes for them (lanes with two or three of them
// in turn, and rounds to order them: 250 tokens, two of them near, 8.4 us, this way 7.5; with all experts a token took 5.5 us).
template <int PER>
__device__ __noinline__ int select_exact(const ScoredArgs& a, const float* row, int lane, int first, int mine, float top, uint32_t mask,
                                         bool groups, int32_t* s_experts) {
  const double kNone = -INFINITY;
  unsigned long long key[PER];  // of the choices (in local memory: registers count for the whole kernel)
  const double sum = a.softmax ? sum_exact(row, first, mine, top) : 1.0;
  double score;
  int expert;
  const int n = groups ? 33 : deal<PER>(mask, lane, first, s_experts, expert);
  if (n <= 32) {
    const double c = choice_exact(a, row, expert, top, sum, score);
    int before = 0;
#pragma unroll 4
    for (int o = 0; o < n; ++o) {
      const double v = __shfl_sync(0xffffffffu, c, o);
      const int e = __shfl_sync(0xffffffffu, expert, o);
      before += v > c || (v == c && e < expert);
    }
    __syncwarp();
    if (lane < n && before < a.K) s_experts[before] = expert;
    __syncwarp();
    return lane < a.K ? s_experts[lane] : 0;
  }
  double t1 = kNone, t2 = kNone;
#pragma unroll 1
  for (uint32_t m = mask; m != 0u; m &= m - 1u) {
    const int i = __ffs((int)m) - 1;
    const double c = choice_exact(a, row, first + i, top, sum, score);
    key[i] = order_key64(c + 0.0);
    if (groups) {
      const double v = a.bias != nullptr || a.group_top == 1 ? c : score;
      t2 = fmax(t2, fmin(t1, v));
      t1 = fmax(t1, v);
    }
  }
  if (groups) {
#pragma unroll 1
    for (int d = a.lanes_per_group >> 1; d >= 1; d >>= 1) {
      const double o1 = __shfl_xor_sync(0xffffffffu, t1, d), o2 = __shfl_xor_sync(0xffffffffu, t2, d);
      t2 = fmax(fmin(t1, o1), fmax(t2, o2));
      t1 = fmax(t1, o1);
    }
    double v = a.group_top == 1 ? t1 : t1 + t2;
    if (!(v == v)) v = kNone;
    const int g = lane >> a.lanes_log2;
    int before = 0;
#pragma unroll 1
    for (int o = 0; o < a.G; ++o) {
      const double w = __shfl_sync(0xffffffffu, v, o << a.lanes_log2);
      before += w > v || (w == v && o < g);
    }
    if (before >= a.top_groups) mask = 0u;
  }
  int id = 0, at = 0;
  unsigned long long best = 0ull;
  bool again = true;  // the lane has to look for its best
#pragma unroll 1
  for (int r = 0; r < a.K; ++r) {
    if (again) {
      best = 0ull;
#pragma unroll 1
      for (uint32_t m = mask; m != 0u; m &= m - 1u) {
        const int i = __ffs((int)m) - 1;
        if (key[i] > best) {  // (ascending i: the lower index stays; no key is zero)
          best = key[i];
          at = i;
        }
      }
    }
    const uint32_t hi = (uint32_t)(best >> 32), hi_max = __reduce_max_sync(0xffffffffu, hi);
    const uint32_t lo = hi == hi_max ? (uint32_t)best : 0u, lo_max = __reduce_max_sync(0xffffffffu, lo);
    const int winner = __ffs((int)__ballot_sync(0xffffffffu, hi == hi_max && (uint32_t)best == lo_max)) - 1;
    const int chosen = __shfl_sync(0xffffffffu, first + at, winner);
    again = lane == winner;
    if (again) mask &= ~(1u << at);
    if (lane == r) id = chosen;
  }
  return id;
}

// Could the fp32 forms of two choices a >= b be in the wrong order?  A sigmoid is off by at most 2^-22 (exp: argument and
// ex2 2^-22 + |l| 2^-24 relative, times s (1 - s); sum and quotient 2^-23 + 2^-24), a softmax score by at most 2^-18 of
// the largest score (its sum of up to 512 terms in at most 37 rounded steps), the addition of the bias by 2^-24 of the result;
// `slack` is twice the scores' part and a fifth more.  Nothing is
// clearly apart from an infinity here: its difference from a finite value is no larger than the bound that it is compared with.
__device__ __forceinline__ bool near_choices(float a, float b, float slack) {
  return !(a - b > slack + 2.4e-7f * fmaxf(fabsf(a), fabsf(b)));
}

// The fp32 forms the choice starts from.  exp2 and the reciprocal are off by 2^-22 and 2^-23 of their results.
__device__ __forceinline__ float fast_exp(float x) {
  float r;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x * 1.4426950408889634f));
  return r;
}
__device__ __forceinline__ float fast_reciprocal(float x) {
  float r;
  asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
  return r;
}
__device__ __forceinline__ float fast_sigmoid(float l) { return fast_reciprocal(1.0f + fast_exp(-l)); }

// Where the bias of a lane's expert i lies in shared memory, so that a warp reads up to 16 bytes a lane at once.  (In registers they left too few
// for the rest.)
template <int PER>
__device__ __forceinline__ int bias_at(int lane, int i) {
  constexpr int kRun = PER < 4 ? PER : 4;
  return (i / kRun * 32 + lane) * kRun + i % kRun;
}

// A token's logits, as its lanes hold them.  PER: experts a lane has room for.  FULL: every lane has that many.
template <int PER, bool FULL>
__device__ __forceinline__ void load_logits(const ScoredArgs& a, int t, int first, int mine, float (&l)[PER]) {
  const float* const row = a.logits + (int64_t)t * a.stride + first;
  if (PER >= 4 && a.vec) {
#pragma unroll
    for (int i = 0; i + 3 < PER; i += 4)
      if (FULL || i < mine) {
        const float4 v = *reinterpret_cast<const float4*>(row + i);
        l[i] = v.x;
        l[i + 1] = v.y;
        l[i + 2] = v.z;
        l[i + 3] = v.w;
      }
  } else {
#pragma unroll
    for (int i = 0; i < PER; ++i)
      if (FULL || i < mine) l[i] = row[i];
  }
}

template <int PER, bool FULL>
__device__ __forceinline__ void route_token(const ScoredArgs& a, int t, int lane, const float (&l)[PER], const float* s_bias, int first,
                                            int mine_, int32_t* s_experts, int32_t* s_ids, int32_t* s_counts, unsigned long long* s_scores) {
  const int mine = FULL ? PER : mine_;
  const float* const row = a.logits + (int64_t)t * a.stride;
  const float kNone = __int_as_float(0xff800000);
  float top = kNone, sum = 1.0f, slack = 0.0f;
  bool near = false;        // two choices are too near to each other
  bool near_group = false;  // ... or two groups, or there is a NaN, or too little that is not -inf: everything is decided again
  float key[PER];           // what is compared (-inf: there is no such expert, or as good as none)
  float z[PER];
  if (a.softmax) {  // (fmaxf reads a NaN as -inf)
#pragma unroll
    for (int i = 0; i < PER; ++i)
      if (FULL || i < mine) top = fmaxf(top, l[i]);
    top = reduce_max(top);
    // (renormalised weights are quotients of the chosen exponentials, and the largest of those is 1: 1e-20 beside it is nothing)
    if (a.bias != nullptr || !a.renormalise || a.G > 1) {
      sum = 0.0f;
#pragma unroll
      for (int i = 0; i < PER; ++i) {
        const float x = fmaxf(l[i], kNone);
        z[i] = FULL || i < mine ? (x == top ? 1.0f : fast_exp(x - top)) : 0.0f;
        sum += z[i];
      }
      sum = warp_sum(sum);
    }
  }
  const float inverse = fast_reciprocal(sum);
  if (a.bias != nullptr) {
    slack = a.softmax ? 9.2e-6f * inverse : 5.8e-7f;
    float bias[PER];
#pragma unroll
    for (int i = 0; i < PER; ++i) bias[i] = s_bias[bias_at<PER>(lane, i)];
#pragma unroll
    for (int i = 0; i < PER; ++i) {
      const float c = (a.softmax ? z[i] * inverse : fast_sigmoid(l[i])) + bias[i];
      near_group = near_group || ((FULL || i < mine) && !(c == c));
      key[i] = FULL || i < mine ? c : kNone;
    }
    if (a.softmax) {  // (z of a NaN is 0)
#pragma unroll
      for (int i = 0; i < PER; ++i) near_group = near_group || ((FULL || i < mine) && !(l[i] == l[i]));
    }
  } else {
#pragma unroll
    for (int i = 0; i < PER; ++i) {
      near_group = near_group || ((FULL || i < mine) && !(l[i] == l[i]));
      key[i] = FULL || i < mine ? l[i] : kNone;
    }
  }
  float sorted[PER];
#pragma unroll
  for (int i = 0; i < PER; ++i) sorted[i] = key[i];
  sort_desc<PER>(sorted);
  bool keep = true;  // the lane's group stays
  if (a.G > 1) {
    // the two largest choices of the lane, then of its group
    float t1 = sorted[0], t2 = sorted[1];
    for (int d = a.lanes_per_group >> 1; d >= 1; d >>= 1) {
      const float o1 = __shfl_xor_sync(0xffffffffu, t1, d), o2 = __shfl_xor_sync(0xffffffffu, t2, d);
      t2 = fmaxf(fminf(t1, o1), fmaxf(t2, o2));
      t1 = fmaxf(t1, o1);
    }
    float group_slack = slack;
    float off = 0.0f;  // what the group's fp32 value is off by at most, the scores' part apart
    const float least = a.group_top == 2 ? t2 : t1;  // what an expert has to reach to count for its group
    if (a.group_top == 2) {
      if (a.bias == nullptr) {  // the order of scores is that of logits
        if (a.softmax) {
          t1 = t1 == top ? inverse : fast_exp(t1 - top) * inverse;
          t2 = t2 == top ? inverse : fast_exp(t2 - top) * inverse;
          group_slack = 9.2e-6f * inverse;
        } else {
          t1 = fast_sigmoid(t1);
          t2 = fast_sigmoid(t2);
          group_slack = 5.8e-7f;
        }
      }
      // two choices and their sum, each rounded: 2^-24 of the larger choice twice, and of the sum, which is twice that at most or, where
      // the two cancel, nearly nothing
      if (a.bias != nullptr) off = 2.4e-7f * fmaxf(fabsf(t1), fabsf(t2));
      t1 += t2;
      if (!(fabsf(t1) <= 3.4028235e38f)) off = 0.0f;
      group_slack *= 2.0f;
    }
    // rounds over the groups: the lanes of the largest value drop out
    const int g = lane >> a.lanes_log2;
    near_group = near_group || !(t1 == t1);
    const float value = g < a.G ? t1 : kNone;
    float left = value, last = kNone;
    for (int r = 0; r < a.top_groups; ++r) {
      last = reduce_max(left);
      left = left == last ? kNone : left;
    }
    keep = g < a.G && value >= last;
    // (every lane takes part in these, so not behind conditions of its own)
    const float next = reduce_max(keep || g >= a.G ? kNone : value + off);  // as much as a group that goes may be
    if (a.bias != nullptr && a.group_top == 2) last = last == kNone ? kNone : -reduce_max(keep ? off - value : kNone);  // as little as one that stays may be
    if (last == kNone) {
      near_group = true;
    } else if (__popc(__ballot_sync(0xffffffffu, keep)) != a.top_groups << a.lanes_log2) {  // equal values: the lower groups
      near_group = near_group || a.bias != nullptr || a.group_top == 2;                      // (fp32 forms: decided again)
      int before = 0;
#pragma unroll 1
      for (int o = 0; o < a.G; ++o) {
        const float v = __shfl_sync(0xffffffffu, value, o << a.lanes_log2);
        before += v > value || (v == value && o < g);
      }
      keep = g < a.G && before < a.top_groups;
    } else if ((a.bias != nullptr || a.group_top == 2) && near_choices(last, next, group_slack)) {
      // Groups clearly above the best one that goes stay, groups clearly below the least one that stays go; between the others ...
      const bool sure = keep && !near_choices(value - off, next, group_slack);
      const bool question = g < a.G && !sure && (keep || near_choices(last, value + off, group_slack));
      uint32_t mask = 0u;
#pragma unroll
      for (int i = 0; i < PER; ++i) {
        const bool in = question && (FULL || i < mine) && (key[i] >= least || near_choices(least, key[i], 2.0f * slack));
        mask |= in ? 1u << i : 0u;
      }
      bool decided;
      keep = groups_exact<PER>(a, row, lane, first, mine, top, sure, question, mask, s_experts, decided);
      near_group = near_group || !decided;
    }
    if (!keep) sorted[0] = kNone;  // (the others are not reached before -inf is the best there is)
  }
  // Rounds: lane r ends with the r-th largest key and the lanes that had it at their head.  Every lane that has the largest
  // key drops it, which is one lane unless keys are equal.
  float my_key = kNone;
  uint32_t my_lanes = 0u;
  for (int r = 0; r < a.K; ++r) {
    const float best = reduce_max(sorted[0]);
    const bool mine_is_best = sorted[0] == best;
    const uint32_t lanes = __ballot_sync(0xffffffffu, mine_is_best);
    if (lane == r) {
      my_key = best;
      my_lanes = lanes;
    }
#pragma unroll
    for (int i = 0; i + 1 < PER; ++i) sorted[i] = mine_is_best ? sorted[i + 1] : sorted[i];
    sorted[PER - 1] = mine_is_best ? kNone : sorted[PER - 1];
  }
  if (a.bias != nullptr) {
    float after = __shfl_down_sync(0xffffffffu, my_key, 1);
    const float next = reduce_max(sorted[0]);
    if (lane == a.K - 1) after = next;
    if (lane < a.K) near = near || near_choices(my_key, after, slack);
  }
  const bool shared = lane < a.K && (my_lanes & (my_lanes - 1u)) != 0u;
  if (a.bias != nullptr) {
    near = near || shared;  // equal fp32 forms say nothing about the choices
  } else if (__any_sync(0xffffffffu, shared)) {
    // equal logits in several lanes (logits that were bf16 have them often): again, the lowest lane alone drops its key
#pragma unroll
    for (int i = 0; i < PER; ++i) sorted[i] = keep ? key[i] : kNone;
    sort_desc<PER>(sorted);
    for (int r = 0; r < a.K; ++r) {
      const float best = reduce_max(sorted[0]);
      const uint32_t lanes = __ballot_sync(0xffffffffu, sorted[0] == best), lowest = lanes & (0u - lanes);
      if (lane == r) {
        my_key = best;
        my_lanes = lowest;
      }
      if ((lowest >> lane) & 1u) {
#pragma unroll
        for (int i = 0; i + 1 < PER; ++i) sorted[i] = sorted[i + 1];
        sorted[PER - 1] = kNone;
      }
    }
  }
  // (keys of -inf do not tell experts from places without one)
  near_group = __any_sync(0xffffffffu, near_group || (lane < a.K && (my_key == kNone || my_lanes == 0u)));
  near = near_group || __any_sync(0xffffffffu, near);
  int id;
  if (near) {
    // experts in question: choices that are not clearly below the K-th
    const float least = __shfl_sync(0xffffffffu, my_key, a.K - 1);
    uint32_t mask = 0u;
#pragma unroll
    for (int i = 0; i < PER; ++i) {
      const bool in = (FULL || i < mine) && (near_group || (keep && (near_choices(least, key[i], 2.0f * slack) || key[i] >= least)));
      mask |= in ? 1u << i : 0u;
    }
    id = select_exact<PER>(a, row, lane, first, mine, top, mask, near_group && a.G > 1, s_experts);
  } else {
    const int my_lane = (__ffs((int)my_lanes) - 1) & 31;
    int at = 0;
    const float before = __shfl_up_sync(0xffffffffu, my_key, 1);
    if (!__any_sync(0xffffffffu, lane > 0 && lane < a.K && before == my_key)) {
      // (downwards: of equal keys of the lane, one of them chosen and one not, the first counts)
#pragma unroll
      for (int i = PER - 1; i >= 0; --i) at = __shfl_sync(0xffffffffu, key[i], my_lane) == my_key ? i : at;
    } else {  // equal keys of one lane are taken in the order of their indices
      const uint32_t same = __match_any_sync(0xffffffffu, __float_as_uint(__fadd_rn(my_key, 0.0f))) & __match_any_sync(0xffffffffu, my_lane);
      int skip = __popc(same & ((1u << lane) - 1u));
#pragma unroll
      for (int i = 0; i < PER; ++i) {
        const float k = __shfl_sync(0xffffffffu, key[i], my_lane);
        if (k == my_key) {
          if (skip == 0) at = i;
          --skip;
        }
      }
    }
    id = __shfl_sync(0xffffffffu, first, my_lane) + at;
  }
  // the chosen experts' weights (the quotients are off by two units in the last place at most)
  float s = 0.0f;
  if (lane < a.K) {
    const float x = no_nan(row[id]);
    s = a.softmax ? (x == top ? 1.0f : expf(x - top)) : __fdividef(1.0f, 1.0f + expf(-x));
  }
  float w = s;
  if (a.renormalise) w = __fdividef(s, warp_sum(s) + 1e-20f * sum);  // (softmax: s is sum times the score)
  else if (a.softmax) w = __fdividef(s, sum);
  if (lane < a.K) {
    a.ids[(int64_t)t * a.K + lane] = id;
    a.gate[(int64_t)t * a.K + lane] = w * a.scale;
    if (s_ids != nullptr) s_ids[lane] = id;
    if (s_counts != nullptr) atomicAdd(&s_counts[id], 1);
    // (the numerators take the weight before its scale, at most one: their sums are reported in 48 bits)
    if (s_scores != nullptr) atomicAdd(&s_scores[id], score_quantum(w, a.conf[t]));
  }
}

// The tokens begin + warp, begin + warp + n_warps, ... of a CTA; the next one's logits are on their way while one is routed.
template <int PER, bool FULL>
__device__ __forceinline__ void route_tokens(const ScoredArgs& a, int begin, int end, int warp, int n_warps, int lane, const float* s_bias, int first,
                                             int mine, int32_t* s_experts, int32_t* s_ids, int32_t* s_counts, unsigned long long* s_scores) {
  float l[PER];
  int t = begin + warp;
  if (t < end) load_logits<PER, FULL>(a, t, first, mine, l);
  for (; t < end; t += n_warps) {
    float now[PER];
#pragma unroll
    for (int i = 0; i < PER; ++i) now[i] = l[i];
    if (t + n_warps < end) load_logits<PER, FULL>(a, t + n_warps, first, mine, l);
    route_token<PER, FULL>(a, t, lane, now, s_bias, first, mine, s_experts + warp * kExactLanes, s_ids != nullptr ? s_ids + (t - begin) * a.K : nullptr,
                           s_counts, s_scores);
  }
}

// The experts of a lane.
__device__ __forceinline__ void lane_experts(const ScoredArgs& a, int lane, int& first, int& mine) {
  const int g = lane >> a.lanes_log2, sub = lane - (g << a.lanes_log2);
  first = g < a.G ? g * a.group_size + sub * a.per_lane : 0;
  mine = g < a.G ? max(0, min(a.per_lane, a.group_size - sub * a.per_lane)) : 0;
}
// The lanes' biases to shared memory.
template <int PER>
__device__ __forceinline__ void fetch_bias(const ScoredArgs& a, int warp, int n_warps, int lane, int first, int mine, float* s_bias) {
  if (a.bias == nullptr) return;
  for (int i = warp; i < PER; i += n_warps) s_bias[bias_at<PER>(lane, i)] = i < mine ? a.bias[first + i] : 0.0f;
  __syncthreads();
}

// Dynamic shared memory: [E] scores (where wanted), [E] counts (where wanted).
template <int PER, bool FULL>
__global__ void __launch_bounds__(route_warps(PER) * 32, 1)
route_scored_kernel(const __grid_constant__ ScoredArgs a) {
  extern __shared__ __align__(16) uint8_t s_dyn[];
  __shared__ __align__(16) float s_bias[32 * PER];
  __shared__ int32_t s_experts[route_warps(PER) * kExactLanes];
  const int warp = threadIdx.x >> 5, n_warps = blockDim.x >> 5, lane = threadIdx.x & 31;
  unsigned long long* const s_scores = a.scores != nullptr ? reinterpret_cast<unsigned long long*>(s_dyn) : nullptr;
  const bool counting = a.hist != nullptr || a.counts != nullptr;
  int32_t* const s_counts = counting ? reinterpret_cast<int32_t*>(s_dyn + (s_scores != nullptr ? (size_t)a.E * 8 : 0)) : nullptr;
  griddep_launch_dependents();
  if (counting) {
    for (int e = threadIdx.x; e < a.E; e += blockDim.x) {
      s_counts[e] = 0;
      if (s_scores != nullptr) s_scores[e] = 0ull;
    }
    __syncthreads();
  }
  griddep_wait();
  int first, mine;
  lane_experts(a, lane, first, mine);
  fetch_bias<PER>(a, warp, n_warps, lane, first, mine, s_bias);
  const int seg = (int)blockIdx.x / a.parts, part = (int)blockIdx.x - seg * a.parts;
  const int begin = seg * a.seg_tokens + part * a.part_tokens;
  const int end = min(min(begin + a.part_tokens, (seg + 1) * a.seg_tokens), a.T);
  route_tokens<PER, FULL>(a, begin, end, warp, n_warps, lane, s_bias, first, mine, s_experts, nullptr, s_counts, s_scores);
  if (!counting) return;
  __syncthreads();
  for (int e = threadIdx.x; e < a.E; e += blockDim.x) {
    const int n = s_counts[e];
    if (a.hist != nullptr) a.hist[(size_t)blockIdx.x * a.hist_stride + e] = (uint16_t)n;  // (a CTA has fewer than 2^16 tokens)
    if (n == 0) continue;
    if (a.counts != nullptr) atomicAdd(&a.counts[e], n);
    if (a.seg_counts != nullptr) atomicAdd(&a.seg_counts[seg * a.E + e], n);
    if (s_scores != nullptr && s_scores[e] != 0ull) atomicAdd(&a.scores[e], s_scores[e]);
  }
}

// ---- the order by expert ----------------------------------------------------------------------
// Exclusive prefix over threads (one value each) of a CTA of WARPS warps.
template <int WARPS>
__device__ __forceinline__ int cta_prefix(int v, int* s_warp) {
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  int incl = v;
#pragma unroll
  for (int d = 1; d < 32; d <<= 1) {
    const int o = __shfl_up_sync(0xffffffffu, incl, d);
    if (lane >= d) incl += o;
  }
  if (lane == 31) s_warp[warp] = incl;
  __syncthreads();
  int before = incl - v;
  for (int w = 0; w < warp; ++w) before += s_warp[w];
  return before;
}

// Rows of the assignments of a CTA's n tokens (ids: K of each token; the first of them is number a0) in the stable order by expert. Every warp
// counts the experts of a contiguous part (s_rows: [kScoredWarps][E], zeros), start(e, n of the CTA) says where the CTA's rows of an
// expert begin, and every warp hands out its part's rows in order, a token at a time: its experts differ, so that its lanes need
// not look for equal ones among them (32 assignments at a time with a match among the lanes took four times as long).
template <typename Start>
__device__ __forceinline__ void place_rows(const int32_t* ids, int n, int K, int64_t a0, int E, int* s_rows, int32_t* __restrict__ perm, Start start) {
  static_assert(kScoredThreads >= OLED_MAX_EXPERTS, "a thread per expert");
  static_assert(OLED_MAX_TOPK <= 32, "a lane per expert of a token");
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int per_warp = (n + kScoredWarps - 1) / kScoredWarps, first = min(n, warp * per_warp), last = min(n, first + per_warp);
  int* const mine = s_rows + warp * E;
  for (int i = first * K + lane; i < last * K; i += 32) atomicAdd(&mine[ids[i]], 1);
  __syncthreads();
  const int e = threadIdx.x;
  int total = 0, part[kScoredWarps];
  if (e < E)
#pragma unroll
    for (int w = 0; w < kScoredWarps; ++w) {
      part[w] = s_rows[w * E + e];
      total += part[w];
    }
  int at = start(e, total);
  if (e < E)
#pragma unroll
    for (int w = 0; w < kScoredWarps; ++w) {
      s_rows[w * E + e] = at;
      at += part[w];
    }
  __syncthreads();
  // (as many whole tokens as there are lanes for are fetched at once, and the next ones meanwhile)
  const int tokens = 32 / K, mine_of = lane / K;
  int id = mine_of < tokens && first + mine_of < last ? ids[first * K + lane] : -1;
  for (int t = first; t < last; t += tokens) {
    const int next = mine_of < tokens && t + tokens + mine_of < last ? ids[(t + tokens) * K + lane] : -1;
    for (int j = 0; j < tokens; ++j) {
      if (mine_of == j && id >= 0) {
        const int row = mine[id];
        mine[id] = row + 1;
        perm[row] = (int32_t)(a0 + t * K + lane);
      }
      __syncwarp();
    }
    id = next;
  }
}

constexpr int kScoredCtas = 148;  // at most: one an SM
// More than half of an SM's shared memory, so that no SM takes two CTAs while others have none: they start as SMs become free.
constexpr size_t kPlaceSmem = 120 * 1024;
static_assert(kPlaceSmem >= (size_t)kScoredWarps * OLED_MAX_EXPERTS * sizeof(int), "a row of counts per warp");

// Every CTA adds up the histograms of all of them itself, 148 rows of E 16-bit counts out of L2: cheaper than a kernel in between that leaves
// it one row to read (32768 tokens, 256 experts in groups: 40.4 us with one, 33.8 without and with one CTA an SM; 8-bit counts 33.5).
__global__ void __launch_bounds__(kScoredThreads)
place_kernel(const int32_t* __restrict__ ids, int T, int K, int E, int part_tokens, const uint16_t* __restrict__ hist, int hist_stride,
             int32_t* __restrict__ counts, int32_t* __restrict__ offsets, int32_t* __restrict__ perm) {
  extern __shared__ int s_rows[];  // [kScoredWarps][E]
  __shared__ int s_warp[kScoredWarps];
  constexpr int kFours = OLED_MAX_EXPERTS / 4, kTogether = 10;  // expert e's sums are at [e % 4][e / 4]
  __shared__ int s_all[OLED_MAX_EXPERTS], s_before[OLED_MAX_EXPERTS];
  griddep_launch_dependents();
  for (int i = threadIdx.x; i < kScoredWarps * E; i += kScoredThreads) s_rows[i] = 0;
  for (int i = threadIdx.x; i < OLED_MAX_EXPERTS; i += kScoredThreads) s_all[i] = s_before[i] = 0;
  griddep_wait();
  __syncthreads();
  // A thread per four experts and every `step`-th row, from the CTA's own row on: all of them on the same one at a time would wait for its L2
  // slice.
  const int fours = hist_stride / 4, step = kScoredThreads / fours, rows = (int)gridDim.x;
  const int first = (int)threadIdx.x / fours, four = (int)threadIdx.x - first * fours;
  if (first < step) {
    const uint2* const column = reinterpret_cast<const uint2*>(hist) + four;
    int all[4] = {}, before[4] = {};
    for (int i0 = first; i0 < rows; i0 += step * kTogether) {
      uint2 c[kTogether];
#pragma unroll
      for (int u = 0; u < kTogether; ++u) {
        const int i = i0 + u * step, r = i + (int)blockIdx.x < rows ? i + (int)blockIdx.x : i + (int)blockIdx.x - rows;
        c[u] = i < rows ? column[(size_t)r * fours] : make_uint2(0u, 0u);
      }
#pragma unroll
      for (int u = 0; u < kTogether; ++u) {
        const bool is_before = i0 + u * step + (int)blockIdx.x >= rows;  // (rows from the CTA's own on come first)
        const int n[4] = {(int)(c[u].x & 0xffffu), (int)(c[u].x >> 16), (int)(c[u].y & 0xffffu), (int)(c[u].y >> 16)};
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          all[j] += n[j];
          before[j] += is_before ? n[j] : 0;
        }
      }
    }
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      atomicAdd(&s_all[j * kFours + four], all[j]);
      atomicAdd(&s_before[j * kFours + four], before[j]);
    }
  }
  const int begin = (int)blockIdx.x * part_tokens, end = min(begin + part_tokens, T);
  const int64_t a0 = (int64_t)begin * K;
  place_rows(ids + a0, end - begin, K, a0, E, s_rows, perm, [&](int e, int) {  // (behind a barrier)
    const int at = e % 4 * kFours + e / 4, all = e < E ? s_all[at] : 0, start = cta_prefix<kScoredWarps>(all, s_warp);
    if (blockIdx.x == 0 && e < E) {
      counts[e] = all;
      offsets[e] = start;
      if (e == E - 1) offsets[E] = start + all;
    }
    return start + (e < E ? s_before[at] : 0);
  });
}

// Few tokens: routing and order in one launch by one cluster of up to eight CTAs, which add up their counts through
// distributed shared memory.  (A launch costs the caller more than these kernels the GPU.)
constexpr int kOneLaunch = 4096;                        // assignments
constexpr int kClusterIds = kOneLaunch / 8 + OLED_MAX_TOPK;  // of a CTA (16 tokens each with fewer than eight CTAs)
template <int PER, bool FULL>
__global__ void __launch_bounds__(kScoredThreads)
route_cluster_kernel(const __grid_constant__ ScoredArgs a, int32_t* __restrict__ counts, int32_t* __restrict__ offsets,
                     int32_t* __restrict__ perm) {
  extern __shared__ int s_rows[];  // [kScoredWarps][E]
  __shared__ int s_total[OLED_MAX_EXPERTS];
  __shared__ int32_t s_ids[kClusterIds];
  __shared__ int s_warp[kScoredWarps];
  __shared__ __align__(16) float s_bias[32 * PER];
  __shared__ int32_t s_experts[kScoredWarps * kExactLanes];
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, n_ctas = gridDim.x, rank = blockIdx.x;
  griddep_launch_dependents();
  for (int i = threadIdx.x; i < kScoredWarps * a.E; i += kScoredThreads) s_rows[i] = 0;
  griddep_wait();
  int first, mine;
  lane_experts(a, lane, first, mine);
  fetch_bias<PER>(a, warp, kScoredWarps, lane, first, mine, s_bias);
  const int begin = min(rank * a.part_tokens, a.T), end = min(begin + a.part_tokens, a.T);
  route_tokens<PER, FULL>(a, begin, end, warp, kScoredWarps, lane, s_bias, first, mine, s_experts, s_ids, nullptr, nullptr);
  __syncthreads();
  place_rows(s_ids, end - begin, a.K, (int64_t)begin * a.K, a.E, s_rows, perm, [&](int e, int total) {
    int all = total, before = 0;
    if (n_ctas > 1) {
      if (e < a.E) s_total[e] = total;
      cluster_sync_all();
      if (e < a.E) {
        all = 0;
        const uint32_t at = smem_u32(&s_total[e]);
        int v[8];
#pragma unroll
        for (int c = 0; c < 8; ++c)
          if (c < n_ctas) asm volatile("ld.shared::cluster.u32 %0, [%1];" : "=r"(v[c]) : "r"(map_to_cta(at, (uint32_t)c)) : "memory");
#pragma unroll
        for (int c = 0; c < 8; ++c)
          if (c < n_ctas) {
            if (c < rank) before += v[c];
            all += v[c];
          }
      }
    }
    const int start = cta_prefix<kScoredWarps>(e < a.E ? all : 0, s_warp);
    if (rank == 0 && e < a.E) {
      counts[e] = all;
      offsets[e] = start;
      if (e == a.E - 1) offsets[a.E] = start + all;
    }
    return start + before;
  });
  if (n_ctas > 1) cluster_sync_all();  // nobody leaves while another CTA may still read its counts
}

// How many CTAs share a routing of T tokens.  Up to kOneLaunch assignments a cluster sorts its own, which takes no scratch;
// beyond, routing leaves a histogram per CTA and a second kernel of as many CTAs sorts.  A warp takes four tokens and more only where every
// SM has that many.
bool one_launch(int T, int K) { return (int64_t)T * K <= kOneLaunch; }
int scored_parts(int T) {
  const int parts = std::min((T + 3) / 4, kScoredCtas);
  const int part_tokens = (T + parts - 1) / parts;
  return (T + part_tokens - 1) / part_tokens;  // (none of them empty)
}
int hist_stride(int E) { return (E + 3) / 4 * 4; }
int cluster_ctas(int T) {
  int n = 1;
  while (n < 8 && n * kScoredWarps < T) n *= 2;
  return n;
}

bool routing_ok(const oled_routing* r) {
  if (!r) return false;
  if (r->n_experts <= 0 || r->n_experts > OLED_MAX_EXPERTS || r->top_k <= 0 || r->top_k > OLED_MAX_TOPK ||
      (r->score != OLED_SCORE_SOFTMAX && r->score != OLED_SCORE_SIGMOID) || r->n_groups <= 0 || r->n_groups > 32 ||
      r->n_experts % r->n_groups != 0 || r->top_groups <= 0 || r->top_groups > r->n_groups || r->group_top < 1 || r->group_top > 2 ||
      (r->renormalise != 0 && r->renormalise != 1) || !std::isfinite(r->scale))
    return false;
  const int size = r->n_experts / r->n_groups;
  if (r->n_groups > 1 && r->group_top > size) return false;
  return r->top_k <= r->top_groups * size;
}

ScoredArgs scored_args(const oled_routing& r, const float* logits, int64_t stride, const float* bias, int T, int32_t* ids, float* gate) {
  ScoredArgs a{};
  a.logits = logits;
  a.bias = bias;
  a.stride = stride;
  a.ids = ids;
  a.gate = gate;
  a.T = T;
  a.E = r.n_experts;
  a.K = r.top_k;
  a.G = r.n_groups;
  a.top_groups = r.top_groups;
  a.group_top = r.group_top;
  a.softmax = r.score == OLED_SCORE_SOFTMAX;
  a.renormalise = r.renormalise;
  a.scale = r.scale;
  // (a token that may use every group has no use for them)
  if (a.top_groups == a.G) a.G = a.top_groups = 1;
  a.group_size = a.E / a.G;
  a.lanes_log2 = 5;
  while ((32 >> a.lanes_log2) < a.G) --a.lanes_log2;
  const int lanes = a.lanes_per_group = 1 << a.lanes_log2;
  a.per_lane = (a.group_size + lanes - 1) / lanes;
  // 16-byte loads where every lane's experts are whole vectors on 16-byte boundaries
  a.vec = a.per_lane % 4 == 0 && a.group_size % 4 == 0 && stride % 4 == 0 && !off_boundary(logits, 16);
  return a;
}

// Calls f with the kernel's PER and FULL as constants.
template <typename F>
cudaError_t with_layout(const ScoredArgs& a, F f) {
  // FULL: as many lanes as there are have as many experts as the kernel has room for
  const bool full = a.lanes_per_group * a.G == 32 && a.per_lane * a.lanes_per_group == a.group_size;
  using std::integral_constant;
  auto pick = [&](auto per) {
    if (full && a.per_lane == decltype(per)::value) return f(per, integral_constant<bool, true>{});
    return f(per, integral_constant<bool, false>{});
  };
  if (a.per_lane <= 2) return pick(integral_constant<int, 2>{});
  if (a.per_lane <= 4) return pick(integral_constant<int, 4>{});
  if (a.per_lane <= 8) return pick(integral_constant<int, 8>{});
  if (a.per_lane <= 16) return pick(integral_constant<int, 16>{});
  return f(integral_constant<int, 32>{}, integral_constant<bool, false>{});  // (full lanes have 16 experts at most)
}

cudaError_t launch_scored(cudaStream_t st, const ScoredArgs& a, int ctas) {
  const size_t smem = (a.scores != nullptr ? (size_t)a.E * 8 : 0) + (a.hist != nullptr || a.counts != nullptr ? (size_t)a.E * 4 : 0);
  return with_layout(a, [&](auto per, auto full) {
    return launch_pdl(route_scored_kernel<decltype(per)::value, decltype(full)::value>, dim3((unsigned)ctas),
                      dim3(32 * std::min(route_warps(decltype(per)::value), a.part_tokens)), smem, st, a);
  });
}

cudaError_t launch_route_cluster(cudaStream_t st, const ScoredArgs& a, int ctas, int32_t* counts, int32_t* offsets, int32_t* perm) {
  return with_layout(a, [&](auto per, auto full) {
    return launch_cluster(route_cluster_kernel<decltype(per)::value, decltype(full)::value>, dim3((unsigned)ctas), dim3(kScoredThreads),
                          (size_t)kScoredWarps * a.E * sizeof(int), st, ctas, a, counts, offsets, perm);
  });
}

}  // namespace

bool routing_valid(const oled_routing* r) { return routing_ok(r); }

// The routing of a step: counts, per-segment counts and reuse-score numerators are added to zeroed arrays.
cudaError_t launch_route_step(cudaStream_t st, const oled_routing& r, const float* logits, const float* bias, const float* conf,
                              int T, int32_t* ids, float* gate, int32_t* counts, unsigned long long* scores, int32_t* seg_counts,
                              int seg_tokens) {
  ScoredArgs a = scored_args(r, logits, r.n_experts, bias, T, ids, gate);
  a.counts = counts;
  a.scores = scores;
  a.conf = conf;
  a.seg_counts = seg_counts;
  int segments = 1;
  a.seg_tokens = T;
  a.parts = scored_parts(T);
  if (seg_counts != nullptr) {
    segments = (T + seg_tokens - 1) / seg_tokens;
    a.seg_tokens = seg_tokens;
    a.parts = std::max(1, std::min((seg_tokens + 3) / 4, kScoredCtas / segments));
  }
  a.part_tokens = (a.seg_tokens + a.parts - 1) / a.parts;
  return launch_scored(st, a, segments * a.parts);
}

}  // namespace oled

extern "C" size_t oled_route_scored_scratch(const oled_routing* routing, int32_t n_tokens) {
  using namespace oled;
  if (!routing_ok(routing) || n_tokens <= 0 || n_tokens > OLED_MAX_ROUTE_TOKENS || one_launch(n_tokens, routing->top_k)) return 0;
  return (size_t)scored_parts(n_tokens) * (size_t)hist_stride(routing->n_experts) * sizeof(uint16_t) + 4;  // (+ 4: on 8-byte boundaries)
}

extern "C" int oled_route_scored(const oled_routing* routing, const float* logits, int64_t logits_stride, const float* bias,
                                 int32_t n_tokens, void* cuda_stream, int32_t* ids, float* gate, int32_t* counts, int32_t* offsets,
                                 int32_t* perm, void* scratch, size_t scratch_bytes) {
  using namespace oled;
  if (!routing_ok(routing) || n_tokens < 0 || !stride_ok(logits_stride, routing->n_experts)) return OLED_ERR_INVALID_ARG;
  if (n_tokens > OLED_MAX_ROUTE_TOKENS) return OLED_ERR_TOO_MANY_TOKENS;
  const bool order = counts != nullptr;
  if (order != (offsets != nullptr) || (n_tokens > 0 && order != (perm != nullptr))) return OLED_ERR_INVALID_ARG;
  if (off_boundary(logits, 4) || off_boundary(bias, 4) || off_boundary(ids, 4) || off_boundary(gate, 4) || off_boundary(counts, 4) ||
      off_boundary(offsets, 4) || off_boundary(perm, 4) || off_boundary(scratch, 4))
    return OLED_ERR_INVALID_ARG;
  cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
  const int E = routing->n_experts, K = routing->top_k, T = n_tokens;
  if (T == 0) {
    if (order && (cudaMemsetAsync(counts, 0, (size_t)E * sizeof(int32_t), st) != cudaSuccess ||
                  cudaMemsetAsync(offsets, 0, (size_t)(E + 1) * sizeof(int32_t), st) != cudaSuccess)) {
      cudaGetLastError();
      return OLED_ERR_CUDA;
    }
    return OLED_OK;
  }
  if (!logits || !ids || !gate) return OLED_ERR_INVALID_ARG;
  const bool whole = !order || one_launch(T, K);
  if (!whole && (!scratch || scratch_bytes < oled_route_scored_scratch(routing, T))) return OLED_ERR_INVALID_ARG;
  {
    const int64_t n = (int64_t)T * K * 4;
    const RowRange r[] = {{logits, logits_stride * 4, (int64_t)E * 4, T}, {bias, 0, (int64_t)E * 4, 1}, {ids, 0, n, 1}, {gate, 0, n, 1},
                          {counts, 0, (int64_t)E * 4, 1}, {offsets, 0, (int64_t)(E + 1) * 4, 1}, {perm, 0, n, 1},
                          {whole ? nullptr : scratch, 0, (int64_t)oled_route_scored_scratch(routing, T), 1}};
    for (int i = 2; i < 8; ++i)
      for (int j = 0; j < i; ++j)
        if (rows_overlap(r[i], r[j])) return OLED_ERR_INVALID_ARG;
  }
  ScoredArgs a = scored_args(*routing, logits, logits_stride, bias, T, ids, gate);
  a.seg_tokens = T;
  cudaError_t err;
  if (order && whole) {
    const int ctas = cluster_ctas(T);
    a.part_tokens = (T + ctas - 1) / ctas;
    err = launch_route_cluster(st, a, ctas, counts, offsets, perm);
  } else {
    a.parts = scored_parts(T);
    a.part_tokens = (T + a.parts - 1) / a.parts;
    if (order) a.hist = reinterpret_cast<uint16_t*>((reinterpret_cast<uintptr_t>(scratch) + 7) & ~(uintptr_t)7);
    a.hist_stride = hist_stride(E);
    err = launch_scored(st, a, a.parts);
    // (it indexes by what the routing has stored: it is launched only behind one that was)
    if (err == cudaSuccess && order) err = cudaFuncSetAttribute(place_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)kPlaceSmem);
    if (err == cudaSuccess && order)
      err = launch_pdl(place_kernel, dim3((unsigned)a.parts), dim3(kScoredThreads), kPlaceSmem, st,
                       (const int32_t*)ids, T, K, E, a.part_tokens, (const uint16_t*)a.hist, a.hist_stride, counts, offsets, perm);
  }
  return cudaGetLastError() == cudaSuccess && err == cudaSuccess ? OLED_OK : OLED_ERR_CUDA;
}
