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
// the same warp.  That is a few tokens in a thousand with a bias, none without one (logits are compared as they are).
//
// A warp per token.  Its lanes are dealt to the groups (32 / G each, G rounded up to a power of two), a lane's experts are
// consecutive, so that lower lanes hold lower experts and a group never shares a lane with another.  Every lane
// sorts its keys once (a network of maxima and minima in registers); then each of the top_k rounds is one warp maximum
// over the lanes' heads, a vote for the lowest lane that has it, and a shift in that lane.
// Bound by the instructions of a token (some 250 at 256 experts top-8; the logits' bytes would take a third of the time).
#include <algorithm>
#include <cmath>

#include "kernels.h"
#include "route_math.h"
#include "row_args.h"

namespace oled {
namespace {

constexpr int kScoredWarps = 8;
constexpr int kScoredThreads = kScoredWarps * 32;

struct ScoredArgs {
  const float* logits;
  const float* bias;
  int64_t stride;
  int32_t* ids;
  float* gate;
  int T, E, K, G, top_groups, group_top, softmax, renormalise;
  float scale;
  int group_size, lanes_per_group, per_lane, vec;
  // tokens of CTA c: segment c / parts, of seg_tokens tokens, and there the part c % parts, of part_tokens
  int parts, seg_tokens, part_tokens;
  // (nullptr: not wanted) per expert and CTA, [E][n_ctas]
  int32_t* hist;
  // (nullptr: not wanted) zeroed arrays of a step: counts [E], per-segment counts [n_segments][E], reuse-score numerators [E]
  int32_t* counts;
  int32_t* seg_counts;
  unsigned long long* scores;
  const float* conf;
};

__device__ __forceinline__ float key_value(uint32_t key) {
  return __uint_as_float((key & 0x80000000u) ? key ^ 0x80000000u : ~key);
}
__device__ __forceinline__ float warp_max(float v) {
#pragma unroll
  for (int d = 16; d >= 1; d >>= 1) v = fmaxf(v, __shfl_xor_sync(0xffffffffu, v, d));
  return v;
}
__device__ __forceinline__ float warp_sum(float v) {
#pragma unroll
  for (int d = 16; d >= 1; d >>= 1) v += __shfl_xor_sync(0xffffffffu, v, d);
  return v;
}
__device__ __forceinline__ float no_nan(float v) { return v == v ? v : __int_as_float(0xff800000); }
// exp(l - top): one for the largest logit even where it is infinite
__device__ __forceinline__ float softmax_term(float l, float top) { return l == top ? 1.0f : __expf(l - top); }

// Descending order of N keys in registers.
template <int N>
__device__ __forceinline__ void sort_desc(uint32_t (&k)[N]) {
#pragma unroll
  for (int size = 2; size <= N; size <<= 1)
#pragma unroll
    for (int step = size >> 1; step >= 1; step >>= 1)
#pragma unroll
      for (int i = 0; i < N; ++i) {
        const int j = i ^ step;
        if (j > i) {
          const uint32_t hi = max(k[i], k[j]), lo = min(k[i], k[j]);
          const bool down = (i & size) == 0 || size == N;
          k[i] = down ? hi : lo;
          k[j] = down ? lo : hi;
        }
      }
}

// The choice of one token in fp64, by a warp: lane r < K ends with the id of rank r.  Experts e = lane + 32 i.  (Loops that
// are not unrolled keep the arrays in local memory: the registers of this rare path count for the whole kernel.)
__device__ __noinline__ int select_exact(const ScoredArgs& a, const float* row, int lane) {
  constexpr int kPer = OLED_MAX_EXPERTS / 32;
  const double kNone = -INFINITY;
  double score[kPer], choice[kPer];
  double top = kNone;
#pragma unroll 1
  for (int i = 0; i < kPer; ++i) {
    const int e = lane + 32 * i;
    score[i] = e < a.E ? (double)no_nan(row[e]) : kNone;
    top = fmax(top, score[i]);
  }
  for (int d = 16; d >= 1; d >>= 1) top = fmax(top, __shfl_xor_sync(0xffffffffu, top, d));
  double sum = 0.0;
#pragma unroll 1
  for (int i = 0; i < kPer; ++i) {
    const int e = lane + 32 * i;
    if (e >= a.E) continue;
    const double l = score[i];
    score[i] = a.softmax ? (l == top ? 1.0 : exp(l - top)) : 1.0 / (1.0 + exp(-l));
    sum += score[i];
    choice[i] = a.bias != nullptr ? 0.0 : l;
  }
  for (int d = 16; d >= 1; d >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, d);
  uint32_t allowed = 0xffffffffu;  // groups
#pragma unroll 1
  for (int i = 0; i < kPer; ++i) {
    const int e = lane + 32 * i;
    if (e >= a.E) continue;
    if (a.softmax) score[i] /= sum;
    if (a.bias != nullptr) {
      const double c = score[i] + (double)a.bias[e];
      choice[i] = row[e] == row[e] && c == c ? c : kNone;
      score[i] = choice[i];
    }
  }
  if (a.G > 1 && a.top_groups < a.G) {
    double mine = kNone;  // the value of group `lane`
#pragma unroll 1
    for (int g = 0; g < a.G; ++g) {
      double t1 = kNone, t2 = kNone;
#pragma unroll 1
      for (int i = 0; i < kPer; ++i) {
        const int e = lane + 32 * i;
        if (e < g * a.group_size || e >= (g + 1) * a.group_size) continue;
        const double v = a.group_top == 1 ? choice[i] : score[i];
        t2 = fmax(t2, fmin(t1, v));
        t1 = fmax(t1, v);
      }
      for (int d = 16; d >= 1; d >>= 1) {
        const double o1 = __shfl_xor_sync(0xffffffffu, t1, d), o2 = __shfl_xor_sync(0xffffffffu, t2, d);
        t2 = fmax(fmin(t1, o1), fmax(t2, o2));
        t1 = fmax(t1, o1);
      }
      double v = a.group_top == 1 ? t1 : t1 + t2;
      if (!(v == v)) v = kNone;
      if (lane == g) mine = v;
    }
    int before = 0;
#pragma unroll 1
    for (int g = 0; g < a.G; ++g) {
      const double v = __shfl_sync(0xffffffffu, mine, g);
      before += v > mine || (v == mine && g < lane);
    }
    allowed = __ballot_sync(0xffffffffu, lane < a.G && before < a.top_groups);
  }
  uint32_t left = 0u;
#pragma unroll 1
  for (int i = 0; i < kPer; ++i) {
    const int e = lane + 32 * i;
    if (e < a.E && ((allowed >> (e / a.group_size)) & 1u)) left |= 1u << i;
  }
  int id = 0;
#pragma unroll 1
  for (int r = 0; r < a.K; ++r) {
    double bv = 0.0;
    int be = 0x7fffffff;
#pragma unroll 1
    for (int i = 0; i < kPer; ++i)
      if ((left >> i) & 1u)
        if (be == 0x7fffffff || choice[i] > bv) {
          bv = choice[i];
          be = lane + 32 * i;
        }
    for (int d = 16; d >= 1; d >>= 1) {
      const double ov = __shfl_xor_sync(0xffffffffu, bv, d);
      const int oe = __shfl_xor_sync(0xffffffffu, be, d);
      if (oe != 0x7fffffff && (be == 0x7fffffff || ov > bv || (ov == bv && oe < be))) {
        bv = ov;
        be = oe;
      }
    }
    if ((be & 31) == lane) left &= ~(1u << (be >> 5));
    if (lane == r) id = be;
  }
  return id;
}

// Could the fp32 forms of two choices a >= b be in the wrong order?  A sigmoid is off by at most 2^-22 (exp: argument and
// ex2 2^-22 + |l| 2^-24 relative, times s (1 - s); sum and quotient 2^-23 + 2^-24), a softmax score by at most 2^-18 of
// the largest score (its sum of up to 512 terms in at most 37 rounded steps), the addition of the bias by 2^-24 of the result;
// `slack` is twice the scores' part and a fifth more.  Differences of infinities are NaN: not told apart here either.
__device__ __forceinline__ bool near_choices(float a, float b, float slack) {
  return !(a - b > slack + 2.4e-7f * fmaxf(fabsf(a), fabsf(b)));
}

// PER: experts a lane has room for.
template <int PER>
__device__ __forceinline__ void route_token(const ScoredArgs& a, int t, int lane, const float (&bias)[PER], int first, int mine,
                                            int32_t* s_counts, unsigned long long* s_scores) {
  const float* const row = a.logits + (int64_t)t * a.stride;
  float l[PER];
  if (a.vec) {
#pragma unroll
    for (int i = 0; i < PER; i += 4)
      if (PER >= 4 && i < mine) {
        const float4 v = *reinterpret_cast<const float4*>(row + first + i);
        l[i] = v.x;
        if (i + 1 < PER) l[i + 1] = v.y;
        if (i + 2 < PER) l[i + 2] = v.z;
        if (i + 3 < PER) l[i + 3] = v.w;
      }
  } else {
#pragma unroll
    for (int i = 0; i < PER; ++i)
      if (i < mine) l[i] = row[first + i];
  }
  const float kNone = __int_as_float(0xff800000);
  float top = kNone, sum = 1.0f;
  uint32_t nan = 0u;
#pragma unroll
  for (int i = 0; i < PER; ++i) {
    if (i >= mine) l[i] = kNone;
    if (!(l[i] == l[i])) {
      nan |= 1u << i;
      l[i] = kNone;
    }
  }
  float c[PER];
#pragma unroll
  for (int i = 0; i < PER; ++i) c[i] = l[i];
  if (a.softmax) {
#pragma unroll
    for (int i = 0; i < PER; ++i) top = fmaxf(top, l[i]);
    top = warp_max(top);
    sum = 0.0f;
#pragma unroll
    for (int i = 0; i < PER; ++i) {
      const float z = i < mine ? softmax_term(l[i], top) : 0.0f;
      sum += z;
      if (a.bias != nullptr) c[i] = z;
    }
    sum = warp_sum(sum);
  }
  const float inverse = __fdividef(1.0f, sum);
  float slack = 0.0f;
  bool near = false;
  if (a.bias != nullptr) {
    slack = a.softmax ? 9.2e-6f * inverse : 5.8e-7f;
#pragma unroll
    for (int i = 0; i < PER; ++i) {
      const float s = a.softmax ? c[i] * inverse : __fdividef(1.0f, 1.0f + __expf(-l[i]));
      c[i] = (nan >> i) & 1u ? kNone : no_nan(s + bias[i]);
    }
  }
  uint32_t key[PER], sorted[PER];
#pragma unroll
  for (int i = 0; i < PER; ++i) key[i] = i < mine ? order_key(__fadd_rn(c[i], 0.0f)) : 0u;  // (-0 as +0)
  if (a.G > 1 && a.top_groups < a.G) {
    float t1 = kNone, t2 = kNone;
#pragma unroll
    for (int i = 0; i < PER; ++i)
      if (i < mine) {
        t2 = fmaxf(t2, fminf(t1, c[i]));
        t1 = fmaxf(t1, c[i]);
      }
    for (int d = a.lanes_per_group >> 1; d >= 1; d >>= 1) {
      const float o1 = __shfl_xor_sync(0xffffffffu, t1, d), o2 = __shfl_xor_sync(0xffffffffu, t2, d);
      t2 = fmaxf(fminf(t1, o1), fmaxf(t2, o2));
      t1 = fmaxf(t1, o1);
    }
    float value = t1, group_slack = slack;
    const bool exact = a.bias == nullptr && a.group_top == 1;
    if (a.group_top == 2) {
      if (a.bias == nullptr) {  // the order of scores is that of logits
        if (a.softmax) {
          t1 = softmax_term(t1, top) * inverse;
          t2 = softmax_term(t2, top) * inverse;
          group_slack = 9.2e-6f * inverse;
        } else {
          t1 = __fdividef(1.0f, 1.0f + __expf(-t1));
          t2 = __fdividef(1.0f, 1.0f + __expf(-t2));
          group_slack = 5.8e-7f;
        }
      }
      value = no_nan(t1 + t2);
      group_slack *= 2.0f;
    }
    const int g = lane / a.lanes_per_group;
    int before = 0;
    for (int o = 0; o < a.G; ++o) {
      const float v = __shfl_sync(0xffffffffu, value, o * a.lanes_per_group);
      before += v > value || (v == value && o < g);
      if (!exact && o != g && g < a.G) near = near || near_choices(fmaxf(v, value), fminf(v, value), group_slack);
    }
    if (before >= a.top_groups) {
#pragma unroll
      for (int i = 0; i < PER; ++i) key[i] = 0u;
    }
  }
#pragma unroll
  for (int i = 0; i < PER; ++i) sorted[i] = key[i];
  sort_desc<PER>(sorted);
  uint32_t my_key = 0u, next = 0u;
  int my_lane = 0;
  for (int r = 0; r < a.K; ++r) {
    const uint32_t best = __reduce_max_sync(0xffffffffu, sorted[0]);
    const int winner = __ffs((int)__ballot_sync(0xffffffffu, sorted[0] == best)) - 1;
    if (lane == r) {
      my_key = best;
      my_lane = winner;
    }
    if (lane == winner) {
#pragma unroll
      for (int i = 0; i + 1 < PER; ++i) sorted[i] = sorted[i + 1];
      sorted[PER - 1] = 0u;
    }
  }
  next = __reduce_max_sync(0xffffffffu, sorted[0]);
  {
    uint32_t after = __shfl_down_sync(0xffffffffu, my_key, 1);
    if (lane == a.K - 1) after = next;
    if (a.bias != nullptr && lane < a.K && after != 0u) near = near || near_choices(key_value(my_key), key_value(after), slack);
  }
  int id;
  if (__any_sync(0xffffffffu, near)) {
    id = select_exact(a, row, lane);
  } else {
    // equal keys of one lane are taken in the order of their indices
    int skip = 0;
    {
      const uint32_t before = __shfl_up_sync(0xffffffffu, my_key, 1);
      if (__any_sync(0xffffffffu, lane > 0 && lane < a.K && before == my_key)) {
        const uint32_t same = __match_any_sync(0xffffffffu, my_key) & __match_any_sync(0xffffffffu, my_lane);
        skip = __popc(same & ((1u << lane) - 1u));
      }
    }
    int at = 0;
#pragma unroll
    for (int i = 0; i < PER; ++i) {
      const uint32_t k = __shfl_sync(0xffffffffu, key[i], my_lane);
      if (k == my_key) {
        if (skip == 0) at = i;
        --skip;
      }
    }
    id = __shfl_sync(0xffffffffu, first, my_lane) + at;
  }
  // the chosen experts' weights
  float s = 0.0f;
  if (lane < a.K) {
    const float x = no_nan(row[id]);
    s = a.softmax ? (x == top ? 1.0f : expf(x - top)) : __fdiv_rn(1.0f, 1.0f + expf(-x));
  }
  float w = s;
  if (a.renormalise) w = __fdiv_rn(s, warp_sum(s) + 1e-20f * sum);  // (softmax: s is sum times the score)
  else if (a.softmax) w = __fdiv_rn(s, sum);
  if (lane < a.K) {
    a.ids[(int64_t)t * a.K + lane] = id;
    a.gate[(int64_t)t * a.K + lane] = w * a.scale;
    if (s_counts != nullptr) atomicAdd(&s_counts[id], 1);
    // (the numerators take the weight before its scale, at most one: their sums are reported in 48 bits)
    if (s_scores != nullptr) atomicAdd(&s_scores[id], score_quantum(w, a.conf[t]));
  }
}

// Dynamic shared memory: [E] scores (where wanted), [E] counts (where wanted).
template <int PER>
__global__ void __launch_bounds__(kScoredThreads)
route_scored_kernel(const __grid_constant__ ScoredArgs a) {
  extern __shared__ __align__(16) uint8_t s_dyn[];
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  unsigned long long* const s_scores = a.scores != nullptr ? reinterpret_cast<unsigned long long*>(s_dyn) : nullptr;
  const bool counting = a.hist != nullptr || a.counts != nullptr;
  int32_t* const s_counts = counting ? reinterpret_cast<int32_t*>(s_dyn + (s_scores != nullptr ? (size_t)a.E * 8 : 0)) : nullptr;
  griddep_launch_dependents();
  if (counting) {
    for (int e = threadIdx.x; e < a.E; e += kScoredThreads) {
      s_counts[e] = 0;
      if (s_scores != nullptr) s_scores[e] = 0ull;
    }
    __syncthreads();
  }
  griddep_wait();
  const int g = lane / a.lanes_per_group, sub = lane - g * a.lanes_per_group;
  const int first = g < a.G ? g * a.group_size + sub * a.per_lane : 0;
  const int mine = g < a.G ? max(0, min(a.per_lane, a.group_size - sub * a.per_lane)) : 0;
  float bias[PER];
#pragma unroll
  for (int i = 0; i < PER; ++i) bias[i] = a.bias != nullptr && i < mine ? a.bias[first + i] : 0.0f;
  const int seg = (int)blockIdx.x / a.parts, part = (int)blockIdx.x - seg * a.parts;
  const int begin = seg * a.seg_tokens + part * a.part_tokens;
  const int end = min(min(begin + a.part_tokens, (seg + 1) * a.seg_tokens), a.T);
  for (int t = begin + warp; t < end; t += kScoredWarps) route_token<PER>(a, t, lane, bias, first, mine, s_counts, s_scores);
  if (!counting) return;
  __syncthreads();
  for (int e = threadIdx.x; e < a.E; e += kScoredThreads) {
    const int n = s_counts[e];
    if (a.hist != nullptr) a.hist[(size_t)e * gridDim.x + blockIdx.x] = n;
    if (n == 0) continue;
    if (a.counts != nullptr) atomicAdd(&a.counts[e], n);
    if (a.seg_counts != nullptr) atomicAdd(&a.seg_counts[seg * a.E + e], n);
    if (s_scores != nullptr && s_scores[e] != 0ull) atomicAdd(&a.scores[e], s_scores[e]);
  }
}

// ---- the order by expert ----------------------------------------------------------------------
constexpr int kSortWarps = 16;

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

// counts and prefixes of an expert over the CTAs: a warp per expert, in place.
__global__ void __launch_bounds__(256)
scan_hist_kernel(int32_t* hist, int n_ctas, int E, int32_t* counts) {
  const int e = (int)blockIdx.x * 8 + ((int)threadIdx.x >> 5), lane = threadIdx.x & 31;
  griddep_launch_dependents();
  griddep_wait();
  if (e >= E) return;
  int32_t* const row = hist + (size_t)e * n_ctas;
  int carry = 0;
  for (int i0 = 0; i0 < n_ctas; i0 += 128) {  // four values a lane at a time
    int v[4], sum = 0;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const int i = i0 + lane * 4 + j;
      v[j] = i < n_ctas ? row[i] : 0;
      sum += v[j];
    }
    int incl = sum;
#pragma unroll
    for (int d = 1; d < 32; d <<= 1) {
      const int o = __shfl_up_sync(0xffffffffu, incl, d);
      if (lane >= d) incl += o;
    }
    int at = carry + incl - sum;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const int i = i0 + lane * 4 + j;
      if (i < n_ctas) row[i] = at;
      at += v[j];
    }
    carry += __shfl_sync(0xffffffffu, incl, 31);
  }
  if (lane == 0) counts[e] = carry;
}

// Rows of one CTA's assignments in the stable order by expert.  hist == nullptr: one CTA has them all and makes the
// counts too.  Every warp counts the experts of a contiguous part, then hands out its part's rows in order.
__global__ void __launch_bounds__(kSortWarps * 32)
place_kernel(const int32_t* __restrict__ ids, int T, int K, int E, int part_tokens, const int32_t* __restrict__ hist,
             int32_t* counts, int32_t* __restrict__ offsets, int32_t* __restrict__ perm) {
  extern __shared__ int s_rows[];  // [kSortWarps][E]
  __shared__ int s_warp[kSortWarps];
  static_assert(kSortWarps * 32 >= OLED_MAX_EXPERTS, "a thread per expert");
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  griddep_launch_dependents();
  for (int i = threadIdx.x; i < kSortWarps * E; i += kSortWarps * 32) s_rows[i] = 0;
  griddep_wait();
  __syncthreads();
  const int64_t a0 = (int64_t)blockIdx.x * part_tokens * K, a1 = min(a0 + (int64_t)part_tokens * K, (int64_t)T * K);
  const int n = (int)(a1 - a0), per_warp = (n + kSortWarps * 32 - 1) / (kSortWarps * 32) * 32;
  const int first = warp * per_warp, last = min(n, first + per_warp);
  int* const mine = s_rows + warp * E;
  for (int i0 = first; i0 < last; i0 += 32)
    if (i0 + lane < last) atomicAdd(&mine[ids[a0 + i0 + lane]], 1);
  __syncthreads();
  const int e = threadIdx.x;
  int total = 0;
  if (e < E) {
    for (int w = 0; w < kSortWarps; ++w) {
      const int c = s_rows[w * E + e];
      s_rows[w * E + e] = total;
      total += c;
    }
    if (hist == nullptr) counts[e] = total;
    else total = counts[e];
  }
  int start = cta_prefix<kSortWarps>(e < E ? total : 0, s_warp);
  if (e < E) {
    if (blockIdx.x == 0) {
      offsets[e] = start;
      if (e == E - 1) offsets[E] = start + total;
    }
    if (hist != nullptr) start += hist[(size_t)e * gridDim.x + blockIdx.x];
    for (int w = 0; w < kSortWarps; ++w) s_rows[w * E + e] += start;
  }
  __syncthreads();
  for (int i0 = first; i0 < last; i0 += 32) {
    const int id = i0 + lane < last ? ids[a0 + i0 + lane] : -1;
    const uint32_t same = __match_any_sync(0xffffffffu, id);
    const int rank = __popc(same & ((1u << lane) - 1u));
    if (id >= 0) perm[mine[id] + rank] = (int32_t)(a0 + i0 + lane);
    __syncwarp();
    if (id >= 0 && rank == 0) mine[id] += __popc(same);
    __syncwarp();
  }
}

// How many CTAs share a routing of T tokens, and how.  Up to kOneSort assignments are sorted by one CTA, which takes no
// scratch; beyond, a CTA sorts what it routed and a kernel in between adds up the CTAs' histograms.
constexpr int kOneSort = 4096;
constexpr int kScoredCtas = 148 * 4;
bool one_sort(int T, int K) { return (int64_t)T * K <= kOneSort; }
int scored_parts(int T) {
  const int parts = std::min((T + kScoredWarps - 1) / kScoredWarps, kScoredCtas);
  const int part_tokens = (T + parts - 1) / parts;
  return (T + part_tokens - 1) / part_tokens;  // (none of them empty)
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
  int lanes = 32;
  while (32 / lanes < a.G) lanes >>= 1;
  a.lanes_per_group = lanes;
  a.per_lane = (a.group_size + lanes - 1) / lanes;
  // 16-byte loads where every lane's experts are whole vectors on 16-byte boundaries
  a.vec = a.per_lane % 4 == 0 && a.group_size % 4 == 0 && stride % 4 == 0 && !off_boundary(logits, 16);
  return a;
}

cudaError_t launch_scored(cudaStream_t st, const ScoredArgs& a, int ctas) {
  const size_t smem = (a.scores != nullptr ? (size_t)a.E * 8 : 0) + (a.hist != nullptr || a.counts != nullptr ? (size_t)a.E * 4 : 0);
  const dim3 grid((unsigned)ctas), block(kScoredThreads);
  if (a.per_lane <= 2) return launch_pdl(route_scored_kernel<2>, grid, block, smem, st, a);
  if (a.per_lane <= 4) return launch_pdl(route_scored_kernel<4>, grid, block, smem, st, a);
  if (a.per_lane <= 8) return launch_pdl(route_scored_kernel<8>, grid, block, smem, st, a);
  if (a.per_lane <= 16) return launch_pdl(route_scored_kernel<16>, grid, block, smem, st, a);
  return launch_pdl(route_scored_kernel<32>, grid, block, smem, st, a);
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
    a.parts = std::max(1, std::min((seg_tokens + kScoredWarps - 1) / kScoredWarps, kScoredCtas / segments));
  }
  a.part_tokens = (a.seg_tokens + a.parts - 1) / a.parts;
  return launch_scored(st, a, segments * a.parts);
}

}  // namespace oled

extern "C" size_t oled_route_scored_scratch(const oled_routing* routing, int32_t n_tokens) {
  using namespace oled;
  if (!routing_ok(routing) || n_tokens <= 0 || n_tokens > OLED_MAX_ROUTE_TOKENS || one_sort(n_tokens, routing->top_k)) return 0;
  return (size_t)scored_parts(n_tokens) * (size_t)routing->n_experts * sizeof(int32_t);
}

extern "C" int oled_route_scored(const oled_routing* routing, const float* logits, int64_t logits_stride, const float* bias,
                                 int32_t n_tokens, void* cuda_stream, int32_t* ids, float* gate, int32_t* counts, int32_t* offsets,
                                 int32_t* perm, void* scratch, size_t scratch_bytes) {
  using namespace oled;
  if (!routing_ok(routing) || n_tokens < 0 || logits_stride < routing->n_experts) return OLED_ERR_INVALID_ARG;
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
  const bool whole = !order || one_sort(T, K);
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
  a.parts = scored_parts(T);
  a.seg_tokens = T;
  a.part_tokens = (T + a.parts - 1) / a.parts;
  if (!whole) a.hist = static_cast<int32_t*>(scratch);
  cudaError_t err = launch_scored(st, a, a.parts);
  const size_t smem = (size_t)kSortWarps * E * sizeof(int);
  // (each of these indexes by what the one before has stored: it is launched only behind one that was)
  if (err == cudaSuccess && order && whole)
    err = launch_pdl(place_kernel, dim3(1), dim3(kSortWarps * 32), smem, st, (const int32_t*)ids, T, K, E, T, (const int32_t*)nullptr,
                     counts, offsets, perm);
  if (err == cudaSuccess && order && !whole) {
    err = launch_pdl(scan_hist_kernel, dim3((unsigned)((E + 7) / 8)), dim3(256), 0, st, a.hist, a.parts, E, counts);
    if (err == cudaSuccess)
      err = launch_pdl(place_kernel, dim3((unsigned)a.parts), dim3(kSortWarps * 32), smem, st, (const int32_t*)ids, T, K, E,
                       a.part_tokens, (const int32_t*)a.hist, counts, offsets, perm);
  }
  return cudaGetLastError() == cudaSuccess && err == cudaSuccess ? OLED_OK : OLED_ERR_CUDA;
}
