// Routing to experts: scores, groups, the k best, their weights (rk_moe_route), and the list of (token, slot) pairs by
// expert that the expert products walk (rk_moe_group).
#include <cuda_bf16.h>

#include "rk_internal.h"

namespace rk {
namespace {

// ------------------------------------------------------------------------------------------------------------
// rk_moe_route: a warp per token, a few tokens in turn.  The lanes are split evenly over the groups (L lanes per group, L a
// power of two), and a lane holds neighbouring experts of its group, so that a group's rank is a reduction over L lanes and
// the order of lanes and places is the experts' own.
//
// Scores are compared in 64 bits: with a few hundred experts the k-th and the next score of a token are closer than fp32
// rounding about once in 10^4 tokens, and the choice would depend on the instruction that computed them.  Hence the order
// is first taken in fp32, and kept where every decision in it (k + 1 neighbouring scores, the last group that takes part and the
// first that does not) is clearer than the error of the fp32 scores, bounded below.  Where only the order of scores is open,
// those few are compared in 64 bits, one per lane; other open tokens are done again as a whole (6 to 10 us more for the call that
// meets one: 777 tokens of 160 experts 11.8 -> 5.7 us, 32768 of 256 39 -> 34).  Equal fp32 logits are open, too, since a key
// holds its place in their last bits: 32768 tokens of nothing but zeros 165 us, in bf16 32.
// The weights of the chosen experts are computed in 64 bits, for the tokens of a warp together.
//
// A warp's cost is instructions, not the logits' bytes: every lane sorts its keys once, and the k rounds of "largest key of
// the warp, its lane moves up" are about 20 each.  32768 tokens, 256 experts, 8 of them, sigmoid and bias: 34 us (33.6 MB of fp32
// logits: 5.2 us); 64 tokens, 8 groups: 4.4 us, most of it launch and code that runs for the first time.  (Device time in a captured
// loop of ten, as all figures here.)
// ------------------------------------------------------------------------------------------------------------
constexpr int kRouteWarps = 2;  // small thread blocks: few tokens spread over more SMs (64 tokens: 4.5 us, with eight 5.2)
constexpr double kNone = -__builtin_huge_val();
constexpr unsigned kAll = 0xffffffffu;

__device__ __forceinline__ double max_f64(double a, double b) { return a > b ? a : b; }

template <bool kBf16>
__device__ __forceinline__ float route_logit(const RouteParams& p, int64_t token, int expert) {
  const int64_t at = token * p.stride + expert;
  return kBf16 ? __bfloat162float(static_cast<const __nv_bfloat16*>(p.logits)[at]) : static_cast<const float*>(p.logits)[at];
}

// The chosen experts in 64 bits: lane q's is returned, -1 where none is left, -2 for a token with a NaN among its scores.
template <int kPer, bool kBf16>
__device__ __noinline__ int route_exact(const RouteParams& p, int64_t token) {
  const int lane = threadIdx.x & 31, width = 1 << p.lanes_log2, g = lane >> p.lanes_log2, sub = lane & (width - 1);
  const int begin = g * p.group_size + sub * p.per, count = g < p.n_groups ? max(0, min(p.per, p.group_size - sub * p.per)) : 0;
  double c[kPer];
  bool bad = false;
  double top = kNone;
#pragma unroll
  for (int i = 0; i < kPer; ++i) {
    const float x = i < count ? route_logit<kBf16>(p, token, begin + i) : -__int_as_float(0x7f800000);
    bad |= x != x;
    c[i] = (double)x;
    top = max_f64(top, c[i]);
  }
  double sum = 0.0;
  if (p.softmax) {
#pragma unroll
    for (int d = 16; d > 0; d >>= 1) top = max_f64(top, __shfl_xor_sync(kAll, top, d));
#pragma unroll 1
    for (int i = 0; i < kPer; ++i) sum += c[i] == kNone ? 0.0 : exp(c[i] - top);
#pragma unroll
    for (int d = 16; d > 0; d >>= 1) sum += __shfl_xor_sync(kAll, sum, d);
  }
#pragma unroll
  for (int i = 0; i < kPer; ++i) {
    if (c[i] == kNone) continue;
    const double e = exp(p.softmax ? c[i] - top : -c[i]);
    c[i] = p.softmax ? e / sum : 1.0 / (1.0 + e);
    if (p.bias) c[i] += (double)p.bias[begin + i];
    bad |= c[i] != c[i];
  }
  if (__any_sync(kAll, bad)) return -2;
  if (p.n_groups > 1) {
    double a = kNone, b = kNone;  // the two largest of the group
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
      b = max_f64(b, a < c[i] ? a : c[i]);
      a = max_f64(a, c[i]);
    }
    for (int d = width >> 1; d > 0; d >>= 1) {
      const double a2 = __shfl_xor_sync(kAll, a, d), b2 = __shfl_xor_sync(kAll, b, d);
      b = max_f64(max_f64(b, b2), a < a2 ? a : a2);
      a = max_f64(a, a2);
    }
    const double rank = p.group_top == 2 && b != kNone ? a + b : a;
    int better = 0;
    for (int h = 0; h < p.n_groups; ++h) {
      const double r = __shfl_sync(kAll, rank, h << p.lanes_log2);
      better += r > rank || (r == rank && h < g);
    }
    if (better >= p.top_groups) {
#pragma unroll
      for (int i = 0; i < kPer; ++i) c[i] = kNone;
    }
  }
  int id = -1;
  for (int q = 0; q < p.k; ++q) {
    double best = kNone;
    int at = 0x7fffffff;
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
      if (c[i] > best) {
        best = c[i];
        at = begin + i;
      }
    }
    const int mine = at;
#pragma unroll
    for (int d = 16; d > 0; d >>= 1) {
      const double b2 = __shfl_xor_sync(kAll, best, d);
      const int a2 = __shfl_xor_sync(kAll, at, d);
      if (b2 > best || (b2 == best && a2 < at)) {
        best = b2;
        at = a2;
      }
    }
    if (best == kNone) break;
    if (mine == at) {
#pragma unroll
      for (int i = 0; i < kPer; ++i)
        if (begin + i == at) c[i] = kNone;
    }
    if (lane == q) id = at;
  }
  return id;
}

// fp32 scores.  exp2 and the reciprocal are right to 2^-22 of their values, the exponent is off by 2^-23.5 |x|:
//   sigmoid  s (1 - s) (2^-22 + |x| 2^-23.5) + 2^-22.5 s  <  2^-21
//   softmax  s (2^-21 + |x - top| 2^-23.5 + 2^-21)        <  2^-17 s   up to |x - top| = 80; what is left below that is 0
// A score plus bias is rounded once (2^-24 of it), and its last bits are the place that it has in its lane.  Without a bias
// the logits themselves are the order, and equal logits are equal scores; only where scores of different logits could round
// to the same 64-bit number (logits closer than 2^-45, sigmoid above 15 or both below -700, next to where exp(-x) overflows and
// scores are 0, softmax both 600 below the largest) is it left open.
__device__ __forceinline__ float exp2_fast(float x) {
  float r;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
  return r;
}
__device__ __forceinline__ float reciprocal_fast(float x) {
  float r;
  asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
  return r;
}
__device__ __forceinline__ float max_nan(float a, float b) {
  float r;
  asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b));
  return r;
}
// numbers as integers of the same order; the transformation is its own inverse
__device__ __forceinline__ int ordered(int bits) { return bits ^ ((bits >> 31) & 0x7fffffff); }
constexpr float kLog2e = 1.44269504088896340736f;
// e^d for d <= 0, right to 2^-31: 2^n times the Taylor series of 2^r to degree 8 (|r| <= 1/2)
__device__ __forceinline__ double exp_31(double d) {
  const double x = d * 1.44269504088896340736, n = rint(x), r = (x - n) * 0.69314718055994530942;
  double e = 1.0 / 40320.0;
  const double c[8] = {1.0 / 5040.0, 1.0 / 720.0, 1.0 / 120.0, 1.0 / 24.0, 1.0 / 6.0, 0.5, 1.0, 1.0};
#pragma unroll
  for (int i = 0; i < 8; ++i) e = fma(e, r, c[i]);
  return x < -1000.0 ? 0.0 : __hiloint2double(__double2hiint(e) + ((int)n << 20), __double2loint(e));
}
// Batcher's odd-even merge sort, descending; the loops unroll into a fixed network
template <int kN>
__device__ __forceinline__ void sort_down(int (&v)[kN]) {
#pragma unroll
  for (int p = 1; p < kN; p *= 2) {
#pragma unroll
    for (int k = p; k >= 1; k /= 2) {
#pragma unroll
      for (int j = k % p; j + k < kN; j += 2 * k) {
#pragma unroll
        for (int i = 0; i < k; ++i) {
          if (i + j + k < kN && (i + j) / (2 * p) == (i + j + k) / (2 * p)) {
            const int lo = min(v[i + j], v[i + j + k]), hi = max(v[i + j], v[i + j + k]);
            v[i + j] = hi;
            v[i + j + k] = lo;
          }
        }
      }
    }
  }
}

template <int kPer, bool kBf16>
__global__ void __launch_bounds__(32 * kRouteWarps, kPer <= 8 ? 14 : 1) moe_route_kernel(const RouteParams p) {
  constexpr int kPlace = kPer <= 2 ? 1 : kPer <= 8 ? 7 : kPer <= 16 ? 15 : kPer <= 32 ? 31 : 63;  // bits of a key for its place
  constexpr float kKeyStep = (float)(kPlace + 2) * 0x1p-23f;                                     // ... and what that and the sum cost
  constexpr int kNoKey = (int)0x80800000;  // no finite number comes below it
  const int lane = threadIdx.x & 31, width = 1 << p.lanes_log2, g = lane >> p.lanes_log2, sub = lane & (width - 1);
  const int span = p.k <= 8 ? 8 : 16, turns = p.turns;  // lanes for a token's choice; tokens of a warp
  const int64_t first = ((int64_t)blockIdx.x * kRouteWarps + (threadIdx.x >> 5)) * turns;
  if (first >= p.n) return;
  const float inf = __int_as_float(0x7f800000);
  // this lane's experts: `count` from `begin` on
  const int begin = g * p.group_size + sub * p.per;
  const int count = g < p.n_groups ? max(0, min(p.per, p.group_size - sub * p.per)) : 0;
  float bias[kPer];
#pragma unroll
  for (int i = 0; i < kPer; ++i) bias[i] = p.bias && i < count ? p.bias[begin + i] : 0.f;
  auto load = [&](int64_t token, float (&x)[kPer]) {
    if constexpr (!kBf16 && kPer % 4 == 0) {
      if (p.whole) {  // every lane has kPer experts, 16-byte aligned
        const float4* src = reinterpret_cast<const float4*>(static_cast<const float*>(p.logits) + token * p.stride + begin);
#pragma unroll
        for (int i = 0; i < kPer / 4; ++i) {
          const float4 v = src[i];
          x[4 * i] = v.x;
          x[4 * i + 1] = v.y;
          x[4 * i + 2] = v.z;
          x[4 * i + 3] = v.w;
        }
        return;
      }
    }
    if constexpr (kBf16 && kPer % 8 == 0) {
      if (p.whole) {
        const uint4* src = reinterpret_cast<const uint4*>(static_cast<const __nv_bfloat16*>(p.logits) + token * p.stride + begin);
#pragma unroll
        for (int i = 0; i < kPer / 8; ++i) {
          const uint4 v = src[i];
          const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
          for (int j = 0; j < 8; ++j) x[8 * i + j] = __uint_as_float(j & 1 ? w[j >> 1] & 0xffff0000u : w[j >> 1] << 16);
        }
        return;
      }
    }
#pragma unroll
    for (int i = 0; i < kPer; ++i) x[i] = i < count ? route_logit<kBf16>(p, token, begin + i) : -inf;
  };
  float ahead[kPer];
  load(first, ahead);
  int id = -1;  // lane turn * span + q: choice q of the token
  double sum = 1.0, top_mine = 0.0;  // of the softmax (that of renormalised weights drops out)
#pragma unroll 1
  for (int turn = 0; turn < turns && first + turn < p.n; ++turn) {
    const int64_t token = first + turn;
    float x[kPer], top = -inf, scale = 1.f;
    int key[kPer];
#pragma unroll
    for (int i = 0; i < kPer; ++i) x[i] = ahead[i];
    if (turn + 1 < turns && token + 1 < p.n) load(token + 1, ahead);
    if (p.softmax) {
#pragma unroll
      for (int i = 0; i < kPer; ++i) top = fmaxf(top, x[i]);
#pragma unroll
      for (int d = 16; d > 0; d >>= 1) top = fmaxf(top, __shfl_xor_sync(kAll, top, d));
      if (p.bias || p.n_groups > 1) {
        float all = 0.f;
#pragma unroll
        for (int i = 0; i < kPer; ++i) all += exp2_fast((x[i] - top) * kLog2e);
#pragma unroll
        for (int d = 16; d > 0; d >>= 1) all += __shfl_xor_sync(kAll, all, d);
        scale = reciprocal_fast(all);
      }
    }
    float worst = 0.f;  // NaN or +inf where a score is: those tokens go the exact way
    bool clear = true, closed = false;
    if (p.bias || p.n_groups > 1) {
      float s[kPer], a = -inf, b = -inf, largest = 0.f;
#pragma unroll
      for (int i = 0; i < kPer; ++i) {
        s[i] = p.softmax ? exp2_fast((x[i] - top) * kLog2e) * scale : reciprocal_fast(1.f + exp2_fast(-x[i] * kLog2e));
        s[i] = x[i] == -inf ? -inf : s[i] + bias[i];
        worst = max_nan(worst, s[i]);
      }
      if (p.n_groups > 1) {
#pragma unroll
        for (int i = 0; i < kPer; ++i) {
          b = fmaxf(b, fminf(a, s[i]));
          a = fmaxf(a, s[i]);
          largest = fmaxf(largest, s[i] == -inf ? 0.f : fabsf(s[i]));
        }
        const bool plain = !p.bias && p.group_top == 1;  // the largest logits are the order of the ranks
        if (plain) {
          a = -inf;
#pragma unroll
          for (int i = 0; i < kPer; ++i) a = fmaxf(a, x[i]);
        }
        for (int d = width >> 1; d > 0; d >>= 1) {
          const float a2 = __shfl_xor_sync(kAll, a, d), b2 = __shfl_xor_sync(kAll, b, d);
          b = fmaxf(fmaxf(b, b2), fminf(a, a2));
          a = fmaxf(a, a2);
          largest = fmaxf(largest, __shfl_xor_sync(kAll, largest, d));
        }
        const float rank = p.group_top == 2 && b != -inf ? a + b : a;
        // twice the error of a sum of two scores, twice that for two sums, and the sum's own rounding
        const float near = (p.softmax ? 0x1p-14f * scale : 0x1p-18f) + 4.f * kKeyStep * largest + 0x1p-100f;
        int better = 0;
        for (int h = 0; h < p.n_groups; ++h) {
          const float r = __shfl_sync(kAll, rank, h << p.lanes_log2);
          better += r > rank || (r == rank && h < g);
        }
        closed = better >= p.top_groups;
        // the worst group that takes part against the best one that does not: their order among themselves is nobody's concern
        float worst_in = g < p.n_groups && !closed ? rank : inf, best_out = g < p.n_groups && closed ? rank : -inf;
#pragma unroll
        for (int d = 16; d > 0; d >>= 1) {
          worst_in = fminf(worst_in, __shfl_xor_sync(kAll, worst_in, d));
          best_out = fmaxf(best_out, __shfl_xor_sync(kAll, best_out, d));
        }
        const float gap = closed ? worst_in - rank : rank - best_out;
        if (g < p.n_groups && best_out != -inf && rank != -inf) {
          const float larger = closed ? worst_in : rank;
          clear = plain ? gap == 0.f || (gap > 0x1p-45f && (p.softmax ? larger - top > -600.f : larger < 15.f && larger > -700.f)) : gap > near;
        }
      }
#pragma unroll
      for (int i = 0; i < kPer; ++i) key[i] = __float_as_int(p.bias ? s[i] : x[i]);
    } else {
#pragma unroll
      for (int i = 0; i < kPer; ++i) key[i] = __float_as_int(x[i]);
    }
    if (!p.bias) {
#pragma unroll
      for (int i = 0; i < kPer; ++i) worst = max_nan(worst, x[i]);
    }
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
      key[i] = (ordered(key[i]) & ~kPlace) | (kPlace - i);
      if (closed) key[i] = (int)0x80000000;
    }
    sort_down(key);
    // k rounds and one more: the largest key of the warp, equal ones by their lane (the experts of a lane, and the lanes, are in
    // order); its lane moves up.  Lane q keeps choice q: its key, and the lane that had it.
    int won = (int)0x80000000, from = 0, n_won = 0;
    auto draw = [&]() -> bool {
      const int v = __reduce_max_sync(kAll, key[0] & ~kPlace);
      if (v < kNoKey) return false;
      const int owner = __ffs(__ballot_sync(kAll, (key[0] & ~kPlace) == v)) - 1;
      const int whole = __shfl_sync(kAll, key[0], owner);
      won = lane == n_won ? whole : won;
      from = lane == n_won ? owner : from;
      const bool up = lane == owner;
#pragma unroll
      for (int i = 0; i + 1 < kPer; ++i) key[i] = up ? key[i + 1] : key[i];
      key[kPer - 1] = up ? (int)0x80000000 : key[kPer - 1];
      ++n_won;
      return true;
    };
    while (n_won <= p.k && draw()) {
    }
    auto expert = [&] { return (from >> p.lanes_log2) * p.group_size + (from & (width - 1)) * p.per + kPlace - (won & kPlace); };
    // is v certainly in front of v2 (keys without their places), or an equal logit in the right order?
    auto apart = [&](int v, int v2) -> bool {
      const float c = __int_as_float(ordered(v)), c2 = __int_as_float(ordered(v2));
      if (p.bias) return c - c2 > (p.softmax ? 0x1p-16f * scale : 0x1p-20f) + kKeyStep * (fabsf(c) + fabsf(c2)) + 0x1p-100f;
      // equal keys are equal logits in bf16 (the places have bits of their own), in their right order, and the next smaller bf16 number
      // scores less here
      return (kBf16 || v != v2) && (fmaxf(fabsf(c), fabsf(c2)) >= 0x1p-20f || c - c2 > 0x1p-36f) && (p.softmax ? c - top > -600.f : c < 15.f && c > -700.f);
    };
    bool sure = true;
    {
      const int next = __shfl_down_sync(kAll, won, 1);
      if (lane < p.k && lane + 1 < n_won) sure = apart(won & ~kPlace, next & ~kPlace);
    }
    int mine = lane < p.k && lane < n_won ? expert() : -1;
    bool exact = !__all_sync(kAll, clear && worst < inf);
    if (kBf16 && !exact && !p.bias && !__all_sync(kAll, sure)) {
      // equal logits elsewhere (zeros of a padded token, masks): the order of those up to the k-th is right, and if the next one equals
      // the k-th, the largest logit below has to score less
      const int v = won & ~kPlace, next = __shfl_down_sync(kAll, v, 1), last = __shfl_sync(kAll, v, p.k - 1);
      int below = (int)0x80000000;
#pragma unroll
      for (int i = 0; i < kPer; ++i) {
        const int o = ordered(__float_as_int(x[i])) & ~kPlace;
        below = o < last ? max(below, o) : below;
      }
      below = __reduce_max_sync(kAll, below);
      if (lane < p.k && lane + 1 < n_won && v == next) sure = lane + 1 < p.k || below < kNoKey || apart(last, below);
    }
    if (!exact && !__all_sync(kAll, sure)) {
      // The order of a few is open: those, as far down as they may belong to the k, are compared in 64 bits, one per lane.
      const int last = __shfl_sync(kAll, won, p.k - 1) & ~kPlace;
      exact = p.softmax ? p.bias != nullptr || __int_as_float(ordered(last)) - top <= -600.f
                        : !p.bias && __int_as_float(ordered(__shfl_sync(kAll, won, 0) & ~kPlace)) >= 15.f;
      while (!exact && n_won > p.k && !apart(last, __shfl_sync(kAll, won, n_won - 1) & ~kPlace)) {
        exact = n_won == 32;
        if (exact || !draw()) break;
      }
      if (!exact) {
        double d = kNone;
        const int at = lane < n_won ? expert() : 0x7fffffff;
        if (lane < n_won) {
          d = (double)route_logit<kBf16>(p, token, at);
          if (!p.softmax) {
            d = 1.0 / (1.0 + exp(-d));
            if (p.bias) d += (double)p.bias[at];
          } else if (d - (double)top <= -600.0) {
            exact = true;
          }
        }
        int front = 0;
        for (int j = 0; j < n_won; ++j) {
          const double other = __shfl_sync(kAll, d, j);
          const int other_at = __shfl_sync(kAll, at, j);
          front += other > d || (other == d && other_at < at);
          exact |= p.softmax && lane < n_won && other != d && fabs(other - d) <= 0x1p-45;
        }
        mine = -1;
        for (int j = 0; j < n_won; ++j) {
          const int place = __shfl_sync(kAll, front, j), other_at = __shfl_sync(kAll, at, j);
          if (lane < p.k && place == lane) mine = other_at;
        }
        exact = __any_sync(kAll, exact);
      }
    }
    if (exact) mine = route_exact<kPer, kBf16>(p, token);
    const int q_mine = lane - turn * span;
    mine = __shfl_sync(kAll, mine, q_mine & 31);
    const bool here = q_mine >= 0 && q_mine < p.k;
    if (here) {
      id = mine;
      top_mine = (double)top;
    }
    if (p.softmax && !p.renorm) {  // the sum in 64 bits, to which the weights are held
      double all = 0.0;
#pragma unroll
      for (int i = 0; i < kPer; ++i) all += x[i] == -inf ? 0.0 : exp_31((double)x[i] - (double)top);
#pragma unroll
      for (int d = 16; d > 0; d >>= 1) all += __shfl_xor_sync(kAll, all, d);
      if (here) sum = all;
    }
  }
  // ---- weights ----
  const int turn = lane / span, q = lane - turn * span;
  const int64_t token = first + turn;
  const bool out = q < p.k && turn < turns && token < p.n;
  double w = 0.0;
  if (out && id >= 0) {
    const double x = (double)route_logit<kBf16>(p, token, id);
    w = p.softmax ? exp(x - top_mine) / sum : 1.0 / (1.0 + exp(-x));
  }
  if (p.renorm) {
    double all = w;
    for (int d = span >> 1; d > 0; d >>= 1) all += __shfl_xor_sync(kAll, all, d);
    w = all > 0.0 ? w / all : 0.0;
  }
  if (out) {
    p.ids[token * p.k + q] = id < 0 ? -1 : id;
    p.weights[token * p.k + q] = id == -2 ? __int_as_float(0x7fc00000) : (float)(w * (double)p.scale);
  }
}

// ------------------------------------------------------------------------------------------------------------
// rk_moe_group: a stable counting sort of the pairs by expert, by one cluster, without a workspace.
// Every warp owns a run of consecutive pairs and a count per expert in shared memory.  Scans over warps, over the cluster's
// blocks (through distributed shared memory) and over experts turn the counts into places; a second walk over the same run
// writes the list: lanes with the same expert find one another by votes on the bits of its number (match.any takes an SM
// 70 clocks).  What bounds it: short lists, the chain of launch, loads, scans and stores (384 pairs: 5.0 us); long ones, the
// votes of the cluster's SMs (262144 pairs: 18.6 us).
// ------------------------------------------------------------------------------------------------------------
constexpr int kGroupThreads = 1024, kGroupWarps = kGroupThreads / 32;
constexpr int kGroupAhead = 8;  // steps whose ids a warp loads together

__device__ __forceinline__ int ld_cluster_s32(uint32_t addr) {
  int v;
  asm volatile("ld.shared::cluster.s32 %0, [%1];" : "=r"(v) : "r"(addr) : "memory");
  return v;
}

// kBits: of an expert's number
template <int kBits>
__global__ void __launch_bounds__(kGroupThreads, 1) moe_group_kernel(const GroupParams p) {
  extern __shared__ int group_smem[];
  int* count = group_smem;                        // [warps][experts]
  int* total = count + kGroupWarps * p.n_experts; // [experts]: this block's pairs
  int* base = total + p.n_experts;                // [experts]: first place of this block's pairs
  __shared__ int warp_sum[kGroupWarps], sum_all;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, n_e = p.n_experts;
  const int n_blocks = gridDim.x, rank = blockIdx.x;  // one cluster
  const int64_t n = p.n * p.k;
  const int64_t run = ((n + (int64_t)n_blocks * kGroupThreads - 1) / ((int64_t)n_blocks * kGroupThreads)) * 32;
  const int64_t lo = ((int64_t)rank * kGroupWarps + warp) * run, hi = lo + run < n ? lo + run : n;
  int* mine = count + warp * n_e;
  const int64_t rest = n - (int64_t)rank * kGroupWarps * run;
  const int busy = rest <= 0 ? 0 : rest >= kGroupWarps * run ? kGroupWarps : (int)((rest + run - 1) / run);  // warps with pairs
  for (int i = threadIdx.x; i < busy * n_e; i += kGroupThreads) count[i] = 0;
  __syncthreads();
  auto expert_of = [&](int64_t i) -> int {
    if (i >= hi) return -1;
    const int e = p.ids[i];
    if ((unsigned)e >= (unsigned)n_e) return -1;
    if (p.keep != nullptr) {
      const uint32_t t = (uint32_t)i / (uint32_t)p.k;
      if (!((p.keep[t] >> ((uint32_t)i - t * (uint32_t)p.k)) & 1)) return -1;
    }
    return e;
  };
  int e[kGroupAhead];
  for (int64_t i = lo; i < hi; i += 32 * kGroupAhead) {
#pragma unroll
    for (int j = 0; j < kGroupAhead; ++j) e[j] = expert_of(i + 32 * j + lane);
#pragma unroll
    for (int j = 0; j < kGroupAhead; ++j)
      if (e[j] >= 0) atomicAdd(mine + e[j], 1);
  }
  __syncthreads();
  for (int x = threadIdx.x; x < n_e; x += kGroupThreads) {
    int v[kGroupWarps], sum = 0;
#pragma unroll
    for (int w = 0; w < kGroupWarps; ++w) v[w] = w < busy ? count[w * n_e + x] : 0;
#pragma unroll
    for (int w = 0; w < kGroupWarps; ++w) {
      if (w < busy) count[w * n_e + x] = sum;
      sum += v[w];
    }
    total[x] = sum;
  }
  __syncwarp();
  cluster_arrive();
  cluster_wait();
  {  // n_experts <= kGroupThreads: one expert per thread
    const int e = threadIdx.x;
    int sum = 0, before = 0;
    if (e < n_e) {
      for (int b = 0; b < n_blocks; ++b) {
        const int v = ld_cluster_s32(mapa_shared(smem_u32(total + e), b));
        if (b < rank) before += v;
        sum += v;
      }
    }
    int x = sum;
    for (int d = 1; d < 32; d <<= 1) {
      const int v = __shfl_up_sync(0xffffffffu, x, d);
      if (lane >= d) x += v;
    }
    if (lane == 31) warp_sum[warp] = x;
    __syncthreads();
    int first = x - sum;
    for (int w = 0; w < warp; ++w) first += warp_sum[w];
    if (e < n_e) {
      base[e] = first + before;
      if (rank == 0) p.row_off[e] = first;
    }
    if (e == kGroupThreads - 1) {
      sum_all = first + sum;
      if (rank == 0) p.row_off[n_e] = first + sum;
    }
  }
  __syncthreads();
  __syncwarp();
  cluster_arrive();  // no block leaves before the others have read its counts
  auto same_expert = [&](int e) -> unsigned {  // lanes with the same expert; whatever for those without
    unsigned same = __ballot_sync(kAll, e >= 0);
#pragma unroll
    for (int b = 0; b < kBits; ++b) {
      const unsigned not_mine = (unsigned)((int)((unsigned)e << (31 - b)) >> 31);
      same &= ~(__ballot_sync(kAll, (e >> b) & 1) ^ not_mine);
    }
    return same;
  };
  for (int64_t i = lo; i < hi; i += 32 * kGroupAhead) {
    if (run > 32 * kGroupAhead) {  // (a shorter run's are still there)
#pragma unroll
      for (int j = 0; j < kGroupAhead; ++j) e[j] = expert_of(i + 32 * j + lane);
    }
#pragma unroll
    for (int j = 0; j < kGroupAhead; ++j) {
      if (i + 32 * j >= hi) break;
      const unsigned same = same_expert(e[j]), below = same & ((1u << lane) - 1u);
      int at = 0;
      if (e[j] >= 0) at = mine[e[j]];
      __syncwarp();
      if (e[j] >= 0) {
        p.rows[base[e[j]] + at + __popc(below)] = (int32_t)(i + 32 * j + lane);
        if (below == 0u) mine[e[j]] = at + __popc(same);
      }
      __syncwarp();
    }
  }
  for (int64_t i = (int64_t)sum_all + (int64_t)rank * kGroupThreads + threadIdx.x; i < n; i += (int64_t)n_blocks * kGroupThreads) p.rows[i] = -1;
  __syncwarp();
  cluster_wait();
}

// Experts of a lane (`per`, up to 64: 1024 in 17 to 32 groups) are held in registers by loops that unroll, so each width is a kernel,
// and a lane with fewer pads them by -inf: 2, 8, 16, 32 or 64, whose costs differ by more than the padding between them.
// 32768 tokens without groups, sigmoid and bias, 8 chosen: 64 experts 21 us, 128, 160 and 256 34, 384 69, 512 73, 768 212, 1024 227
// (64 tokens: 3.2, 3.9, 3.9, 4.1, 5.6, 5.5, 7.4, 8.6).  Up to 8 fit 14 blocks on an SM; 16 take 152 registers and more take 255, the
// 64-wide one with some of its values in local memory.  16-byte loads need all lanes full (256, 512 and 1024).
template <bool kBf16>
cudaError_t route_dispatch(const RouteParams& p, int per, cudaStream_t stream) {
  const int64_t tokens = kRouteWarps * p.turns;  // of a thread block
  const unsigned grid = (unsigned)((p.n + tokens - 1) / tokens);
  if (per <= 2)
    moe_route_kernel<2, kBf16><<<grid, 32 * kRouteWarps, 0, stream>>>(p);
  else if (per <= 8)
    moe_route_kernel<8, kBf16><<<grid, 32 * kRouteWarps, 0, stream>>>(p);
  else if (per <= 16)
    moe_route_kernel<16, kBf16><<<grid, 32 * kRouteWarps, 0, stream>>>(p);
  else if (per <= 32)
    moe_route_kernel<32, kBf16><<<grid, 32 * kRouteWarps, 0, stream>>>(p);
  else
    moe_route_kernel<64, kBf16><<<grid, 32 * kRouteWarps, 0, stream>>>(p);
  return cudaGetLastError();
}

}  // namespace

namespace {
typedef void (*GroupKernel)(const GroupParams);
const GroupKernel kGroupKernels[10] = {moe_group_kernel<1>, moe_group_kernel<2>, moe_group_kernel<3>, moe_group_kernel<4>, moe_group_kernel<5>,
                                       moe_group_kernel<6>, moe_group_kernel<7>, moe_group_kernel<8>, moe_group_kernel<9>, moe_group_kernel<10>};
GroupKernel group_kernel(int n_experts) {
  int bits = 1;
  while (1 << bits < n_experts) ++bits;
  return kGroupKernels[bits - 1];
}
cudaLaunchConfig_t group_config(int n_blocks, int n_experts, cudaLaunchAttribute* attr, cudaStream_t stream) {
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(n_blocks);
  cfg.blockDim = dim3(kGroupThreads);
  cfg.dynamicSmemBytes = (size_t)(kGroupWarps + 2) * n_experts * 4;
  cfg.stream = stream;
  attr->id = cudaLaunchAttributeClusterDimension;
  attr->val.clusterDim.x = n_blocks;
  attr->val.clusterDim.y = attr->val.clusterDim.z = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  return cfg;
}
}  // namespace

cudaError_t experts_setup(int32_t* group_blocks) {
  cudaError_t e = cudaSuccess;
  for (GroupKernel kernel : kGroupKernels) {
    if (e == cudaSuccess) e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (kGroupWarps + 2) * kMaxExperts * 4);
    if (e == cudaSuccess) e = cudaFuncSetAttribute(kernel, cudaFuncAttributeNonPortableClusterSizeAllowed, 1);
  }
  if (e != cudaSuccess) return e;
  // 16 blocks where the device has room for such a cluster
  cudaLaunchAttribute attr;
  const cudaLaunchConfig_t cfg = group_config(16, kMaxExperts, &attr, nullptr);
  int n = 0;
  *group_blocks = cudaOccupancyMaxActiveClusters(&n, kGroupKernels[9], &cfg) == cudaSuccess && n > 0 ? 16 : 8;
  cudaGetLastError();
  return cudaSuccess;
}

cudaError_t launch_moe_route(RouteParams p, int sm_count, cudaStream_t stream) {
  p.lanes_log2 = 5;
  while (p.lanes_log2 > 0 && (32 >> p.lanes_log2) < p.n_groups) --p.lanes_log2;  // 32 / lanes per group >= groups
  const int per = (p.group_size + (1 << p.lanes_log2) - 1) >> p.lanes_log2;
  // a warp takes several tokens (their weights are computed together) once every SM has 32 warps at work
  const int span = p.k <= 8 ? 8 : 16;
  const int64_t turns = p.n / (32 * (int64_t)sm_count);
  p.turns = turns < 1 ? 1 : turns > 32 / span ? 32 / span : (int32_t)turns;
  p.per = per;
  const int64_t in_16 = p.bf16 ? 8 : 4;
  p.whole = (per == 8 || per == 16 || per == 32) && (per << p.lanes_log2) == p.group_size && (p.n_groups << p.lanes_log2) == 32 &&
            (reinterpret_cast<uintptr_t>(p.logits) & 15u) == 0 && p.stride % in_16 == 0;
  return p.bf16 ? route_dispatch<true>(p, per, stream) : route_dispatch<false>(p, per, stream);
}

cudaError_t launch_moe_group(const GroupParams& p, int32_t group_blocks, cudaStream_t stream) {
  // Up to eight blocks, one step (32 pairs) of a warp costs more than the barriers of a cluster twice the size; sixteen pay from four
  // steps on (256 experts, in 1 / 2 / 4 / 8 / 16 blocks: 768 pairs 5.5 / 5.5 / 5.7 / 6.1 / 6.7 us, 6144 pairs
  // 8.8 / 7.2 / 6.8 / 6.3 / 7.0, 49152 pairs 40.6 / 22.9 / 14.5 / 9.4 / 8.2)
  const int64_t pairs = p.n * p.k;
  int blocks = 1;
  while (blocks < 8 && pairs > (int64_t)blocks * kGroupThreads) blocks *= 2;
  if (pairs > 4 * 8 * kGroupThreads) blocks = group_blocks;
  cudaLaunchAttribute attr;
  const cudaLaunchConfig_t cfg = group_config(blocks, p.n_experts, &attr, stream);
  return cudaLaunchKernelEx(&cfg, group_kernel(p.n_experts), p);
}

}  // namespace rk
