// Sampling a token from each row of logits: temperature, top-k, top-p, min-p, and one given random number per row.
//
// p_i = exp((l_i - max) / T), as whole numbers of 2^-42 (a token below 2^-42 of the largest weighs nothing).  Whole numbers
// add up to the same sum in any order, so that sums, cuts and the chosen token depend on the inputs alone, and their error
// (2^-42 per token) is far below the distance at which two neighbouring tokens' borders could be confused.  The
// exponential is taken in double: 256 x = i + r with i whole, 2^-i/256 from a table and a shift, 2^-r/256 by its Taylor
// series to degree 3 (|r| <= 1/2: 1.4e-13).  A token costs eleven double-precision instructions that way, which bounds the
// passes that need every token's weight; conversions from fp32 are done in integers, which takes infinities along.
//
// The three filters each keep a prefix of one order, falling logit and then rising index, so together they keep the tokens
// not below one (logit, index) pair, the cut.  A row belongs to a cluster of thread blocks, each with a run of consecutive tokens.
//   1. the largest logit (and whether there is a NaN)
//   2. up to 256 for top-k: the tokens that reach a logit which at least k tokens do (step 1 found one on its way) go to the
//      first block, which sorts them and needs nothing more.
//      Otherwise, where top-k or top-p is on: counts, and estimates of the weights, in bins of 1/64 octave in fp32, joined in
//      the first block, which picks the bins around the cuts; then exact sums of what is in front of them, while their tokens
//      (some hundred of 128 K) go to the first block's lists, which ranks them, finds the cuts and checks the estimate.
//      Where that fails or a list is too short (thousands of equal logits), the cut is searched for by exact counts and sums,
//      11 bits of (logit, index) at a time.
//   3. sums of what stays, by block and by warp; the block that holds u * total shares out the warp's run that holds it
// The row is read again by each step: it comes out of L2 after the first.
//
// 64 rows of 131072 fp32 logits (33.6 MB, 5.2 us to read once): 24 us without filters, 27 with top-k 50, 56 with top-p 0.9; one
// row of 32001 with all filters 10.  What bounds it: many rows, the instructions of the passes (44 per token where its weight is
// needed); a single row, the chain of cluster barriers and code that runs for the first time.
#include <cuda_bf16.h>

#include "rk_internal.h"

namespace rk {
namespace {

constexpr int kThreads = 512, kWarps = kThreads / 32;
constexpr int kBins = 2048, kBinsPer = kBins / kThreads;
constexpr int kList = 2048, kListPer = kList / kThreads;  // tokens of a cut's bins that are ranked in shared memory
constexpr int kQuick = 256;               // up to here the top k are found without bins
constexpr int kUnitLog2 = 42;             // weights are multiples of 2^-42
constexpr int kSteps = 256;               // i counts 256ths of an octave below the largest
constexpr int kEnd = kUnitLog2 * kSteps;  // from here on tokens weigh nothing
constexpr int kIndexBits = 20, kDigitBits = 11, kKeyBits = 32 + kIndexBits, kDigits = (kKeyBits + kDigitBits - 1) / kDigitBits;
typedef unsigned long long u64;

struct Found {           // what the first block of a row's cluster tells the others
  int bin_k;             // bin of the top-k cut, or -1
  int bin_lo, bin_hi;    // bins around the top-p cut
  int slow;              // a list overflowed, or the cut is outside the bins
  uint32_t count_k;      // tokens in front of bin_k
  u64 total;             // sum of all tokens
  u64 cut;
};

struct Shared {
  double table[kSteps];          // 2^(42 - j/256)
  u64 list[2][kList];            // (key, index) of the tokens in bin_k and in bin_lo .. bin_hi
  u64 mass[kThreads];            // weights of a short list
  uint32_t listed[2];
  uint32_t count[kBins], lo[kBins], hi[kBins];
  u64 slot64b[8];                // one word per block of the cluster
  u64 slot_all[8], slot_above[8];
  u64 slot_part[kWarps];
  uint32_t extra_lo[8 * kWarps], extra_hi[8 * kWarps];  // by warp of the cluster: weights of the listed tokens that stay
  u64 warp64[kWarps];
  uint32_t warp32[kWarps];
  float top[8], low[8];
  uint32_t first[8];
  Found found;
  int pick_bin;
  uint32_t pick_count;           // tokens in front of the picked bin
  u64 pick_mass;                 // and their sum
  u64 pick_own;                  // sum of the picked bin
};

// order of logits: larger key, larger logit; both zeros are one
__device__ __forceinline__ uint32_t key_of(float l) {
  const uint32_t b = __float_as_uint(l + 0.f);
  return b & 0x80000000u ? ~b : b | 0x80000000u;
}
__device__ __forceinline__ float logit_of(uint32_t key) { return __uint_as_float(key & 0x80000000u ? key & 0x7fffffffu : ~key); }
__device__ __forceinline__ u64 composite(float l, int i) { return ((u64)key_of(l) << kIndexBits) | (uint32_t)((1 << kIndexBits) - 1 - i); }

__device__ __forceinline__ u64 ld_cluster_u64(uint32_t addr) {
  u64 v;
  asm volatile("ld.shared::cluster.u64 %0, [%1];" : "=l"(v) : "r"(addr) : "memory");
  return v;
}
__device__ __forceinline__ uint32_t ld_cluster_u32(uint32_t addr) {
  uint32_t v;
  asm volatile("ld.shared::cluster.u32 %0, [%1];" : "=r"(v) : "r"(addr) : "memory");
  return v;
}
__device__ __forceinline__ void st_cluster_u64(uint32_t addr, u64 v) {
  asm volatile("st.shared::cluster.u64 [%0], %1;" ::"r"(addr), "l"(v) : "memory");
}
__device__ __forceinline__ uint32_t add_cluster_u32(uint32_t addr, uint32_t v) {
  uint32_t old;
  asm volatile("atom.shared::cluster.add.u32 %0, [%1], %2;" : "=r"(old) : "r"(addr), "r"(v) : "memory");
  return old;
}
// (the barrier is .aligned: it asks for all lanes of the warp at once, and the code in front may have parted them)
__device__ __forceinline__ void cluster_sync() {
  __syncwarp();
  cluster_arrive();
  cluster_wait();
}

// fp32 -> fp64 for finite numbers, in integers; below fp32's normal numbers it is off by up to 2^-126
__device__ __forceinline__ double widen(float f) {
  const uint32_t b = __float_as_uint(f);
  return __hiloint2double((((int)b >> 3) & (int)0x8fffffffu) + 0x38000000, (int)(b << 29));
}

struct Weights {
  double top, rate;     // the largest logit; 256 log2(e) / T
  const double* table;
  // 256ths of an octave below the largest
  __device__ __forceinline__ double depth(float l) const { return (top - widen(l)) * rate; }
  // the same as a whole number and a rest; any number comes out for logits beyond kEnd
  __device__ __forceinline__ int place(float l, double& rest) const {
    constexpr double kMagic = 6755399441055744.0;  // 1.5 * 2^52: the sum has the nearest whole number in its low word
    const double s = depth(l), t = s + kMagic;
    rest = s - (t - kMagic);
    return __double2loint(t);
  }
  // 2^(42 - (i + rest) / 256)
  __device__ __forceinline__ double scaled(int i, double r) const {
    constexpr double c1 = -0.69314718055994530942 / kSteps, c2 = c1 * c1 / 2.0, c3 = c1 * c1 * c1 / 6.0;
    const double t = table[i & (kSteps - 1)], v = fma(t, r * fma(fma(c3, r, c2), r, c1), t);
    return __hiloint2double(__double2hiint(v) - ((i & ~(kSteps - 1)) << 12), __double2loint(v));
  }
  // what a token weighs, as a whole number in the low 52 bits
  static constexpr double kWhole = 0x1p52;
  static __device__ __forceinline__ u64 units(double scaled_) { return (u64)(__double_as_longlong(scaled_ + kWhole) & ((1ll << 52) - 1)); }
  __device__ __forceinline__ u64 units(float l) const {
    double r;
    const int i = place(l, r);
    return units(scaled(i, r));
  }
};
// The lowest logit for which `in` holds; it holds for `top` and everything down from there to the one looked for.  The lanes
// of a warp (all of them) first test 32 numbers around the guess, four apart, then 32 places of what is left of the order
// of fp32 numbers: two rounds where the guess is good, eight at most.
template <class F>
__device__ __forceinline__ float lowest(float top, float guess, F in) {
  const uint32_t lane = threadIdx.x & 31;
  uint32_t out = key_of(-3.402823466e38f) - 1u, hit = key_of(top);  // `in` does not hold (or nothing is there) / holds
  const uint32_t mid = min(max(key_of(guess), out + 65u), hit);  // (a guess that is no number is as good as any)
  bool near = hit - out > 256u;
  while (hit - out > 1u) {
    const uint32_t at = near ? min(mid - 64u + 4u * lane, hit) : out + 1u + (uint32_t)(((u64)(hit - out - 1u) * lane) >> 5);  // ascending
    near = false;
    const unsigned holds = __ballot_sync(0xffffffffu, in(logit_of(at)));
    const int first = holds != 0u ? __ffs(holds) - 1 : 32;
    const uint32_t at_first = __shfl_sync(0xffffffffu, at, first & 31), at_before = __shfl_sync(0xffffffffu, at, (first + 31) & 31);
    if (first < 32) hit = at_first;
    if (first > 0) out = at_before;
  }
  return logit_of(hit);
}
// Where tokens gather around a cut is first estimated in fp32: bins of 1/64 octave (or any other size: all that is asked of
// them is to follow the order of the logits), the last one without an end.
struct Coarse {
  float top, scale;   // scale = 64 log2(e) / T
  float one;          // units of a bin's largest weight, so that a bin's 32-bit sum holds a whole row
  __device__ __forceinline__ int bin(float l) const {
    return (int)(__float_as_uint(fminf((top - l) * scale, (float)(kBins - 1)) + 8388608.f) & 0x7fffffu);
  }
  // and the weight next to the bin's middle, in units of 1 / one: a linear step is off by 1.5e-5
  __device__ __forceinline__ int bin(float l, uint32_t& weight) const {
    const float q = fminf((top - l) * scale, (float)(kBins - 1)), t = q + 8388608.f;
    weight = __float_as_uint(fmaf(one * -0.01083042f, q - (t - 8388608.f), one) + 8388608.f) & 0x7fffffu;
    return (int)(__float_as_uint(t) & 0x7fffffu);
  }
};
// bins of i: 64 to an octave for the first 16 octaves, then 32
constexpr int kFine = 16 * kSteps;
__device__ __forceinline__ int bin_of(int i) { return i < kFine ? i >> 2 : (kFine >> 2) + ((i - kFine) >> 3); }
static_assert((kFine >> 2) + ((kEnd - kFine) >> 3) <= kBins, "bins");

__device__ __forceinline__ float max_nan(float a, float b) {
  float r;
  asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b));
  return r;
}

// A thread block's run of a row.  A warp has consecutive 16-byte units of it, one per lane and step; units that reach over
// an end of the row are put together from single loads.
template <bool kBf16>
struct Run {
  static constexpr int kUnit = kBf16 ? 8 : 4;
  const uint8_t* base;  // 16-byte aligned, at or in front of the row
  int head, vocab;      // elements between base and the row
  int first, last;      // units of this warp
  int per, warps;       // units of a warp; warps of the cluster that have some

  __device__ __forceinline__ Run(const void* logits, int64_t at, int vocab_, int block, int n_blocks, int warp) : vocab(vocab_) {
    const uintptr_t a = reinterpret_cast<uintptr_t>(logits) + at * (kBf16 ? 2 : 4);
    base = reinterpret_cast<const uint8_t*>(a & ~(uintptr_t)15);
    head = (int)(a & 15) / (kBf16 ? 2 : 4);
    const int n = (head + vocab + kUnit - 1) / kUnit;
    per = (n + n_blocks * kWarps * 32 - 1) / (n_blocks * kWarps * 32) * 32;
    warps = (n + per - 1) / per;
    first = min((block * kWarps + warp) * per, n);
    last = min(first + per, n);
  }
  __device__ __forceinline__ int index(int unit) const { return unit * kUnit - head; }
  __device__ __forceinline__ bool whole(int unit) const { return index(unit) >= 0 && index(unit) + kUnit <= vocab; }
  __device__ __forceinline__ uint4 load(int unit) const {
    const uint8_t* p = base + (int64_t)unit * 16;
    if (whole(unit)) return __ldg(reinterpret_cast<const uint4*>(p));
    uint32_t w[4];  // -inf beyond the row
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      auto inside = [&](int e) { return (unsigned)(index(unit) + e) < (unsigned)vocab; };
      if constexpr (kBf16) {
        const uint16_t* h = reinterpret_cast<const uint16_t*>(p) + 2 * j;
        w[j] = (inside(2 * j) ? (uint32_t)h[0] : 0xff80u) | (inside(2 * j + 1) ? (uint32_t)h[1] : 0xff80u) << 16;
      } else {
        w[j] = inside(j) ? *(reinterpret_cast<const uint32_t*>(p) + j) : 0xff800000u;
      }
    }
    return make_uint4(w[0], w[1], w[2], w[3]);
  }
  static __device__ __forceinline__ float value(const uint4& v, int e) {
    const uint32_t w[4] = {v.x, v.y, v.z, v.w};
    if constexpr (kBf16) return __uint_as_float(e & 1 ? w[e >> 1] & 0xffff0000u : w[e >> 1] << 16);
    return __uint_as_float(w[e]);
  }
  // f(logits, index) for four neighbouring tokens at a time, ascending within a lane, where one has a logit of at least `least`
  // (more than -inf, which stands beyond the row's ends); kAhead units are loaded together
  template <int kAhead, class F>
  __device__ __forceinline__ void each4(float least, F f) const {
    const int lane = threadIdx.x & 31;
    for (int u0 = first + lane; u0 < last; u0 += 32 * kAhead) {
      uint4 v[kAhead];
#pragma unroll
      for (int j = 0; j < kAhead; ++j)
        if (u0 + 32 * j < last) v[j] = load(u0 + 32 * j);
#pragma unroll
      for (int j = 0; j < kAhead; ++j) {
        if (u0 + 32 * j >= last) break;
        four(v[j], u0 + 32 * j, least, f);
      }
    }
  }
  template <class F>
  __device__ __forceinline__ void four(const uint4& v, int unit, float least, F f) const {
#pragma unroll
    for (int q = 0; q < kUnit; q += 4) {
      const float l[4] = {value(v, q), value(v, q + 1), value(v, q + 2), value(v, q + 3)};
      if (fmaxf(fmaxf(l[0], l[1]), fmaxf(l[2], l[3])) >= least) f(l, index(unit) + q);
    }
  }
  // the largest logit, NaN if there is one (in this lane)
  __device__ __forceinline__ float top() const {
    constexpr int kAhead = 4;
    const int lane = threadIdx.x & 31;
    const float none = -__int_as_float(0x7f800000);
    float m = none;
    for (int u0 = first + lane; u0 < last; u0 += 32 * kAhead) {
      uint4 v[kAhead];
#pragma unroll
      for (int j = 0; j < kAhead; ++j) v[j] = u0 + 32 * j < last ? load(u0 + 32 * j) : load(u0);
#pragma unroll
      for (int j = 0; j < kAhead; ++j) {
        if constexpr (kBf16) {
          uint32_t a, b;
          asm("max.NaN.bf16x2 %0, %1, %2;" : "=r"(a) : "r"(v[j].x), "r"(v[j].y));
          asm("max.NaN.bf16x2 %0, %1, %2;" : "=r"(b) : "r"(v[j].z), "r"(v[j].w));
          asm("max.NaN.bf16x2 %0, %1, %2;" : "=r"(a) : "r"(a), "r"(b));
          m = max_nan(m, max_nan(__uint_as_float(a << 16), __uint_as_float(a & 0xffff0000u)));
        } else {
          m = max_nan(max_nan(m, max_nan(__uint_as_float(v[j].x), __uint_as_float(v[j].y))), max_nan(__uint_as_float(v[j].z), __uint_as_float(v[j].w)));
        }
      }
    }
    return m;
  }
};

// Sorts list[0 .. n) descending; n <= kList.  All threads of the block; ends with a barrier.
__device__ __noinline__ void sort_list(u64* list, int n) {
  int size = 2;
  while (size < n) size *= 2;
  for (int i = n + (int)threadIdx.x; i < size; i += kThreads) list[i] = 0ull;
  __syncthreads();
  for (int k = 2; k <= size; k *= 2) {
    for (int j = k >> 1; j > 0; j >>= 1) {
      for (int t = threadIdx.x; t < size / 2; t += kThreads) {
        const int a = 2 * t - (t & (j - 1)), b = a + j;
        const u64 x = list[a], y = list[b];
        if ((x < y) == ((a & k) == 0)) {
          list[a] = y;
          list[b] = x;
        }
      }
      __syncthreads();
    }
  }
}

template <bool kBf16>
__global__ void __launch_bounds__(kThreads, 2) sample_kernel(const SampleParams p) {
  extern __shared__ __align__(16) uint8_t sample_smem[];
  Shared& sh = *reinterpret_cast<Shared*>(sample_smem);
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const int n_blocks = p.blocks, rank = (int)cluster_ctarank();
  const int64_t row = blockIdx.x / n_blocks;
  const unsigned all = 0xffffffffu;
  const float inf = __int_as_float(0x7f800000);
  const Run<kBf16> run(p.logits, row * p.stride, p.vocab, rank, n_blocks, warp);
  auto peer = [&](const void* at, int r) -> uint32_t { return mapa_shared(smem_u32(at), r); };
  auto clear_bins = [&] {
    for (int b = tid; b < kBins; b += kThreads) sh.count[b] = sh.lo[b] = sh.hi[b] = 0u;
  };

  const float temp = p.temperature ? p.temperature[row] : 1.f;
  const int top_k = p.top_k ? p.top_k[row] : 0;
  const float top_p = p.top_p ? p.top_p[row] : 1.f, min_p = p.min_p ? p.min_p[row] : 0.f;
  if (tid < 2) sh.listed[tid] = 0u;
  if (tid < 8 * kWarps) sh.extra_lo[tid] = sh.extra_hi[tid] = 0u;
  for (int j = tid; j < kSteps; j += kThreads) sh.table[j] = exp2((double)kUnitLog2 - (double)j / kSteps);
  clear_bins();

  // ---- 1. the largest logit, and a logit that at least top_k tokens reach: the smallest of the largest logits of that many
  // groups of threads that have tokens ----
  float top = run.top(), reached = top;
  int group_log2 = 9;  // of threads; the last warp's lanes may be without tokens
  static_assert(kThreads == 1 << 9, "threads");
  while (group_log2 > 0 && (group_log2 >= 5 ? run.warps >> (group_log2 - 5) : (run.warps - 1) << (5 - group_log2)) < top_k) --group_log2;
  const int group = 1 << group_log2;
#pragma unroll
  for (int d = 1; d < 32; d <<= 1) {
    top = max_nan(top, __shfl_xor_sync(all, top, d));
    const float o = __shfl_xor_sync(all, reached, d);
    if (d < group) reached = fmaxf(reached, o);
  }
  int groups = __popc(__ballot_sync(all, reached > -inf)) >> min(group_log2, 5);
  if (group < 32) {
    reached = reached > -inf ? reached : inf;
#pragma unroll
    for (int d = 16; d > 0; d >>= 1) reached = fminf(reached, __shfl_xor_sync(all, reached, d));
  }
  if (lane == 0) {
    sh.warp32[warp] = __float_as_uint(top);
    sh.warp64[warp] = ((u64)groups << 32) | __float_as_uint(reached);
  }
  __syncthreads();
  if (tid == 0) {
    float best = -inf;  // of several warps that are a group
    reached = inf;
    groups = 0;
    for (int w = 0; w < kWarps; ++w) {
      const float o = __uint_as_float((uint32_t)sh.warp64[w]);
      top = max_nan(top, __uint_as_float(sh.warp32[w]));
      best = group <= 32 ? o : fmaxf(best, o);
      if ((((w + 1) * 32) & (group - 1)) != 0) continue;
      if (best > -inf) {
        reached = fminf(reached, best);
        groups += group <= 32 ? (int)(sh.warp64[w] >> 32) : 1;
      }
      best = -inf;
    }
    sh.top[rank] = top;
    sh.low[rank] = reached;
    sh.first[rank] = (uint32_t)groups;
  }
  cluster_sync();
  {  // a lane per block
    const bool there = lane < n_blocks;
    const int r = there ? lane : 0;
    top = there ? __uint_as_float(ld_cluster_u32(peer(&sh.top[r], r))) : -inf;
    reached = there ? __uint_as_float(ld_cluster_u32(peer(&sh.low[r], r))) : inf;
    groups = there ? (int)ld_cluster_u32(peer(&sh.first[r], r)) : 0;
#pragma unroll
    for (int d = 4; d > 0; d >>= 1) {
      top = max_nan(top, __shfl_xor_sync(all, top, d));
      reached = fminf(reached, __shfl_xor_sync(all, reached, d));
      groups += __shfl_xor_sync(all, groups, d);
    }
    top = __shfl_sync(all, top, 0);
    reached = __shfl_sync(all, reached, 0);
    groups = __shfl_sync(all, groups, 0);
  }
  if (groups < top_k) reached = -inf;
  const bool dead = !(top > -inf);
  // the first token only (at temperatures below 2^-100 two numbers that differ at all are worlds apart)
  const bool one = !(temp >= 0x1p-100f) || top_p <= 0.f || min_p > 1.f || top_k == 1;
  if (dead || one) {
    uint32_t at = 0xffffffffu;
    if (!dead)
      run.template each4<4>(top, [&](const float(&l)[4], int i) { at = min(at, (uint32_t)(i + (l[0] == top ? 0 : l[1] == top ? 1 : l[2] == top ? 2 : 3))); });
    at = __reduce_min_sync(all, at);
    cluster_sync();  // (the slots have been read)
    if (lane == 0) sh.warp32[warp] = at;
    __syncthreads();
    if (tid == 0) {
      for (int w = 1; w < kWarps; ++w) at = min(at, sh.warp32[w]);
      sh.first[rank] = at;
    }
    cluster_sync();
    if (rank == 0 && tid == 0) {
      for (int r = 1; r < n_blocks; ++r) at = min(at, ld_cluster_u32(peer(&sh.first[r], r)));
      p.tokens[row] = dead ? -1 : (int)at;
      if (p.probs) p.probs[row] = dead ? __int_as_float(0x7fc00000) : 1.f;
    }
    cluster_sync();  // no block leaves while the first one reads
    return;
  }
  Weights w;
  w.top = widen(top);
  w.rate = (double)kSteps * 1.44269504088896340736 / (double)temp;
  w.table = sh.table;

  u64 cut = 0;  // tokens whose composite is at least this stay
  const bool by_mass = top_p < 1.f, by_count = top_k > 1 && top_k < p.vocab;
  // tokens from here on up weigh something (next to +inf nothing else does), and reach min_p
  const float floor_all = top == inf ? top : lowest(top, (float)((double)top - ((double)kEnd - 0.5) / w.rate), [&](float l) {
    double rest;
    return w.depth(l) < (double)kEnd + 1.0 && w.place(l, rest) < kEnd;
  });
  float floor_min = floor_all;
  if (min_p > 0.f && top < inf) {  // (NaN: off)
    const double most = -(double)kSteps * log2((double)min_p);
    floor_min = fmaxf(floor_all, lowest(top, (float)((double)top - most / w.rate), [&](float l) { return w.depth(l) <= most; }));
  }
  const float u = p.u[row];
  auto place_of = [&](u64 total) -> u64 {  // u times a sum of weights, below the sum
    const u64 want = u > 0.f ? (u64)((double)u * (double)total) : 0ull;
    return want < total ? want : total - 1;
  };

  // ---- 2. the cut ----
  // puts a token on one of the first block's lists
  auto keep = [&](int list, float l, int at) {
    const uint32_t slot = add_cluster_u32(peer(&sh.listed[list], 0), 1u);
    if (slot < kList) st_cluster_u64(peer(&sh.list[list][slot], 0), composite(l, at));
  };
  auto mass_of = [&](u64 c) -> u64 { return w.units(logit_of((uint32_t)(c >> kIndexBits))); };
  // Exclusive sums over the block's threads, added to cb and mb.
  auto scan_bins = [&](uint32_t csum, u64 msum, uint32_t& cb, u64& mb) {
    uint32_t cx = csum;
    u64 mx = msum;
#pragma unroll
    for (int d = 1; d < 32; d <<= 1) {
      const uint32_t cv = __shfl_up_sync(all, cx, d);
      const u64 mv = __shfl_up_sync(all, mx, d);
      if (lane >= d) {
        cx += cv;
        mx += mv;
      }
    }
    __syncthreads();
    if (lane == 31) {
      sh.warp32[warp] = cx;
      sh.warp64[warp] = mx;
    }
    __syncthreads();
    cb += cx - csum;
    mb += mx - msum;
    for (int v = 0; v < warp; ++v) {
      cb += sh.warp32[v];
      mb += sh.warp64[v];
    }
  };

  if (by_count && top_k <= kQuick) {
    // The tokens that reach `reached` (some hundred) hold the top k: the first block sorts them and goes through with it.
    const float from = fmaxf(reached, floor_all);
    run.template each4<4>(from, [&](const float(&l)[4], int at) {
#pragma unroll
      for (int e = 0; e < 4; ++e)
        if (l[e] >= from) keep(0, l[e], at + e);
    });
    cluster_sync();
    const int n = (int)min(ld_cluster_u32(peer(&sh.listed[0], 0)), (uint32_t)kList + 1u);
    if (n <= kList) {
      __syncwarp();
      cluster_arrive();
      if (rank == 0) {
        u64* sorted = sh.list[0];
        if (n <= kThreads) {
          const u64 mine = tid < n ? sorted[tid] : 0ull;
          int front = 0;
#pragma unroll 8
          for (int j = 0; j < n; ++j) front += sh.list[0][j] > mine;
          sorted = sh.list[1];
          if (tid < n) sorted[front] = mine;
          __syncthreads();
        } else {
          sort_list(sorted, n);
        }
        const int k = min(top_k, n);
        const u64 mine = tid < k ? sorted[tid] : 0ull, own = tid < k ? mass_of(mine) : 0ull;
        u64 front = 0;
        uint32_t unused = 0;
        scan_bins(0u, own, unused, front);
        if (tid == k - 1) sh.pick_mass = front + own;
        __syncthreads();
        const double most = (double)top_p * (double)sh.pick_mass;
        const bool stays = tid < k && (tid == 0 || ((!(top_p < 1.f) || (double)front < most) && logit_of((uint32_t)(mine >> kIndexBits)) >= floor_min));
        const int stay = __syncthreads_count(stays);  // the first ones
        const uint32_t at = (1u << kIndexBits) - 1u - (uint32_t)(mine & ((1u << kIndexBits) - 1u));
        if (tid == stay - 1) sh.pick_own = front + own;
        sh.mass[tid] = own;
        sh.count[tid] = at;
        __syncthreads();
        const u64 total = sh.pick_own, want = place_of(total);
        if (stays) {
          u64 upto = 0;
#pragma unroll 8
          for (int j = 0; j < stay; ++j) upto += sh.count[j] <= at ? sh.mass[j] : 0ull;
          if (upto > want && upto - own <= want) {
            p.tokens[row] = (int)at;
            double rest;
            const int i = w.place(logit_of((uint32_t)(mine >> kIndexBits)), rest);
            if (p.probs) p.probs[row] = (float)(w.scaled(i, rest) / (double)total);
          }
        }
      }
      __syncwarp();
      cluster_wait();
      return;
    }
    // Too many (equal logits, or falling ones): the bins sort it out.  They are as they were cleared in the beginning: others may
    // add to the first block's from here on, so that it must not clear them now.
    cluster_sync();  // everyone has seen the number
    if (rank == 0 && tid == 0) sh.listed[0] = 0u;  // (two barriers of the cluster before the next token comes)
  }
  bool summed = false;  // the sums of what stays are there already: sh.slot_part, and the first block's extra_*
  if (by_count || by_mass) {
    Coarse bins;
    float p_high = __int_as_float(0x7fc00000);
    bins.top = top;
    bins.scale = fminf((float)(w.rate * (64.0 / kSteps)), 1e30f);
    const int one_log2 = min(21, __clz(p.vocab) - 2);  // x the tokens of a row: below 2^31
    bins.one = (float)(1 << one_log2);
    run.template each4<2>(floor_all, [&](const float(&l)[4], int) {
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        uint32_t weight;
        const int b = bins.bin(l[e], weight);
        if (by_count && l[e] >= floor_all) atomicAdd(&sh.count[b], 1u);
        if (by_mass && l[e] >= floor_all) atomicAdd(&sh.lo[b], weight);
      }
    });
    __syncthreads();
    if (rank != 0) {
      for (int b = tid; b < kBins; b += kThreads) {
        if (by_count && sh.count[b] != 0u) add_cluster_u32(peer(&sh.count[b], 0), sh.count[b]);
        if (by_mass && sh.lo[b] != 0u) add_cluster_u32(peer(&sh.lo[b], 0), sh.lo[b]);
      }
    }
    cluster_sync();
    if (rank == 0) {
      uint32_t c[kBinsPer], n[kBinsPer], csum = 0, cb0 = 0;  // tokens (exact, for top-k), and their estimated weight below
      u64 m[kBinsPer], msum = 0, mb0 = 0;
#pragma unroll
      for (int j = 0; j < kBinsPer; ++j) {
        const int b = tid * kBinsPer + j;
        n[j] = sh.lo[b];
        csum += c[j] = by_count ? sh.count[b] : n[j] >> one_log2;
        msum += m[j] = (u64)((double)n[j] * (double)exp2f(30.f - (float)b * (1.f / 64.f)));
      }
      scan_bins(csum, msum, cb0, mb0);
      if (tid == 0) {
        sh.found.bin_k = sh.found.bin_lo = sh.found.bin_hi = -1;
        sh.found.slow = 0;
        sh.found.cut = 0;
      }
      if (tid == kThreads - 1) sh.pick_mass = mb0 + msum;
      __syncthreads();
      uint32_t cb = cb0;
      u64 mb = mb0;
#pragma unroll
      for (int j = 0; j < kBinsPer; ++j) {
        if (by_count && cb < (uint32_t)top_k && (uint32_t)top_k <= cb + c[j]) {
          sh.found.bin_k = tid * kBinsPer + j;
          sh.found.count_k = cb;
          sh.pick_mass = mb + (u64)((double)m[j] * (double)((uint32_t)top_k - cb) / (double)c[j]);
        }
        cb += c[j];
        mb += m[j];
      }
      __syncthreads();
      if (by_mass) {
        // the bin that the estimate points to, and its neighbours as far as the estimate may be off (a weight is rounded to
        // half a unit of 1 / one, in either direction), up to kAround tokens to either side
        constexpr uint32_t kAround = 96;
        const int last = sh.found.bin_k >= 0 ? sh.found.bin_k : kBins - 1;
        const double want = (double)top_p * (double)sh.pick_mass;
        __syncthreads();  // (pick_mass is written anew)
        cb = cb0;
        mb = mb0;
#pragma unroll
        for (int j = 0; j < kBinsPer; ++j) {
          if (m[j] != 0ull && (double)mb < want && !((double)(mb + m[j]) < want)) {
            sh.pick_bin = tid * kBinsPer + j;
            sh.pick_count = cb;
            sh.pick_own = cb + c[j];
            sh.found.bin_lo = tid * kBinsPer + j;
            sh.pick_mass = mb;
            sh.found.total = mb + m[j];
          }
          cb += c[j];
          mb += m[j];
        }
        __syncthreads();
        if (sh.found.bin_lo >= 0) {
          const int center = min(sh.pick_bin, last);
          const uint32_t front = sh.pick_count, behind = (uint32_t)sh.pick_own;
          const u64 off = (u64)(want / (double)bins.one) + 1ull, mass_front = sh.pick_mass, mass_behind = sh.found.total;
          __syncthreads();
          if (tid == 0) {
            sh.found.bin_lo = center;
            sh.found.bin_hi = center;
          }
          __syncthreads();
          cb = cb0;
          mb = mb0;
#pragma unroll
          for (int j = 0; j < kBinsPer; ++j) {
            const int b = tid * kBinsPer + j;
            const bool near = b < center ? mass_front - (mb + m[j]) <= off : mb - mass_behind <= off;
            if (near && b < center && front - cb <= kAround) atomicMin(&sh.found.bin_lo, b);
            cb += c[j];
            mb += m[j];
            if (near && b > center && b <= last && cb - behind <= kAround) atomicMax(&sh.found.bin_hi, b);
          }
        } else if (tid == 0) {
          sh.found.slow = 1;  // the estimate went wrong (weights beyond the bins)
        }
      }
    }
    cluster_sync();
    const int bin_k = (int)ld_cluster_u32(peer(&sh.found.bin_k, 0));
    const int bin_lo = (int)ld_cluster_u32(peer(&sh.found.bin_lo, 0)), bin_hi = (int)ld_cluster_u32(peer(&sh.found.bin_hi, 0));
    {
      // the tokens of those bins go to the lists; with top-p, the exact sums of what is in front of them and of everything
      // (with top-k, of what is in front of its bin).  From here on the bins are ranges of logits.
      auto edge = [&](int b) {  // the lowest logit of bin b
        return lowest(top, top - ((float)b + 0.5f) / bins.scale, [&](float l) { return bins.bin(l) <= b; });
      };
      const float none = __int_as_float(0x7fc00000);  // no logit is at least that
      const int best = bins.bin(top);
      const float k_low = bin_k >= 0 ? fmaxf(edge(bin_k), floor_all) : floor_all, k_high = bin_k > best ? edge(bin_k - 1) : none;
      if (by_mass) {
        const float p_low = fmaxf(edge(bin_hi), k_low);
        if (bin_lo > best) p_high = edge(bin_lo - 1);
        const float all_low = bin_k >= 0 ? k_high : floor_all;
        double above = 0.0, everything = 0.0;
        run.template each4<2>(k_low, [&](const float(&l)[4], int at) {
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            double rest;
            const int i = w.place(l[e], rest);
            const double u = (w.scaled(i, rest) + w.kWhole) - w.kWhole;
            if (l[e] >= all_low) everything += u;
            if (l[e] >= p_high) above += u;
          }
          const float high = fmaxf(fmaxf(l[0], l[1]), fmaxf(l[2], l[3])), low = fminf(fminf(l[0], l[1]), fminf(l[2], l[3]));
          if (high >= p_low && !(low >= p_high)) {
#pragma unroll
            for (int e = 0; e < 4; ++e)
              if (l[e] >= p_low && !(l[e] >= p_high)) keep(1, l[e], at + e);
          }
          if (bin_k >= 0) {
#pragma unroll
            for (int e = 0; e < 4; ++e)
              if (l[e] >= k_low && !(l[e] >= k_high)) keep(0, l[e], at + e);
          }
        });
        u64 s0 = (u64)everything, s1 = (u64)above;
#pragma unroll
        for (int d = 16; d > 0; d >>= 1) {
          s0 += __shfl_xor_sync(all, s0, d);
          s1 += __shfl_xor_sync(all, s1, d);
        }
        if (lane == 0) {
          sh.warp64[warp] = s0;
          sh.slot_part[warp] = s1;
        }
        __syncthreads();
        if (tid == 0) {
          for (int v = 1; v < kWarps; ++v) {
            s0 += sh.warp64[v];
            s1 += sh.slot_part[v];
          }
          st_cluster_u64(peer(&sh.slot_all[rank], 0), s0);
          st_cluster_u64(peer(&sh.slot_above[rank], 0), s1);
        }
      } else {
        run.template each4<4>(k_low, [&](const float(&l)[4], int at) {
#pragma unroll
          for (int e = 0; e < 4; ++e)
            if (l[e] >= k_low && !(l[e] >= k_high)) keep(0, l[e], at + e);
        });
      }
    }
    cluster_sync();
    if (rank == 0) {
      const uint32_t n_k = bin_k >= 0 ? sh.listed[0] : 0u, n_p = by_mass ? sh.listed[1] : 0u;
      u64 total = 0, above = 0;
      if (by_mass) {
        for (int r = 0; r < n_blocks; ++r) {
          total += sh.slot_all[r];
          above += sh.slot_above[r];
        }
      }
      __syncthreads();
      if (tid == 0) {
        sh.found.total = total;  // (with top-k: made whole by the search by digits, where that is needed)
        if (n_k > kList || n_p > kList) sh.found.slow = 1;
      }
      __syncthreads();
      if (sh.found.slow == 0) {
        // The last token of list[0 .. n) in the order with fewer than want_count in front of it, or (by sum) with less than
        // want_mass; base_*: in front of the list.  Leaves it in pick_own, and the sum up to and with it in pick_mass.
        // Up to one token per thread, a thread counts what is in front of its own; longer lists are sorted.
        auto last_of = [&](u64* list, uint32_t n, bool by_sum, uint32_t base_count, u64 base_mass, uint32_t want_count, double want_mass) {
          if (n <= kThreads) {
            const u64 mine = tid < (int)n ? list[tid] : 0ull, own = tid < (int)n ? mass_of(mine) : 0ull;
            sh.mass[tid] = own;
            __syncthreads();
            if (tid < (int)n) {
              uint32_t front = base_count;
              u64 sum = base_mass;
#pragma unroll 8
              for (uint32_t j = 0; j < n; ++j) {
                const bool before = list[j] > mine;
                front += before;
                sum += before ? sh.mass[j] : 0ull;
              }
              const bool last = front + 1 == base_count + n;
              if (by_sum ? (double)sum < want_mass && (last || !((double)(sum + own) < want_mass)) : front + 1 == want_count) {
                sh.pick_own = mine;
                sh.pick_mass = sum + own;
              }
            }
          } else {
            sort_list(list, (int)n);
            const uint32_t lo = tid * kListPer, hi = min(lo + kListPer, n);
            u64 mine = 0, sum = base_mass;
            for (uint32_t j = lo; j < hi; ++j) mine += mass_of(list[j]);
            uint32_t unused = 0;
            scan_bins(0u, mine, unused, sum);
            for (uint32_t j = lo; j < hi; ++j) {
              const u64 next = sum + mass_of(list[j]);
              if (by_sum ? (double)sum < want_mass && (j + 1 == n || !((double)next < want_mass)) : base_count + j + 1 == want_count) {
                sh.pick_own = list[j];
                sh.pick_mass = next;
              }
              sum = next;
            }
          }
          __syncthreads();
        };
        u64 found = 0;
        if (bin_k >= 0) {
          last_of(sh.list[0], n_k, false, sh.found.count_k, total, (uint32_t)top_k, 0.0);
          total = sh.pick_mass;
          found = sh.pick_own;
          __syncthreads();
        }
        if (by_mass) {
          const double want = (double)top_p * (double)total;
          if (tid == 0) sh.pick_mass = 0;
          __syncthreads();
          last_of(sh.list[1], n_p, true, 0u, above, 0u, want);
          // the cut is where the estimate said if less than `want` lies in front of the list and no less than that up to its end
          if (tid == 0 && (!((double)above < want) || (double)sh.pick_mass < want)) sh.found.slow = 1;
          found = sh.pick_own > found ? sh.pick_own : found;
          for (uint32_t j = tid; j < n_p; j += kThreads) {
            const u64 c = sh.list[1][j];
            if (c < found || !(logit_of((uint32_t)(c >> kIndexBits)) >= floor_min)) continue;
            const int at = (1 << kIndexBits) - 1 - (int)(c & ((1u << kIndexBits) - 1u)), owner = (at + run.head) / Run<kBf16>::kUnit / run.per;
            const u64 u = mass_of(c);
            const uint32_t add = (uint32_t)u, old = atomicAdd(&sh.extra_lo[owner], add);
            const uint32_t carry = (uint32_t)(u >> 32) + (old + add < old ? 1u : 0u);
            if (carry) atomicAdd(&sh.extra_hi[owner], carry);
          }
        }
        if (tid == 0) sh.found.cut = found;
      }
    }
    cluster_sync();
    if (ld_cluster_u32(peer(&sh.found.slow, 0)) == 0u) {
      cut = ld_cluster_u64(peer(&sh.found.cut, 0));
      summed = by_mass && !(floor_min > p_high);  // min_p leaves what is in front of the listed bins
    } else {
      // by digits: counts and sums over the tokens of a bin that share a prefix, 11 bits of (logit, index) further each time
      u64 total = ld_cluster_u64(peer(&sh.found.total, 0));
#pragma unroll 1
      for (int task = 0; task < 2; ++task) {
        const bool by_sum = task == 1;
        if (by_sum ? !by_mass : bin_k < 0) continue;
        const double want_mass = (double)top_p * (double)total;
        int bin = 0;
        uint32_t base_count = 0;
        u64 base_mass = 0, prefix = 0;
#pragma unroll 1
        for (int d = kDigits; d >= 0; --d) {  // the first time over the bins
          const int shift = d * kDigitBits;
          clear_bins();
          __syncthreads();
          run.template each4<1>(floor_all, [&](const float(&l)[4], int at) {
#pragma unroll 1
            for (int e = 0; e < 4; ++e) {
              const float x = e < 2 ? (e == 0 ? l[0] : l[1]) : (e == 2 ? l[2] : l[3]);
              if (!(x >= floor_all)) continue;
              double rest;
              const int i = w.place(x, rest);
              int b = bin_of(i);
              if (d < kDigits) {
                if (b != bin) continue;
                const u64 c = composite(x, at + e);
                if (d < kDigits - 1 && c >> (shift + kDigitBits) != prefix) continue;
                b = kBins - 1 - (int)((c >> shift) & (kBins - 1));  // the largest first
              }
              const u64 u = w.units(w.scaled(i, rest));
              const uint32_t add = (uint32_t)u, old = atomicAdd(&sh.lo[b], add);
              const uint32_t carry = (uint32_t)(u >> 32) + (old + add < old ? 1u : 0u);
              if (carry) atomicAdd(&sh.hi[b], carry);
              atomicAdd(&sh.count[b], 1u);
            }
          });
          cluster_sync();
          // the bin with before < want <= before + its own
          uint32_t c[kBinsPer], csum = 0, cb = base_count;
          u64 m[kBinsPer], msum = 0, mb = base_mass;
#pragma unroll
          for (int j = 0; j < kBinsPer; ++j) {
            const int b = tid * kBinsPer + j;
            c[j] = 0;
            m[j] = 0;
            for (int r = 0; r < n_blocks; ++r) {
              c[j] += ld_cluster_u32(peer(&sh.count[b], r));
              m[j] += ((u64)ld_cluster_u32(peer(&sh.hi[b], r)) << 32) + ld_cluster_u32(peer(&sh.lo[b], r));
            }
            csum += c[j];
            msum += m[j];
          }
          scan_bins(csum, msum, cb, mb);
#pragma unroll
          for (int j = 0; j < kBinsPer; ++j) {
            if (c[j] != 0u && (by_sum ? (double)mb < want_mass && !((double)(mb + m[j]) < want_mass) : cb < (uint32_t)top_k && (uint32_t)top_k <= cb + c[j])) {
              sh.pick_bin = tid * kBinsPer + j;
              sh.pick_count = cb;
              sh.pick_mass = mb;
              sh.pick_own = m[j];
            }
            cb += c[j];
            mb += m[j];
          }
          cluster_sync();  // nobody clears its bins before all have read them
          if (d == kDigits)
            bin = sh.pick_bin;
          else
            prefix = (prefix << kDigitBits) | (u64)(kBins - 1 - sh.pick_bin);
          base_count = sh.pick_count;
          base_mass = sh.pick_mass;
        }
        cut = prefix > cut ? prefix : cut;
        total = base_mass + sh.pick_own;
        __syncthreads();
      }
    }
  }

  // ---- 3. the token ----
  // what stays: the logits above floor_kept, and of those that equal cut_logit the tokens up to cut_at
  float floor_kept = floor_min, cut_logit = -inf;
  int cut_at = 0;
  if (cut != 0) {
    cut_logit = logit_of((uint32_t)(cut >> kIndexBits));
    cut_at = (1 << kIndexBits) - 1 - (int)(cut & ((1u << kIndexBits) - 1));
    floor_kept = fmaxf(floor_kept, cut_logit);
  }
  auto stays = [&](float l, int at) { return l >= floor_kept && (l > cut_logit || at <= cut_at); };
  // the weights of four tokens: whole numbers, so that a thread's sum (little more than 2^10 tokens of up to 2^42) is exact in double
  auto sum4 = [&](const float(&l)[4], int at, double& sum) {
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      double rest;
      const int i = w.place(l[e], rest);
      const double u = (w.scaled(i, rest) + w.kWhole) - w.kWhole;
      if (stays(l[e], at + e)) sum += u;
    }
  };
  u64 sum;
  if (summed) {
    const int owner = rank * kWarps + warp;
    sum = sh.slot_part[warp] + ((u64)ld_cluster_u32(peer(&sh.extra_hi[owner], 0)) << 32) + ld_cluster_u32(peer(&sh.extra_lo[owner], 0));
  } else {
    double thread_sum = 0.0;
    run.template each4<2>(floor_kept, [&](const float(&l)[4], int at) { sum4(l, at, thread_sum); });
    sum = (u64)thread_sum;
#pragma unroll
    for (int d = 16; d > 0; d >>= 1) sum += __shfl_xor_sync(all, sum, d);
  }
  __syncthreads();
  if (lane == 0) sh.warp64[warp] = sum;
  __syncthreads();
  u64 mine = 0;
  for (int v = 0; v < kWarps; ++v) mine += sh.warp64[v];
  if (tid == 0) sh.slot64b[rank] = mine;
  cluster_sync();
  const u64 part_sum = lane < n_blocks ? ld_cluster_u64(peer(&sh.slot64b[lane], lane)) : 0ull;  // a lane per block
  u64 before = lane < rank ? part_sum : 0ull, total = part_sum;
#pragma unroll
  for (int d = 4; d > 0; d >>= 1) {
    before += __shfl_xor_sync(all, before, d);
    total += __shfl_xor_sync(all, total, d);
  }
  before = __shfl_sync(all, before, 0);
  total = __shfl_sync(all, total, 0);
  __syncwarp();
  cluster_arrive();
  const u64 want = place_of(total);
  if (before <= want && want < before + mine) {  // this block has it
    int holder = 0;
    for (; before + sh.warp64[holder] <= want; ++holder) before += sh.warp64[holder];
    // that warp's run in equal parts over all warps
    const Run<kBf16> held(p.logits, row * p.stride, p.vocab, rank, n_blocks, holder);
    const int part = (held.last - held.first + kThreads - 1) / kThreads * 32;
    const int u_first = min(held.first + warp * part, held.last), u_last = min(u_first + part, held.last);
    auto unit_sum = [&](const uint4& v, int unit) -> u64 {
      double t = 0.0;
      run.four(v, unit, floor_kept, [&](const float(&l)[4], int at) { sum4(l, at, t); });
      return (u64)t;
    };
    sum = 0;
    for (int unit = u_first + lane; unit < u_last; unit += 32) sum += unit_sum(run.load(unit), unit);
#pragma unroll
    for (int d = 16; d > 0; d >>= 1) sum += __shfl_xor_sync(all, sum, d);
    if (lane == 0) sh.slot_part[warp] = sum;
    __syncthreads();
    for (int v = 0; v < warp; ++v) before += sh.slot_part[v];
    if (before <= want && want < before + sum) {
      for (int u0 = u_first; u0 < u_last; u0 += 32) {
        const int unit = u0 + lane;
        const uint4 v = unit < u_last ? run.load(unit) : make_uint4(0u, 0u, 0u, 0u);
        const u64 own = unit < u_last ? unit_sum(v, unit) : 0ull;
        u64 x = own;
#pragma unroll
        for (int d = 1; d < 32; d <<= 1) {
          const u64 o = __shfl_up_sync(all, x, d);
          if (lane >= d) x += o;
        }
        const unsigned over = __ballot_sync(all, before + x > want);
        if (over != 0u) {
          if (lane == __ffs(over) - 1) {
            u64 front = before + x - own;
#pragma unroll 1
            for (int e = 0; e < Run<kBf16>::kUnit && front <= want; ++e) {
              const int at = run.index(unit) + e;
              if ((unsigned)at >= (unsigned)p.vocab) continue;
              const float l = kBf16 ? __bfloat162float(static_cast<const __nv_bfloat16*>(p.logits)[row * p.stride + at])
                                    : static_cast<const float*>(p.logits)[row * p.stride + at];
              if (!stays(l, at)) continue;
              double rest;
              const int i = w.place(l, rest);
              const double v = w.scaled(i, rest);
              front += w.units(v);
              if (front > want) {
                p.tokens[row] = at;
                if (p.probs) p.probs[row] = (float)(v / (double)total);
              }
            }
          }
          break;
        }
        before += __shfl_sync(all, x, 31);
      }
    }
  }
  __syncwarp();
  cluster_wait();
}

}  // namespace

cudaError_t sample_setup() {
  cudaError_t e = cudaFuncSetAttribute(sample_kernel<false>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)sizeof(Shared));
  if (e == cudaSuccess) e = cudaFuncSetAttribute(sample_kernel<true>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)sizeof(Shared));
  return e;
}

cudaError_t launch_sample(SampleParams p, int sm_count, cudaStream_t stream) {
  // more blocks per row while the device has places for them (two per SM) and each keeps 2048 tokens
  int blocks = 1;
  while (blocks < 8 && p.n * blocks * 2 <= 2 * sm_count && p.vocab > 4096 * blocks) blocks *= 2;
  if (p.vocab > (1 << 19) && blocks == 1) blocks = 2;  // at most 2^10 tokens per thread (and a unit): sums exact in double
  p.blocks = blocks;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)(p.n * blocks));
  cfg.blockDim = dim3(kThreads);
  cfg.dynamicSmemBytes = sizeof(Shared);
  cfg.stream = stream;
  cudaLaunchAttribute attr;
  attr.id = cudaLaunchAttributeClusterDimension;
  attr.val.clusterDim.x = blocks;
  attr.val.clusterDim.y = attr.val.clusterDim.z = 1;
  cfg.attrs = &attr;
  cfg.numAttrs = 1;
  return p.bf16 ? cudaLaunchKernelEx(&cfg, sample_kernel<true>, p) : cudaLaunchKernelEx(&cfg, sample_kernel<false>, p);
}

}  // namespace rk
