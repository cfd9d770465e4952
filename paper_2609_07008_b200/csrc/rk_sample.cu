// Sampling a token from each row of logits: temperature, top-k, top-p, min-p, and one given random number per row.
//
// p_i = exp((l_i - max) / T), as whole numbers of 2^-42 (a token below 2^-42 of the largest weighs nothing).  Whole numbers
// add up to the same sum in any order, so that sums, cuts and the chosen token depend on the inputs alone, and their error
// (2^-42 per token) is far below the distance at which two neighbouring tokens' borders could be confused.  The
// exponential is taken in double: 256 x = i + r with i whole, 2^-i/256 from a table and a shift, 2^-r/256 by its Taylor
// series to degree 3 (|r| <= 1/2: 1.4e-13).  A token costs eleven double-precision instructions that way, which bounds the
// passes that need every token's weight; 64-bit conversions, four times as slow, are done in integers.
//
// The three filters each keep a prefix of one order, falling logit and then rising index, so together they keep the tokens
// not below one (logit, index) pair, the cut.  A row belongs to a cluster of thread blocks, each with a run of consecutive tokens.
//   1. the largest logit (and whether there is a NaN)
//   2. where top-k or top-p is on: counts and sums in bins of i, joined in the first block; the tokens of the bins that hold
//      a cut (some hundred of 128 K) go to the first block too, which ranks them and finds the cut.
//      Where they are too many (thousands of equal logits), the bin is taken apart by 11 bits of (logit, index) at a time.
//   3. sums of what stays, by block and by warp; the block that holds u * total shares out the warp's run that holds it
// The row is read again by each step: it comes out of L2 after the first.
#include <cuda_bf16.h>

#include "rk_internal.h"

namespace rk {
namespace {

#ifndef SAMPLE_MAX
#define SAMPLE_MAX 8
#define SAMPLE_MIN 4096
#endif
constexpr int kThreads = 512, kWarps = kThreads / 32;
constexpr int kBins = 2048, kBinsPer = kBins / kThreads;
constexpr int kList = 2048, kListPer = kList / kThreads;  // tokens of a cut's bins that are ranked in shared memory
constexpr int kUnitLog2 = 42;                    // weights are multiples of 2^-42
constexpr int kSteps = 256;                      // i counts 256ths of an octave below the largest
constexpr int kEnd = kUnitLog2 * kSteps;         // from here on tokens weigh nothing
constexpr int kIndexBits = 20, kDigitBits = 11, kKeyBits = 32 + kIndexBits, kDigits = (kKeyBits + kDigitBits - 1) / kDigitBits;
typedef unsigned long long u64;

struct Found {           // what the first block of a row's cluster tells the others
  int bin_k;             // bin of the top-k cut, or -1
  int bin_lo, bin_hi;    // bins that may hold the top-p cut; empty if bin_lo > bin_hi
  int slow;              // the lists overflowed
  uint32_t count_k;      // tokens in front of bin_k
  u64 mass_k, mass_lo;   // sums in front of bin_k and of bin_lo
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
  u64 slot_part[kWarps];
  u64 warp64[kWarps];
  uint32_t warp32[kWarps];
  float top[8];
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
__device__ __forceinline__ void cluster_sync() {
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
// The lowest logit for which `in` holds; it holds for all larger ones up to `top`, and `guess` is within a few roundings of it.
template <class F>
__device__ __forceinline__ float lowest(float guess, float top, F in) {
  constexpr float kLowest = -3.402823466e38f;
  float x = fminf(fmaxf(guess, kLowest), top);
  while (x < top && !in(x)) x = nextafterf(x, top);
  while (x > kLowest && in(nextafterf(x, kLowest))) x = nextafterf(x, kLowest);
  return x;
}
// bins of i: 64 to an octave for the first 16 octaves, then 32
constexpr int kFine = 16 * kSteps;
__device__ __forceinline__ int bin_of(int i) { return i < kFine ? i >> 2 : (kFine >> 2) + ((i - kFine) >> 3); }
__device__ __forceinline__ int bin_begin(int b) { return b < kFine >> 2 ? b << 2 : kFine + ((b - (kFine >> 2)) << 3); }
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

  __device__ __forceinline__ Run(const void* logits, int64_t at, int vocab_, int block, int n_blocks, int warp) : vocab(vocab_) {
    const uintptr_t a = reinterpret_cast<uintptr_t>(logits) + at * (kBf16 ? 2 : 4);
    base = reinterpret_cast<const uint8_t*>(a & ~(uintptr_t)15);
    head = (int)(a & 15) / (kBf16 ? 2 : 4);
    const int n = (head + vocab + kUnit - 1) / kUnit, per = (n + n_blocks * kWarps * 32 - 1) / (n_blocks * kWarps * 32) * 32;
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

  if (tid < 2) sh.listed[tid] = 0u;
  for (int j = tid; j < kSteps; j += kThreads) sh.table[j] = exp2((double)kUnitLog2 - (double)j / kSteps);
  clear_bins();

  // ---- 1. the largest logit ----
  float top = run.top();
#pragma unroll
  for (int d = 16; d > 0; d >>= 1) top = max_nan(top, __shfl_xor_sync(all, top, d));
  if (lane == 0) sh.warp32[warp] = __float_as_uint(top);
  __syncthreads();
  if (tid == 0) {
    for (int w = 1; w < kWarps; ++w) top = max_nan(top, __uint_as_float(sh.warp32[w]));
    sh.top[rank] = top;
  }
  cluster_sync();
  top = -inf;
  for (int r = 0; r < n_blocks; ++r) top = max_nan(top, __uint_as_float(ld_cluster_u32(peer(&sh.top[r], r))));
  const float temp = p.temperature ? p.temperature[row] : 1.f;
  const int top_k = p.top_k ? p.top_k[row] : 0;
  const float top_p = p.top_p ? p.top_p[row] : 1.f, min_p = p.min_p ? p.min_p[row] : 0.f;
  const bool dead = !(top > -inf);
  const bool one = !(temp > 0.f) || top_p <= 0.f || min_p > 1.f || top_k == 1;  // the first token only
  if (dead || one) {
    uint32_t at = 0xffffffffu;
    if (!dead)
      run.template each4<4>(top, [&](const float(&l)[4], int i) { at = min(at, (uint32_t)(i + (l[0] == top ? 0 : l[1] == top ? 1 : l[2] == top ? 2 : 3))); });
    at = __reduce_min_sync(all, at);
    __syncthreads();
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
  // The logit `steps` 256ths of an octave below the largest, a little lower (rounding included), but above -inf; next to
  // +inf nothing else counts.
  auto below = [&](double steps) -> float {
    if (top == inf) return top;
    return fmaxf((float)((double)top - steps / w.rate - 1e-6 * fabs((double)top)), -3.402823466e38f);
  };
  const float floor_all = top == inf ? top : lowest((float)((double)top - ((double)kEnd - 0.5) / w.rate), top, [&](float l) {
    double rest;
    return w.depth(l) < (double)kEnd + 1.0 && w.place(l, rest) < kEnd;
  });  // tokens from here on up weigh something

  // ---- 2. the cut ----
  auto add_bin = [&](int b, bool count, bool mass, u64 u) {
    if (count) atomicAdd(&sh.count[b], 1u);
    if (mass) {
      const uint32_t add = (uint32_t)u, old = atomicAdd(&sh.lo[b], add);
      const uint32_t carry = (uint32_t)(u >> 32) + (old + add < old ? 1u : 0u);
      if (carry) atomicAdd(&sh.hi[b], carry);
    }
  };
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

  if (by_count || by_mass) {
    run.template each4<2>(floor_all, [&](const float(&l)[4], int) {
      int i[4];
      u64 u[4];
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        double rest;
        i[e] = w.place(l[e], rest);
        u[e] = by_mass ? w.units(w.scaled(i[e], rest)) : 0ull;
      }
#pragma unroll
      for (int e = 0; e < 4; ++e)
        if (l[e] >= floor_all) add_bin(bin_of(i[e]), by_count, by_mass, u[e]);
    });
    __syncthreads();
    if (rank != 0) {
      for (int b = tid; b < kBins; b += kThreads) {
        if (by_count && sh.count[b] != 0u) add_cluster_u32(peer(&sh.count[b], 0), sh.count[b]);
        if (by_mass && (sh.lo[b] | sh.hi[b]) != 0u) {
          const uint32_t add = sh.lo[b], old = add_cluster_u32(peer(&sh.lo[b], 0), add);
          const uint32_t carry = sh.hi[b] + (old + add < old ? 1u : 0u);
          if (carry) add_cluster_u32(peer(&sh.hi[b], 0), carry);
        }
      }
    }
    cluster_sync();
    if (rank == 0) {
      uint32_t c[kBinsPer], csum = 0, cb0 = 0;
      u64 m[kBinsPer], msum = 0, mb0 = 0;
#pragma unroll
      for (int j = 0; j < kBinsPer; ++j) {
        csum += c[j] = sh.count[tid * kBinsPer + j];
        msum += m[j] = ((u64)sh.hi[tid * kBinsPer + j] << 32) + sh.lo[tid * kBinsPer + j];
      }
      scan_bins(csum, msum, cb0, mb0);
      if (tid == 0) {
        sh.found.bin_k = sh.found.bin_lo = sh.found.bin_hi = -1;
        sh.found.slow = 0;
        sh.found.mass_lo = 0;
        sh.found.cut = 0;
      }
      if (tid == kThreads - 1) sh.found.total = mb0 + msum;
      __syncthreads();
      uint32_t cb = cb0;
      u64 mb = mb0;
#pragma unroll
      for (int j = 0; j < kBinsPer; ++j) {
        if (by_count && cb < (uint32_t)top_k && (uint32_t)top_k <= cb + c[j]) {
          sh.found.bin_k = tid * kBinsPer + j;
          sh.found.count_k = cb;
          sh.found.mass_k = mb;
          sh.pick_own = m[j];
        }
        cb += c[j];
        mb += m[j];
      }
      __syncthreads();
      if (by_mass) {
        // the sum over the top k is known up to what bin_k holds
        const bool limited = sh.found.bin_k >= 0;
        const double least = (double)top_p * (double)(limited ? sh.found.mass_k : sh.found.total);
        const double most = (double)top_p * (double)(limited ? sh.found.mass_k + sh.pick_own : sh.found.total);
        mb = mb0;
#pragma unroll
        for (int j = 0; j < kBinsPer; ++j) {
          if ((double)mb < least && !((double)(mb + m[j]) < least)) {
            sh.found.bin_lo = tid * kBinsPer + j;
            sh.found.mass_lo = mb;
          }
          if ((double)mb < most && !((double)(mb + m[j]) < most)) sh.found.bin_hi = tid * kBinsPer + j;
          mb += m[j];
        }
        __syncthreads();
        if (tid == 0 && sh.found.bin_lo < 0) sh.found.bin_lo = 0;  // the top k lie in the first bin
      }
    }
    cluster_sync();
    const int bin_k = (int)ld_cluster_u32(peer(&sh.found.bin_k, 0));
    const int bin_lo = (int)ld_cluster_u32(peer(&sh.found.bin_lo, 0)), bin_hi = (int)ld_cluster_u32(peer(&sh.found.bin_hi, 0));
    {
      // one window of logits around the bins; the doubles decide inside it
      int from = kBins, to = -1;
      if (bin_k >= 0) from = to = bin_k;
      if (by_mass) {
        from = min(from, bin_lo);
        to = max(to, bin_hi);
      }
      const float high = from <= 0 || top == inf ? inf : (float)((double)top - (double)(bin_begin(from) - 2) / w.rate + 1e-6 * fabs((double)top));
      const float low = fmaxf(floor_all, below((double)bin_begin(to + 1) + 2.0));
      run.template each4<4>(low, [&](const float(&l)[4], int at) {
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          if (!(l[e] >= low && l[e] <= high)) continue;
          double rest;
          const int b = bin_of(w.place(l[e], rest));
          if (b == bin_k) {
            const uint32_t slot = add_cluster_u32(peer(&sh.listed[0], 0), 1u);
            if (slot < kList) st_cluster_u64(peer(&sh.list[0][slot], 0), composite(l[e], at + e));
          }
          if (by_mass && b >= bin_lo && b <= bin_hi) {
            const uint32_t slot = add_cluster_u32(peer(&sh.listed[1], 0), 1u);
            if (slot < kList) st_cluster_u64(peer(&sh.list[1][slot], 0), composite(l[e], at + e));
          }
        }
      });
    }
    cluster_sync();
    if (rank == 0) {
      const uint32_t n_k = bin_k >= 0 ? sh.listed[0] : 0u, n_p = by_mass ? sh.listed[1] : 0u;
      if (n_k > kList || n_p > kList) {
        if (tid == 0) sh.found.slow = 1;
      } else {
        auto mass_of = [&](u64 c) -> u64 { return w.units(logit_of((uint32_t)(c >> kIndexBits))); };
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
        u64 total = sh.found.total, found = 0;
        if (bin_k >= 0) {
          last_of(sh.list[0], n_k, false, sh.found.count_k, sh.found.mass_k, (uint32_t)top_k, 0.0);
          total = sh.pick_mass;
          found = sh.pick_own;
          __syncthreads();
        }
        if (by_mass) {
          last_of(sh.list[1], n_p, true, 0u, sh.found.mass_lo, 0u, (double)top_p * (double)total);
          found = sh.pick_own > found ? sh.pick_own : found;
        }
        if (tid == 0) sh.found.cut = found;
      }
    }
    cluster_sync();
    if (ld_cluster_u32(peer(&sh.found.slow, 0)) == 0u) {
      cut = ld_cluster_u64(peer(&sh.found.cut, 0));
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
              add_bin(b, true, true, w.units(w.scaled(i, rest)));
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
  float floor_kept = floor_all, cut_logit = -inf;
  int cut_at = 0;
  if (cut != 0) {
    cut_logit = logit_of((uint32_t)(cut >> kIndexBits));
    cut_at = (1 << kIndexBits) - 1 - (int)(cut & ((1u << kIndexBits) - 1));
    floor_kept = fmaxf(floor_kept, cut_logit);
  }
  if (min_p > 0.f && top < inf) {  // (NaN: off)
    const double most = -(double)kSteps * log2((double)min_p);
    floor_kept = fmaxf(floor_kept, lowest((float)((double)top - most / w.rate), top, [&](float l) { return w.depth(l) <= most; }));
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
  double thread_sum = 0.0;
  run.template each4<2>(floor_kept, [&](const float(&l)[4], int at) { sum4(l, at, thread_sum); });
  u64 sum = (u64)thread_sum;
#pragma unroll
  for (int d = 16; d > 0; d >>= 1) sum += __shfl_xor_sync(all, sum, d);
  __syncthreads();
  if (lane == 0) sh.warp64[warp] = sum;
  __syncthreads();
  u64 mine = 0;
  for (int v = 0; v < kWarps; ++v) mine += sh.warp64[v];
  if (tid == 0) sh.slot64b[rank] = mine;
  cluster_sync();
  u64 before = 0, total = 0;
  for (int r = 0; r < n_blocks; ++r) {
    const u64 t = ld_cluster_u64(peer(&sh.slot64b[r], r));
    if (r < rank) before += t;
    total += t;
  }
  cluster_arrive();
  const float u = p.u[row];
  u64 want = u > 0.f ? (u64)((double)u * (double)total) : 0ull;
  want = want < total ? want : total - 1;
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
  while (blocks < SAMPLE_MAX && p.n * blocks * 2 <= 2 * sm_count && p.vocab > SAMPLE_MIN * blocks) blocks *= 2;
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
