// Sampling a token from each row of logits: temperature, top-k, top-p, min-p, and one given random number per row.
//
// p_i = exp((l_i - max) / T), as whole numbers of 2^-42 (a token below 2^-43 of the largest weighs nothing).  Whole numbers
// add up to the same sum in any order, so that sums, cuts and the chosen token depend on the inputs alone, and their error
// (2^-43 per token) is far below the distance at which two neighbouring tokens' borders could be confused.  The
// exponential is taken in double: x = n + j / 64 + r, 2^-j/64 from a table, 2^-r by its Taylor series to degree 4
// (|r| <= 1/128: 4e-14).
//
// The three filters each keep a prefix of one order, falling logit and then rising index, so together they keep the tokens
// not below one (logit, index) pair, the cut.  A row belongs to a cluster of thread blocks, each with a run of consecutive tokens.
//   1. the largest logit (and whether there is a NaN)
//   2. where top-k or top-p is on: counts and sums in 2048 bins of (max - l) / T, joined in the first block; the tokens of
//      the bin that holds a cut (some hundred of 128 K) go to the first block too, which sorts them and finds the cut.
//      Where they are too many (thousands of equal logits), the bin is taken apart by 11 bits of (logit, index) at a time.
//   3. sums of what stays, by block and by warp; the warp that holds u * total walks its run
// The row is read again by each step: it comes out of L2 after the first.
#include <cuda_bf16.h>

#include "rk_internal.h"

namespace rk {
namespace {

constexpr int kThreads = 512, kWarps = kThreads / 32;
constexpr int kBins = 2048, kBinsPer = kBins / kThreads;
constexpr int kList = 2048;                      // tokens of a cut's bin that are sorted in shared memory
constexpr int kUnitLog2 = 42;                    // weights are multiples of 2^-42
constexpr float kOctaves = 43.f;                 // weights below 2^-43 round to nothing
constexpr int kIndexBits = 20, kDigitBits = 11, kKeyBits = 32 + kIndexBits, kDigits = (kKeyBits + kDigitBits - 1) / kDigitBits;
constexpr int kUnroll = 4;                       // 16-byte loads that a thread has under way
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
  double table[64];              // 2^(-j/64)
  u64 list[2][kList];            // (key, index) of the tokens in bin_k and in bin_lo .. bin_hi
  uint32_t listed[2];
  uint32_t count[kBins], lo[kBins], hi[kBins];
  u64 slot64[8];                 // one word per block of the cluster
  u64 slot64b[8];
  u64 warp64[kWarps];
  uint32_t warp32[kWarps];
  uint32_t nan[8];
  Found found;
  int pick_bin;
  uint32_t pick_count;           // tokens in front of the picked bin
  u64 pick_mass;                 // and their sum
  u64 pick_own;                  // sum of the picked bin
  uint32_t picked;
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

struct Weights {
  float top;       // the largest logit
  double rate;     // log2(e) / T
  const double* table;
  // octaves below the largest: log2(p_max / p)
  __device__ __forceinline__ double octaves(float l) const { return l == top ? 0.0 : ((double)top - (double)l) * rate; }
  __device__ __forceinline__ double weight(double x) const {  // 2^-x for 0 <= x < 44
    const double s = rint(x * 64.0);
    const double r = fma(s, -0x1p-6, x) * -0.69314718055994530942;
    const double e = fma(fma(fma(fma(r, 1.0 / 24.0, 1.0 / 6.0), r, 0.5), r, 1.0), r, 1.0);
    const int i = (int)s;
    return __hiloint2double((1023 - (i >> 6)) << 20, 0) * (table[i & 63] * e);
  }
};
__device__ __forceinline__ u64 units(double weight) { return (u64)__double2ll_rn(weight * (double)(1ull << kUnitLog2)); }
__device__ __forceinline__ int coarse_bin(double x) { return min((int)((float)x * ((float)kBins / kOctaves)), kBins - 1); }

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
    uint32_t w[4] = {0u, 0u, 0u, 0u};
#pragma unroll
    for (int e = 0; e < kUnit; ++e) {
      if ((unsigned)(index(unit) + e) >= (unsigned)vocab) continue;
      if constexpr (kBf16)
        w[e >> 1] |= (uint32_t) * (reinterpret_cast<const uint16_t*>(p) + e) << (16 * (e & 1));
      else
        w[e] = *(reinterpret_cast<const uint32_t*>(p) + e);
    }
    return make_uint4(w[0], w[1], w[2], w[3]);
  }
  static __device__ __forceinline__ float value(const uint4& v, int e) {
    const uint32_t w[4] = {v.x, v.y, v.z, v.w};
    if constexpr (kBf16) return __uint_as_float(e & 1 ? w[e >> 1] & 0xffff0000u : w[e >> 1] << 16);
    return __uint_as_float(w[e]);
  }
  // f(logit, index) for every token of the warp, ascending within a lane
  template <class F>
  __device__ __forceinline__ void each(F f) const {
    const int lane = threadIdx.x & 31;
    for (int u0 = first + lane; u0 < last; u0 += 32 * kUnroll) {
      uint4 v[kUnroll];
#pragma unroll
      for (int j = 0; j < kUnroll; ++j)
        if (u0 + 32 * j < last) v[j] = load(u0 + 32 * j);
#pragma unroll
      for (int j = 0; j < kUnroll; ++j) {
        if (u0 + 32 * j >= last) break;
        const int i = index(u0 + 32 * j);
#pragma unroll
        for (int e = 0; e < kUnit; ++e)
          if ((unsigned)(i + e) < (unsigned)vocab) f(value(v[j], e), i + e);
      }
    }
  }
};

// Sorts list[0 .. n) descending; n <= kList.  All threads of the block; ends with a barrier.
__device__ __forceinline__ void sort_list(u64* list, int n) {
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
  const Run<kBf16> run(p.logits, row * p.stride, p.vocab, rank, n_blocks, warp);
  auto peer = [&](const void* at, int r) -> uint32_t { return mapa_shared(smem_u32(at), r); };
  auto clear_bins = [&] {
    for (int b = tid; b < kBins; b += kThreads) sh.count[b] = sh.lo[b] = sh.hi[b] = 0u;
  };

  if (tid < 64) sh.table[tid] = exp2(-(double)tid / 64.0);
  if (tid < 2) sh.listed[tid] = 0u;
  clear_bins();

  // ---- 1. the largest logit and the lowest index that has it ----
  u64 best = 0;
  {
    float top = -__int_as_float(0x7f800000);
    int at = 0;
    bool nan = false;
    run.each([&](float l, int i) {
      nan |= l != l;
      if (l > top) {
        top = l;
        at = i;
      }
    });
    best = ((u64)key_of(top) << 32) | (uint32_t)~at;
#pragma unroll
    for (int d = 16; d > 0; d >>= 1) {
      const u64 o = __shfl_xor_sync(all, best, d);
      best = o > best ? o : best;
    }
    if (lane == 0) sh.warp64[warp] = best;
    const int any_nan = __syncthreads_or(nan);
    if (tid == 0) {
      for (int w = 1; w < kWarps; ++w) best = sh.warp64[w] > best ? sh.warp64[w] : best;
      sh.slot64[rank] = best;
      sh.nan[rank] = any_nan;
    }
  }
  cluster_sync();
  uint32_t nan_all = 0;
  best = 0;
  for (int r = 0; r < n_blocks; ++r) {
    const u64 o = ld_cluster_u64(peer(&sh.slot64[r], r));
    nan_all |= ld_cluster_u32(peer(&sh.nan[r], r));
    best = o > best ? o : best;
  }
  const float top = logit_of((uint32_t)(best >> 32));
  const int first = (int)~(uint32_t)best;
  const float temp = p.temperature ? p.temperature[row] : 1.f;
  const bool dead = nan_all || !(top > -__int_as_float(0x7f800000));
  if (dead || !(temp > 0.f)) {
    if (rank == 0 && tid == 0) {
      p.tokens[row] = dead ? -1 : first;
      if (p.probs) p.probs[row] = dead ? __int_as_float(0x7fc00000) : 1.f;
    }
    cluster_sync();  // the others may still be reading this block's slots
    return;
  }
  Weights w;
  w.top = top;
  w.rate = 1.44269504088896340736 / (double)temp;
  w.table = sh.table;

  const int top_k = p.top_k ? p.top_k[row] : 0;
  const float top_p = p.top_p ? p.top_p[row] : 1.f, min_p = p.min_p ? p.min_p[row] : 0.f;
  u64 cut = 0;  // tokens whose composite is at least this stay
  if (top_p <= 0.f || min_p > 1.f || top_k == 1) cut = composite(top, first);
  const bool by_mass = cut == 0 && top_p < 1.f;
  const bool by_count = cut == 0 && top_k > 1 && top_k < p.vocab;
  // logits below this weigh nothing (a little lower than exactly, rounding included): a cheap test in front of the double one
  const float floor_all = top == __int_as_float(0x7f800000) ? top : (float)((double)top - 43.01 / w.rate - 1e-6 * fabs((double)top));

  // ---- 2. the cut ----
  // Adds a token to a bin.
  auto add_bin = [&](int b, bool mass, double x) {
    atomicAdd(&sh.count[b], 1u);
    if (mass) {
      const u64 u = units(w.weight(x));
      const uint32_t add = (uint32_t)u, old = atomicAdd(&sh.lo[b], add);
      const uint32_t carry = (uint32_t)(u >> 32) + (old + add < old ? 1u : 0u);
      if (carry) atomicAdd(&sh.hi[b], carry);
    }
  };
  // This thread's bins kBinsPer * tid ...: exclusive sums over the block (its own bins only, no other blocks').
  auto scan_bins = [&](const uint32_t (&c)[kBinsPer], const u64 (&m)[kBinsPer], uint32_t& cb, u64& mb) {
    uint32_t csum = 0;
    u64 msum = 0;
#pragma unroll
    for (int j = 0; j < kBinsPer; ++j) {
      csum += c[j];
      msum += m[j];
    }
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
  // ---- by digits: for bins too full to be sorted.  Counts and sums over the tokens for which digit(l, x, i) is a bin ----
  auto histogram = [&](auto digit) {
    clear_bins();
    __syncthreads();
    run.each([&](float l, int i) {
      if (l < floor_all) return;
      const double x = w.octaves(l);
      if (!(x < (double)kOctaves)) return;
      const int b = digit(l, x, i);
      if (b >= 0) add_bin(b, true, x);
    });
    cluster_sync();
  };
  // The bin with before < want <= before + its own, in counts (want_count) or sums (want_mass).  base_*: in front of bin 0.
  auto pick = [&](bool by_sum, uint32_t base_count, u64 base_mass, uint32_t want_count, double want_mass) {
    uint32_t c[kBinsPer];
    u64 m[kBinsPer];
#pragma unroll
    for (int j = 0; j < kBinsPer; ++j) {
      const int b = tid * kBinsPer + j;
      c[j] = 0;
      m[j] = 0;
      for (int r = 0; r < n_blocks; ++r) {
        c[j] += ld_cluster_u32(peer(&sh.count[b], r));
        m[j] += ((u64)ld_cluster_u32(peer(&sh.hi[b], r)) << 32) + ld_cluster_u32(peer(&sh.lo[b], r));
      }
    }
    uint32_t cb = base_count;
    u64 mb = base_mass;
    scan_bins(c, m, cb, mb);
#pragma unroll
    for (int j = 0; j < kBinsPer; ++j) {
      if (c[j] != 0u && (by_sum ? (double)mb < want_mass && !((double)(mb + m[j]) < want_mass) : cb < want_count && want_count <= cb + c[j])) {
        sh.pick_bin = tid * kBinsPer + j;
        sh.pick_count = cb;
        sh.pick_mass = mb;
        sh.pick_own = m[j];
      }
      cb += c[j];
      mb += m[j];
    }
    cluster_sync();  // nobody clears its bins before all have read them
  };
  // The last token in the order with before < want; sets `cut` and returns the sum up to and with it.
  auto search = [&](bool by_sum, uint32_t want_count, double want_mass) -> u64 {
    histogram([&](float, double x, int) -> int { return coarse_bin(x); });
    pick(by_sum, 0u, 0ull, want_count, want_mass);
    const int bin = sh.pick_bin;
    uint32_t base_count = sh.pick_count;
    u64 base_mass = sh.pick_mass, prefix = 0;
    for (int d = kDigits - 1; d >= 0; --d) {
      const int shift = d * kDigitBits;
      histogram([&](float l, double x, int i) -> int {
        if (coarse_bin(x) != bin) return -1;
        const u64 c = composite(l, i);
        if (d < kDigits - 1 && c >> (shift + kDigitBits) != prefix) return -1;
        return kBins - 1 - (int)((c >> shift) & (kBins - 1));  // the largest first
      });
      pick(by_sum, base_count, base_mass, want_count, want_mass);
      prefix = (prefix << kDigitBits) | (u64)(kBins - 1 - sh.pick_bin);
      base_count = sh.pick_count;
      base_mass = sh.pick_mass;
    }
    cut = prefix > cut ? prefix : cut;
    return base_mass + sh.pick_own;
  };

  if (by_count || by_mass) {
    run.each([&](float l, int) {
      if (l < floor_all) return;
      const double x = w.octaves(l);
      if (x < (double)kOctaves) add_bin(coarse_bin(x), by_mass, x);
    });
    __syncthreads();
    if (rank != 0) {
      for (int b = tid; b < kBins; b += kThreads) {
        if (sh.count[b] == 0u) continue;
        add_cluster_u32(peer(&sh.count[b], 0), sh.count[b]);
        if (by_mass) {
          const uint32_t add = sh.lo[b], old = add_cluster_u32(peer(&sh.lo[b], 0), add);
          const uint32_t carry = sh.hi[b] + (old + add < old ? 1u : 0u);
          if (carry) add_cluster_u32(peer(&sh.hi[b], 0), carry);
        }
      }
    }
    cluster_sync();
    if (rank == 0) {
      uint32_t c[kBinsPer], cb0 = 0;
      u64 m[kBinsPer], mb0 = 0;
#pragma unroll
      for (int j = 0; j < kBinsPer; ++j) {
        c[j] = sh.count[tid * kBinsPer + j];
        m[j] = ((u64)sh.hi[tid * kBinsPer + j] << 32) + sh.lo[tid * kBinsPer + j];
      }
      scan_bins(c, m, cb0, mb0);
      if (tid == 0) {
        sh.found.bin_k = sh.found.bin_lo = sh.found.bin_hi = -1;
        sh.found.slow = 0;
        sh.found.mass_lo = 0;
        u64 t = 0;
        for (int v = 0; v < kWarps; ++v) t += sh.warp64[v];
        sh.found.total = t;
      }
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
    run.each([&](float l, int i) {
      if (l < floor_all) return;
      const double x = w.octaves(l);
      if (!(x < (double)kOctaves)) return;
      const int b = coarse_bin(x);
      if (b == bin_k) {
        const uint32_t at = add_cluster_u32(peer(&sh.listed[0], 0), 1u);
        if (at < kList) st_cluster_u64(peer(&sh.list[0][at], 0), composite(l, i));
      }
      if (by_mass && b >= bin_lo && b <= bin_hi) {
        const uint32_t at = add_cluster_u32(peer(&sh.listed[1], 0), 1u);
        if (at < kList) st_cluster_u64(peer(&sh.list[1][at], 0), composite(l, i));
      }
    });
    cluster_sync();
    if (rank == 0) {
      const uint32_t n_k = bin_k >= 0 ? sh.listed[0] : 0u, n_p = by_mass ? sh.listed[1] : 0u;
      if (n_k > kList || n_p > kList) {
        if (tid == 0) sh.found.slow = 1;
      } else {
        // a list in order, `per` consecutive places per thread: the sum in front of this thread's places
        auto sum_in_front = [&](const u64* list, uint32_t n, u64 base) -> u64 {
          const uint32_t lo = tid * (kList / kThreads);
          u64 mine = 0;
          for (uint32_t j = lo; j < lo + kList / kThreads && j < n; ++j) mine += units(w.weight(w.octaves(logit_of((uint32_t)(list[j] >> kIndexBits)))));
          u64 x = mine;
#pragma unroll
          for (int d = 1; d < 32; d <<= 1) {
            const u64 v = __shfl_up_sync(all, x, d);
            if (lane >= d) x += v;
          }
          __syncthreads();
          if (lane == 31) sh.warp64[warp] = x;
          __syncthreads();
          x += base - mine;
          for (int v = 0; v < warp; ++v) x += sh.warp64[v];
          return x;
        };
        if (tid == 0) sh.found.cut = 0;
        u64 total = sh.found.total;
        if (bin_k >= 0) {
          sort_list(sh.list[0], (int)n_k);
          const uint32_t at = (uint32_t)top_k - sh.found.count_k - 1;  // place of the k-th token
          if (tid == 0) sh.found.cut = sh.list[0][at];
          if (by_mass) {
            u64 front = sum_in_front(sh.list[0], n_k, sh.found.mass_k);
            for (uint32_t j = tid * (kList / kThreads); j < (tid + 1) * (kList / kThreads) && j <= at; ++j) {
              front += units(w.weight(w.octaves(logit_of((uint32_t)(sh.list[0][j] >> kIndexBits)))));
              if (j == at) sh.pick_mass = front;
            }
            __syncthreads();
            total = sh.pick_mass;
          }
        }
        if (by_mass) {
          sort_list(sh.list[1], (int)n_p);
          const double want = (double)top_p * (double)total;
          u64 front = sum_in_front(sh.list[1], n_p, sh.found.mass_lo);
          for (uint32_t j = tid * (kList / kThreads); j < (tid + 1) * (kList / kThreads) && j < n_p; ++j) {
            const u64 next = front + units(w.weight(w.octaves(logit_of((uint32_t)(sh.list[1][j] >> kIndexBits)))));
            // the last one with less than `want` in front of it
            if ((double)front < want && (!((double)next < want) || j + 1 == n_p)) sh.pick_own = sh.list[1][j];
            front = next;
          }
          __syncthreads();
          if (tid == 0 && sh.pick_own > sh.found.cut) sh.found.cut = sh.pick_own;
        }
      }
    }
    cluster_sync();
    if (ld_cluster_u32(peer(&sh.found.slow, 0)) == 0u) {
      cut = ld_cluster_u64(peer(&sh.found.cut, 0));
    } else {
      u64 total = ld_cluster_u64(peer(&sh.found.total, 0));
      if (bin_k >= 0) total = search(false, (uint32_t)top_k, 0.0);
      if (by_mass) search(true, 0u, (double)top_p * (double)total);
    }
  }

  // ---- 3. the token ----
  const double least = min_p > 1.f ? 1.0 : (double)min_p;  // above 1: the cut has decided; NaN compares false: off
  float floor_kept = fmaxf(floor_all, logit_of(max((uint32_t)(cut >> kIndexBits), key_of(-__int_as_float(0x7f800000)))));
  if (min_p > 0.f && top < __int_as_float(0x7f800000))
    floor_kept = fmaxf(floor_kept, (float)((double)top - (0.01 - (double)log2f((float)least)) / w.rate - 1e-6 * fabs((double)top)));
  auto stays = [&](float l, int i, double& weight) -> u64 {
    if (l < floor_kept) return 0ull;
    const double x = w.octaves(l);
    if (!(x < (double)kOctaves)) return 0ull;
    const double mine = w.weight(x);
    if (mine < least || composite(l, i) < cut) return 0ull;
    weight = mine;
    return units(mine);
  };
  u64 sum = 0;
  double weight = 0.0;
  run.each([&](float l, int i) { sum += stays(l, i, weight); });
#pragma unroll
  for (int d = 16; d > 0; d >>= 1) sum += __shfl_xor_sync(all, sum, d);
  __syncthreads();
  if (lane == 0) sh.warp64[warp] = sum;
  __syncthreads();
  if (tid == 0) {
    u64 t = 0;
    for (int v = 0; v < kWarps; ++v) t += sh.warp64[v];
    sh.slot64b[rank] = t;
  }
  cluster_sync();
  u64 before = 0, total = 0;
  for (int r = 0; r < n_blocks; ++r) {
    const u64 t = ld_cluster_u64(peer(&sh.slot64b[r], r));
    if (r < rank) before += t;
    total += t;
  }
  cluster_arrive();
  for (int v = 0; v < warp; ++v) before += sh.warp64[v];
  const float u = p.u[row];
  u64 want = u > 0.f ? (u64)((double)u * (double)total) : 0ull;
  want = want < total ? want : total - 1;
  if (before <= want && want < before + sum) {
    for (int u0 = run.first; u0 < run.last; u0 += 32) {
      const int unit = u0 + lane;
      u64 mine = 0;
      uint4 v = make_uint4(0u, 0u, 0u, 0u);
      if (unit < run.last) {
        v = run.load(unit);
#pragma unroll
        for (int e = 0; e < Run<kBf16>::kUnit; ++e)
          if ((unsigned)(run.index(unit) + e) < (unsigned)p.vocab) mine += stays(run.value(v, e), run.index(unit) + e, weight);
      }
      u64 x = mine;
#pragma unroll
      for (int d = 1; d < 32; d <<= 1) {
        const u64 o = __shfl_up_sync(all, x, d);
        if (lane >= d) x += o;
      }
      const unsigned over = __ballot_sync(all, before + x > want);
      if (over != 0u) {
        if (lane == __ffs(over) - 1) {
          u64 front = before + x - mine;
#pragma unroll
          for (int e = 0; e < Run<kBf16>::kUnit; ++e) {
            const int i = run.index(unit) + e;
            if ((unsigned)i >= (unsigned)p.vocab || front > want) continue;
            front += stays(run.value(v, e), i, weight);
            if (front > want) {
              p.tokens[row] = i;
              if (p.probs) p.probs[row] = (float)(weight * (double)(1ull << kUnitLog2) / (double)total);
            }
          }
        }
        break;
      }
      before += __shfl_sync(all, x, 31);
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
  while (blocks < 8 && p.n * blocks * 2 <= 2 * sm_count && p.vocab > 4096 * blocks) blocks *= 2;
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
