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
//   2. where top-k or top-p is on: counts and sums in 2048 bins of (max - l) / T; the bin that holds the cut is taken
//      apart by 11 bits of (logit, index) at a time until the cut is one token
//   3. sums of what stays, by block and by warp; the warp that holds u * total walks its run
#include <cuda_bf16.h>

#include "rk_internal.h"

namespace rk {
namespace {

constexpr int kThreads = 512, kWarps = kThreads / 32;
constexpr int kBins = 2048;
constexpr int kUnitLog2 = 42;                    // weights are multiples of 2^-42
constexpr float kOctaves = 43.f;                 // weights below 2^-43 round to nothing
constexpr int kIndexBits = 20, kDigitBits = 11, kKeyBits = 32 + kIndexBits, kDigits = (kKeyBits + kDigitBits - 1) / kDigitBits;
typedef unsigned long long u64;

struct Shared {
  double table[64];              // 2^(-j/64)
  u64 slot64[8];                 // one word per block of the cluster
  u64 slot64b[8];
  u64 warp64[kWarps];
  uint32_t warp32[kWarps];
  uint32_t nan[8];
  int pick_bin;
  uint32_t pick_count;           // tokens in front of the picked bin
  u64 pick_mass;                 // and their sum
  u64 pick_own;                  // sum of the picked bin
  uint32_t picked;
  uint32_t count[kBins], lo[kBins], hi[kBins];
};

// order of logits: larger key, larger logit; both zeros are one
__device__ __forceinline__ uint32_t key_of(float l) {
  const uint32_t b = __float_as_uint(l + 0.f);
  return b & 0x80000000u ? ~b : b | 0x80000000u;
}
__device__ __forceinline__ float logit_of(uint32_t key) { return __uint_as_float(key & 0x80000000u ? key & 0x7fffffffu : ~key); }

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
__device__ __forceinline__ void cluster_sync() {
  cluster_arrive();
  cluster_wait();
}

struct Row {
  float top;       // the largest logit
  double rate;     // log2(e) / T
  const double* table;
  // weight in octaves below the largest: log2(p_max / p)
  __device__ __forceinline__ double octaves(float l) const {
    return l == top ? 0.0 : ((double)top - (double)l) * rate;
  }
  __device__ __forceinline__ double weight(double x) const {  // 2^-x for 0 <= x < 44
    const double s = rint(x * 64.0);
    const double r = fma(s, -0x1p-6, x) * -0.69314718055994530942;
    const double e = fma(fma(fma(fma(r, 1.0 / 24.0, 1.0 / 6.0), r, 0.5), r, 1.0), r, 1.0);
    const int i = (int)s;
    return __hiloint2double((1023 - (i >> 6)) << 20, 0) * (table[i & 63] * e);
  }
};

template <bool kBf16>
__global__ void __launch_bounds__(kThreads) sample_kernel(const SampleParams p) {
  __shared__ Shared sh;
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const int n_blocks = p.blocks, rank = (int)cluster_ctarank();
  const int64_t row = blockIdx.x / n_blocks;
  const unsigned all = 0xffffffffu;
  const float* row_f = static_cast<const float*>(p.logits) + row * p.stride;
  const __nv_bfloat16* row_h = static_cast<const __nv_bfloat16*>(p.logits) + row * p.stride;
  const int per = ((p.vocab + n_blocks * kThreads - 1) / (n_blocks * kThreads)) * 32;  // tokens per warp
  const int lo = (rank * kWarps + warp) * per;
  const int hi = min(lo + per, p.vocab);
  auto logit = [&](int i) -> float { return kBf16 ? __bfloat162float(row_h[i]) : row_f[i]; };
  auto peer = [&](const void* at, int r) -> uint32_t { return mapa_shared(smem_u32(at), r); };

  if (tid < 64) sh.table[tid] = exp2(-(double)tid / 64.0);

  // ---- 1. the largest logit and the lowest index that has it ----
  u64 best = 0;
  bool nan = false;
  for (int i = lo + lane; i < hi; i += 32) {
    const float l = logit(i);
    nan |= l != l;
    const u64 c = ((u64)key_of(l) << 32) | (uint32_t)~i;
    best = c > best ? c : best;
  }
#pragma unroll
  for (int d = 16; d > 0; d >>= 1) {
    const u64 o = __shfl_xor_sync(all, best, d);
    best = o > best ? o : best;
  }
  const int any_nan = __syncthreads_or(nan);
  if (lane == 0) sh.warp64[warp] = best;
  __syncthreads();
  if (tid == 0) {
    for (int w = 1; w < kWarps; ++w) best = sh.warp64[w] > best ? sh.warp64[w] : best;
    sh.slot64[rank] = best;
    sh.nan[rank] = any_nan;
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
  Row w;
  w.top = top;
  w.rate = 1.44269504088896340736 / (double)temp;
  w.table = sh.table;
  const double one = (double)(1ull << kUnitLog2);
  auto units = [&](double weight) -> u64 { return (u64)__double2ll_rn(weight * one); };
  auto composite = [&](float l, int i) -> u64 { return ((u64)key_of(l) << kIndexBits) | (uint32_t)((1 << kIndexBits) - 1 - i); };

  const int top_k = p.top_k ? p.top_k[row] : 0;
  const float top_p = p.top_p ? p.top_p[row] : 1.f, min_p = p.min_p ? p.min_p[row] : 0.f;
  u64 cut = 0;  // tokens whose composite is at least this stay
  const u64 first_composite = composite(top, first);
  if (top_p <= 0.f || min_p > 1.f || top_k == 1) cut = first_composite;
  const bool by_mass = cut == 0 && top_p < 1.f;
  const bool by_count = cut == 0 && top_k > 1 && top_k < p.vocab;

  // ---- 2. the cut ----
  // Counts and sums over the tokens for which digit(l, x, i) is a bin; all blocks end with the cluster's.
  auto histogram = [&](bool mass, auto digit) {
    for (int b = tid; b < kBins; b += kThreads) sh.count[b] = sh.lo[b] = sh.hi[b] = 0u;
    __syncthreads();
    for (int i = lo + lane; i < hi; i += 32) {
      const float l = logit(i);
      const double x = w.octaves(l);
      if (!(x < (double)kOctaves)) continue;
      const int b = digit(l, x, i);
      if (b < 0) continue;
      atomicAdd(&sh.count[b], 1u);
      if (mass) {
        const u64 u = units(w.weight(x));
        const uint32_t add = (uint32_t)u, old = atomicAdd(&sh.lo[b], add);
        const uint32_t carry = (uint32_t)(u >> 32) + (old + add < old ? 1u : 0u);
        if (carry) atomicAdd(&sh.hi[b], carry);
      }
    }
    cluster_sync();
  };
  // The bin with before < want <= before + its own, in counts (want_count) or sums (want_mass).  base_*: in front of bin 0.
  // Returns false if all bins together do not reach it; pick_* are then the totals.
  auto pick = [&](bool by_sum, uint32_t base_count, u64 base_mass, uint32_t want_count, double want_mass) -> bool {
    constexpr int kPer = kBins / kThreads;
    uint32_t c[kPer], csum = 0;
    u64 m[kPer], msum = 0;
#pragma unroll
    for (int j = 0; j < kPer; ++j) {
      const int b = tid * kPer + j;
      c[j] = 0;
      m[j] = 0;
      for (int r = 0; r < n_blocks; ++r) {
        c[j] += ld_cluster_u32(peer(&sh.count[b], r));
        m[j] += ((u64)ld_cluster_u32(peer(&sh.hi[b], r)) << 32) + ld_cluster_u32(peer(&sh.lo[b], r));
      }
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
    if (lane == 31) {
      sh.warp32[warp] = cx;
      sh.warp64[warp] = mx;
    }
    if (tid == 0) sh.picked = 0u;
    __syncthreads();
    uint32_t cb = base_count + cx - csum;
    u64 mb = base_mass + mx - msum;
    for (int v = 0; v < warp; ++v) {
      cb += sh.warp32[v];
      mb += sh.warp64[v];
    }
#pragma unroll
    for (int j = 0; j < kPer; ++j) {
      const bool here = c[j] != 0u && (by_sum ? (double)mb < want_mass && !((double)(mb + m[j]) < want_mass) : cb < want_count && want_count <= cb + c[j]);
      if (here) {
        sh.pick_bin = tid * kPer + j;
        sh.pick_count = cb;
        sh.pick_mass = mb;
        sh.pick_own = m[j];
        sh.picked = 1u;
      }
      cb += c[j];
      mb += m[j];
    }
    __syncthreads();
    const bool found = sh.picked != 0u;
    if (!found && tid == kThreads - 1) {
      sh.pick_count = cb;
      sh.pick_mass = mb;
    }
    __syncthreads();
    cluster_sync();  // nobody clears its bins before all have read them
    return found;
  };
  const float bin_scale = (float)kBins / kOctaves;
  auto coarse = [&](float, double x, int) -> int { return min((int)((float)x * bin_scale), kBins - 1); };
  // From the picked coarse bin down to one token; sets `cut` and returns the sum up to and with it.
  auto refine = [&](bool by_sum, uint32_t want_count, double want_mass) -> u64 {
    const int bin = sh.pick_bin;
    uint32_t base_count = sh.pick_count;
    u64 base_mass = sh.pick_mass, prefix = 0;
    for (int d = kDigits - 1; d >= 0; --d) {
      const int shift = d * kDigitBits;
      histogram(true, [&](float l, double x, int i) -> int {
        if (coarse(l, x, i) != bin) return -1;
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
    u64 total = 0;
    bool known = false;
    if (by_count) {
      histogram(by_mass, coarse);
      if (pick(false, 0u, 0ull, (uint32_t)top_k, 0.0)) {
        total = refine(false, (uint32_t)top_k, 0.0);
        known = true;
      }
    }
    if (by_mass) {
      histogram(true, coarse);
      if (!known) {
        pick(true, 0u, 0ull, 0u, 1e300);  // all of them
        total = sh.pick_mass;
      }
      const double want = (double)top_p * (double)total;
      if (pick(true, 0u, 0ull, 0u, want)) refine(true, 0u, want);
    }
  }

  // ---- 3. the token ----
  const double least = min_p > 1.f ? 1.0 : (double)min_p;  // above 1: the cut has decided; NaN compares false: off
  auto stays = [&](float l, int i, double& weight) -> u64 {
    const double x = w.octaves(l);
    if (!(x < (double)kOctaves)) return 0ull;
    weight = w.weight(x);
    if (weight < least || composite(l, i) < cut) return 0ull;
    return units(weight);
  };
  u64 sum = 0;
  double weight = 0.0;
  for (int i = lo + lane; i < hi; i += 32) sum += stays(logit(i), i, weight);
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
    for (int i0 = lo; i0 < hi; i0 += 32) {
      const int i = i0 + lane;
      const u64 mine = i < hi ? stays(logit(i), i, weight) : 0ull;
      u64 run = mine;
#pragma unroll
      for (int d = 1; d < 32; d <<= 1) {
        const u64 v = __shfl_up_sync(all, run, d);
        if (lane >= d) run += v;
      }
      const unsigned over = __ballot_sync(all, before + run > want);
      if (over != 0u) {
        if (lane == __ffs(over) - 1) {
          p.tokens[row] = i;
          if (p.probs) p.probs[row] = (float)(weight * one / (double)total);
        }
        break;
      }
      before += __shfl_sync(all, run, 31);
    }
  }
  cluster_wait();
}

}  // namespace

cudaError_t launch_sample(SampleParams p, int sm_count, cudaStream_t stream) {
  int blocks = 1;
  while (blocks < 8 && (p.vocab > 16384 * blocks || (int64_t)p.n * blocks * 2 <= sm_count) && p.vocab > 2048 * blocks) blocks *= 2;
  p.blocks = blocks;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)(p.n * blocks));
  cfg.blockDim = dim3(kThreads);
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
