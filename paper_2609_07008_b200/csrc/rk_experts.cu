// Routing to experts: scores, groups, the k best, their weights (rk_moe_route), and the list of (token, slot) pairs by
// expert that the expert products walk (rk_moe_group).
#include <cuda_bf16.h>

#include "rk_internal.h"

namespace rk {
namespace {

// ------------------------------------------------------------------------------------------------------------
// rk_moe_route: one token per warp.  The lanes are split evenly over the groups (L lanes per group, L a power of two), lane
// `sub` of group g holds experts sub, sub + L, ... of the group, so that a group's rank is a reduction over L neighbours.
// Scores are compared in 64 bits: with a few hundred experts the k-th and the next score of a token are closer than fp32
// rounding about once in 10^4 tokens, and the choice would depend on the instruction that computed them.
// ------------------------------------------------------------------------------------------------------------
constexpr int kRouteWarps = 8;
constexpr double kNone = -__builtin_huge_val();

__device__ __forceinline__ double max_f64(double a, double b) { return a > b ? a : b; }

template <int kPer, bool kBf16>
__global__ void __launch_bounds__(32 * kRouteWarps) moe_route_kernel(const RouteParams p) {
  const int64_t token = (int64_t)blockIdx.x * kRouteWarps + (threadIdx.x >> 5);
  if (token >= p.n) return;
  const int lane = threadIdx.x & 31;
  const int width = 1 << p.lanes_log2;  // lanes per group
  const int g = lane >> p.lanes_log2, sub = lane & (width - 1);
  const unsigned all = 0xffffffffu;
  double s[kPer], c[kPer];
  bool bad = false;
  double top = kNone;
#pragma unroll
  for (int i = 0; i < kPer; ++i) {
    const int j = sub + i * width;
    float x = -__int_as_float(0x7f800000);
    if (g < p.n_groups && j < p.group_size) {
      const int64_t at = token * p.stride + g * p.group_size + j;
      x = kBf16 ? __bfloat162float(static_cast<const __nv_bfloat16*>(p.logits)[at]) : static_cast<const float*>(p.logits)[at];
    }
    bad |= x != x;
    s[i] = (double)x;
    top = max_f64(top, s[i]);
  }
  if (p.softmax) {
#pragma unroll
    for (int d = 16; d > 0; d >>= 1) top = max_f64(top, __shfl_xor_sync(all, top, d));
    double sum = 0.0;
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
      c[i] = s[i] == kNone ? kNone : 0.0;
      s[i] = s[i] == kNone ? 0.0 : exp(s[i] - top);
      sum += s[i];
    }
#pragma unroll
    for (int d = 16; d > 0; d >>= 1) sum += __shfl_xor_sync(all, sum, d);
#pragma unroll
    for (int i = 0; i < kPer; ++i) s[i] /= sum;
  } else {
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
      c[i] = s[i] == kNone ? kNone : 0.0;
      s[i] = s[i] == kNone ? 0.0 : 1.0 / (1.0 + exp(-s[i]));
    }
  }
#pragma unroll
  for (int i = 0; i < kPer; ++i) {
    const int j = sub + i * width;
    if (c[i] == kNone) continue;
    c[i] = s[i];
    if (p.bias) c[i] += (double)p.bias[g * p.group_size + j];
    bad |= c[i] != c[i];
  }
  int32_t* ids = p.ids + token * p.k;
  float* weights = p.weights + token * p.k;
  if (__any_sync(all, bad)) {
    if (lane < p.k) {
      ids[lane] = -1;
      weights[lane] = __int_as_float(0x7fc00000);
    }
    return;
  }
  if (p.n_groups > 1) {
    // the two largest of the group
    double a = kNone, b = kNone;
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
      b = max_f64(b, a < c[i] ? a : c[i]);
      a = max_f64(a, c[i]);
    }
    for (int d = width >> 1; d > 0; d >>= 1) {
      const double a2 = __shfl_xor_sync(all, a, d), b2 = __shfl_xor_sync(all, b, d);
      b = max_f64(max_f64(b, b2), a < a2 ? a : a2);
      a = max_f64(a, a2);
    }
    const double rank = p.group_top == 2 && b != kNone ? a + b : a;
    int better = 0;
    for (int h = 0; h < p.n_groups; ++h) {
      const double r = __shfl_sync(all, rank, h << p.lanes_log2);
      better += r > rank || (r == rank && h < g);
    }
    if (better >= p.top_groups) {
#pragma unroll
      for (int i = 0; i < kPer; ++i) c[i] = kNone;
    }
  }
  // the k best, one after another
  double w = 0.0, sum = 0.0;
  int id = -1;
  for (int q = 0; q < p.k; ++q) {
    double best = kNone, score = 0.0;
    int at = 0x7fffffff;
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
      if (c[i] > best) {
        best = c[i];
        score = s[i];
        at = g * p.group_size + sub + i * width;
      }
    }
    const int mine = at;
#pragma unroll
    for (int d = 16; d > 0; d >>= 1) {
      const double b2 = __shfl_xor_sync(all, best, d), s2 = __shfl_xor_sync(all, score, d);
      const int a2 = __shfl_xor_sync(all, at, d);
      if (b2 > best || (b2 == best && a2 < at)) {
        best = b2;
        score = s2;
        at = a2;
      }
    }
    if (best == kNone) break;
    if (mine == at) {
#pragma unroll
      for (int i = 0; i < kPer; ++i)
        if (g * p.group_size + sub + i * width == at) c[i] = kNone;
    }
    sum += score;
    if (lane == q) {
      w = score;
      id = at;
    }
  }
  if (lane < p.k) {
    if (p.renorm) w = sum > 0.0 ? w / sum : 0.0;
    ids[lane] = id;
    weights[lane] = (float)(w * (double)p.scale);
  }
}

// ------------------------------------------------------------------------------------------------------------
// rk_moe_group: a stable counting sort of the pairs by expert, by one cluster, without atomics and without a workspace.
// Every warp owns a run of consecutive pairs and a count per expert in shared memory; lanes with the same expert find one
// another by match.any, the lowest of them adds their number.  Scans over warps, over the cluster's blocks (through
// distributed shared memory) and over experts turn the counts into places; a second walk over the same run writes the list.
// ------------------------------------------------------------------------------------------------------------
constexpr int kGroupThreads = 1024, kGroupWarps = kGroupThreads / 32;

__device__ __forceinline__ int ld_cluster_s32(uint32_t addr) {
  int v;
  asm volatile("ld.shared::cluster.s32 %0, [%1];" : "=r"(v) : "r"(addr) : "memory");
  return v;
}

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
  for (int e = threadIdx.x; e < kGroupWarps * n_e; e += kGroupThreads) count[e] = 0;
  __syncthreads();
  auto expert_of = [&](int64_t i) -> int {
    if (i >= hi) return -1;
    const int e = p.ids[i];
    if ((unsigned)e >= (unsigned)n_e) return -1;
    if (p.keep != nullptr) {
      const int64_t t = i / p.k;
      if (!((p.keep[t] >> (int)(i - t * p.k)) & 1)) return -1;
    }
    return e;
  };
  for (int64_t i = lo; i < hi; i += 32) {
    const int e = expert_of(i + lane);
    const unsigned same = __match_any_sync(0xffffffffu, e);
    if (e >= 0 && lane == __ffs(same) - 1) mine[e] += __popc(same);
    __syncwarp();
  }
  __syncthreads();
  for (int e = threadIdx.x; e < n_e; e += kGroupThreads) {
    int sum = 0;
    for (int w = 0; w < kGroupWarps; ++w) {
      const int v = count[w * n_e + e];
      count[w * n_e + e] = sum;
      sum += v;
    }
    total[e] = sum;
  }
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
  cluster_arrive();  // no block leaves before the others have read its counts
  for (int64_t i = lo; i < hi; i += 32) {
    const int e = expert_of(i + lane);
    const unsigned same = __match_any_sync(0xffffffffu, e);
    const unsigned below = same & ((1u << lane) - 1u);
    int at = 0;
    if (e >= 0) at = mine[e];
    __syncwarp();
    if (e >= 0) {
      p.rows[base[e] + at + __popc(below)] = (int32_t)(i + lane);
      if (below == 0u) mine[e] = at + __popc(same);
    }
    __syncwarp();
  }
  for (int64_t i = (int64_t)sum_all + (int64_t)rank * kGroupThreads + threadIdx.x; i < n; i += (int64_t)n_blocks * kGroupThreads) p.rows[i] = -1;
  cluster_wait();
}

template <bool kBf16>
cudaError_t route_dispatch(const RouteParams& p, int per, cudaStream_t stream) {
  const unsigned grid = (unsigned)((p.n + kRouteWarps - 1) / kRouteWarps);
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

cudaError_t experts_setup() {
  return cudaFuncSetAttribute(moe_group_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (kGroupWarps + 2) * kMaxExperts * 4);
}

cudaError_t launch_moe_route(RouteParams p, cudaStream_t stream) {
  p.lanes_log2 = 5;
  while (p.lanes_log2 > 0 && (32 >> p.lanes_log2) < p.n_groups) --p.lanes_log2;  // 32 / lanes per group >= groups
  const int per = (p.group_size + (1 << p.lanes_log2) - 1) >> p.lanes_log2;
  return p.bf16 ? route_dispatch<true>(p, per, stream) : route_dispatch<false>(p, per, stream);
}

cudaError_t launch_moe_group(const GroupParams& p, cudaStream_t stream) {
  // eight blocks where their walks (32 pairs per warp and step) are longer than the cluster's two barriers
  const int n_blocks = p.n * p.k > 4 * kGroupThreads ? 8 : 1;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(n_blocks);
  cfg.blockDim = dim3(kGroupThreads);
  cfg.dynamicSmemBytes = (size_t)(kGroupWarps + 2) * p.n_experts * 4;
  cfg.stream = stream;
  cudaLaunchAttribute attr;
  attr.id = cudaLaunchAttributeClusterDimension;
  attr.val.clusterDim.x = n_blocks;
  attr.val.clusterDim.y = attr.val.clusterDim.z = 1;
  cfg.attrs = &attr;
  cfg.numAttrs = 1;
  return cudaLaunchKernelEx(&cfg, moe_group_kernel, p);
}

}  // namespace rk
