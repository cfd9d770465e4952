// Products of a few token rows with 4-bit weight matrices (the decode-time projections W_uv, W_a, W_b):
//   y[t][m][i] = sum_k x[t][m][k] * n[m][i][k] * s[m][i][k / group],   n in -7..7, s in bf16.
//
// The weights are read once and are the whole cost: k/2 + 2 k/group bytes per output row.  A warp takes 16 output
// rows and 64-wide blocks of k: its 32 lanes read one contiguous 512-byte block, 16 bytes each, which hold exactly the
// A fragments of four m16n8k16 products.  Code n + 8 in the low mantissa bits of 0x4300 is the bf16 number 136 + n;
// subtracting 136 is exact, so the products are exact and sum in fp32; the scale multiplies the finished sum of a
// group in fp32.  mma.sync is the right instruction here: the tokens (N = 8 per product) would leave a tcgen05 tile
// almost empty, and the tensor work is a fraction of what the dequantisation costs anyway.
//
// Fragment order: step s of a block, lane t of a quad, holds k = 32 (s >> 1) + 8 t + 4 (s & 1) + {0, 1 | 2, 3}.  Any
// order of k serves a sum; this one makes a lane's x values of two steps 16 contiguous bytes and keeps each pair of
// steps inside 32 consecutive k, the smallest group.
#include <cuda_bf16.h>

#include "rk_internal.h"

namespace rk {
namespace {

constexpr int kWarps = 8, kThreads = 32 * kWarps;
constexpr int kMaxBlocks = 4;                           // 64-wide blocks of k whose x a warp keeps in registers
constexpr int kSliceBlocks = kWarps * kMaxBlocks;       // blocks of k of one thread block at a time: 2048 k
constexpr int kMaxSplit = 8;                            // thread blocks that share k (a portable cluster)
constexpr int kStages = 2;
constexpr int kBatch = 2;                               // tiles per stage
constexpr int kUnit = 512;                              // fp32 sums of one 16 x 8 product, in fragment order
constexpr int kMaxRun = 32;                             // products of one thread block in all
constexpr int kSmemBytes = 108 * 1024;                  // two thread blocks share an SM

// d = a b + (first ? 0 : d)
template <bool kFirst>
__device__ __forceinline__ void mma_16816(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
  if constexpr (kFirst) {
    asm(
        "mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%10, %10, %10, %10};"
        : "=f"(d[0]), "=f"(d[1]), "=f"(d[2]), "=f"(d[3])
        : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1), "f"(0.f));
  } else {
    asm(
        "mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
        : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
        : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
  }
}

__device__ __forceinline__ void unpack_codes(uint32_t v, uint32_t (&a)[4]) {
  const uint32_t k136 = 0x43084308u;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    uint32_t t;  // (v >> 4 i) & 0x000f000f | 0x43004300
    asm("lop3.b32 %0, %1, %2, %3, 0xea;" : "=r"(t) : "r"(v >> (4 * i)), "r"(0x000f000fu), "r"(0x43004300u));
    const __nv_bfloat162 n = __hsub2(*reinterpret_cast<const __nv_bfloat162*>(&t), *reinterpret_cast<const __nv_bfloat162*>(&k136));
    a[i] = *reinterpret_cast<const uint32_t*>(&n);
  }
}

__device__ __forceinline__ void bulk_load(uint32_t dst, const void* src, uint32_t bytes, uint32_t bar) {
  asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];" ::"r"(dst), "l"(src),
               "r"(bytes), "r"(bar)
               : "memory");
}

__device__ __forceinline__ float load_peer(uint32_t at) {
  float v;
  asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(v) : "r"(at) : "memory");
  return v;
}

// A thread block owns a slice of k and a run of 16-row tiles; x of its slice stays in its warps' registers (as B
// fragments, kBlocks blocks of 64 per warp) while the weights of tile after tile pass by, two tiles' slices of codes and
// scales per pipeline stage.  So x is read once per cluster and not once per tile: for 16 tokens x weighs twice a tile's
// codes.  The thread blocks of a cluster hold the slices of the same run; sums go lanes -> warps (in warp order, through
// shared memory) -> slices (in rank order, out of the peers' shared memory), so that results do not depend on timing.
// Measured: 16384 -> 7168 with 16 tokens 26 us, 8192 -> 4096 with one token 8.2 us, 64 matrices of 512 -> 128 with five tokens
// 3.9 us, two of 1024 -> 256 with one 3.3 us.  With x in the pipeline beside the codes, once per pair of tiles, they took 52,
// 10.4, 4.3 and 3.1 us.  The large ones are bound by the latencies of unpack -> product -> scale with 16 warps per SM (the
// registers that hold x leave no room for more; ALU 33 %, tensor pipe 28 %, issue slots 39 % busy), the small ones by the
// start of a kernel and one trip to memory.
template <int NT, int kGroup, int kBlocks>
__global__ void __launch_bounds__(kThreads, 2) rk_matvec4_kernel(const __grid_constant__ Matvec4Params p) {
  extern __shared__ __align__(128) uint8_t smem[];
  __shared__ __align__(8) uint64_t bars[kStages];
  __shared__ int abort_word;
  constexpr int kUnits = kBatch * NT;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
  const int tiles = p.n_out >> 4, kb = p.k >> 6;
  const int rank = (int)(blockIdx.x % p.split), unit = (int)(blockIdx.x / p.split);
  const int mat = unit / p.runs, tile0 = (unit - mat * p.runs) * p.run;
  const int n_tiles = min(p.run, tiles - tile0), n_batches = (n_tiles + kBatch - 1) / kBatch;
  const int64_t tok0 = (int64_t)blockIdx.y * 8 * NT;
  const int n_tok = (int)min((int64_t)8 * NT, p.n_tok - tok0);
  const uint32_t smem_base = smem_u32(smem), bar0 = smem_u32(bars);
  const uint32_t tile_bytes = p.stage_bytes / kBatch, off_red = p.stages * p.stage_bytes, off_out = off_red + p.red_bytes;
  volatile int* abort_flag = &abort_word;
  // 64-wide blocks of k in this thread block's slice of a pass; none behind the end
  auto blocks = [&](int pass) -> int { return max(0, min(p.slice, kb - (pass * p.split + rank) * p.slice)); };
  auto load = [&](int pass, int batch, int s) {  // one thread
    const int b0 = (pass * p.split + rank) * p.slice, nb = blocks(pass);
    if (nb == 0) return;
    const int g0 = b0 * 64 / kGroup, ng = nb * 64 / kGroup, groups = p.k / kGroup;
    const int n = min(kBatch, n_tiles - batch * kBatch);
    const int64_t tile = (int64_t)mat * tiles + tile0 + batch * kBatch;
    mbar_arrive_expect_tx(bar0 + 8u * s, (uint32_t)(n * (nb * 512 + ng * 32)));
    for (int i = 0; i < n; ++i) {
      const uint32_t dst = smem_base + (uint32_t)s * p.stage_bytes + (uint32_t)i * tile_bytes;
      bulk_load(dst, p.codes + ((tile + i) * kb + b0) * 32, (uint32_t)nb * 512u, bar0 + 8u * s);
      bulk_load(dst + (uint32_t)p.slice * 512u, p.scales + ((tile + i) * groups + g0) * 8, (uint32_t)ng * 32u, bar0 + 8u * s);
    }
  };
  int next_pass = 0, next_batch = 0;  // of the next load
  auto load_next = [&](int s) {
    if (next_pass == p.passes) return;
    if (threadIdx.x == 0 && p.starve == 0) load(next_pass, next_batch, s);
    if (++next_batch == n_batches) {
      next_batch = 0;
      ++next_pass;
    }
  };
  if (threadIdx.x == 0) {
    abort_word = 0;
    for (int s = 0; s < kStages; ++s) mbar_init(bar0 + 8u * s, 1);
    fence_mbar_init_cluster();
  }
  for (int s = 0; s < p.stages; ++s) load_next(s);
  __syncthreads();

  float* const out = reinterpret_cast<float*>(smem + off_out);
  int s = 0;
  uint32_t phases = 0u;  // bit s: the parity of stage s
  bool ok = true;
  for (int pass = 0; ok && pass < p.passes; ++pass) {
    const int b0 = (pass * p.split + rank) * p.slice, nb = blocks(pass);
    // This warp's blocks are warp * kBlocks + i.  One beyond the slice has x = 0 and the weights of the slice's last block, so it adds
    // zeros (or the NaN that block gives anyway).
    uint4 xv[kBlocks][NT][2];
#pragma unroll
    for (int i = 0; i < kBlocks; ++i) {
      const int at = warp * kBlocks + i;
#pragma unroll
      for (int n = 0; n < NT; ++n) {
        // a token beyond the last repeats it: its column of the product is not stored, and columns do not mix
        const __nv_bfloat16* src = static_cast<const __nv_bfloat16*>(p.x) + (tok0 + min(8 * n + g, n_tok - 1)) * p.x_stride +
                                   (int64_t)mat * p.k + (int64_t)(b0 + at) * 64 + t * 8;
        xv[i][n][0] = xv[i][n][1] = make_uint4(0u, 0u, 0u, 0u);
        if (at < nb) {
          xv[i][n][0] = __ldg(reinterpret_cast<const uint4*>(src));
          xv[i][n][1] = __ldg(reinterpret_cast<const uint4*>(src + 32));
        }
      }
    }
#pragma unroll 1
    for (int batch = 0; batch < n_batches; ++batch) {
      uint8_t* const red = smem + off_red;
      if (nb > 0) ok = mbar_wait_bounded<false>(bar0 + 8u * s, (phases >> s) & 1u, p.wait_ns, abort_flag, p.status, 62, batch);
      ok = __all_sync(0xffffffffu, ok);
      const uint8_t* tile = smem + (uint32_t)s * p.stage_bytes;
      const int n = min(kBatch, n_tiles - batch * kBatch);
#pragma unroll 1
      for (int j = 0; j < n; ++j, tile += tile_bytes) {
        float acc[NT][4];
#pragma unroll
        for (int u = 0; u < NT; ++u) acc[u][0] = acc[u][1] = acc[u][2] = acc[u][3] = 0.f;
        if (ok && nb > 0) {
          const uint32_t* sc = reinterpret_cast<const uint32_t*>(tile + (uint32_t)p.slice * 512u) + g;
          float d[NT][4];
          auto add = [&](uint32_t sv) {
            const float lo = __uint_as_float(sv << 16), hi = __uint_as_float(sv & 0xffff0000u);
#pragma unroll
            for (int u = 0; u < NT; ++u) {
              acc[u][0] = fmaf(d[u][0], lo, acc[u][0]);
              acc[u][1] = fmaf(d[u][1], lo, acc[u][1]);
              acc[u][2] = fmaf(d[u][2], hi, acc[u][2]);
              acc[u][3] = fmaf(d[u][3], hi, acc[u][3]);
            }
          };
#pragma unroll
          for (int i = 0; i < kBlocks; ++i) {
            const int at = min(warp * kBlocks + i, nb - 1);
            const uint4 wv = *reinterpret_cast<const uint4*>(tile + at * 512 + lane * 16);
            const uint32_t words[4] = {wv.x, wv.y, wv.z, wv.w};
            // two blocks make a group of 128 where a warp has both; slices are even, so they are its blocks 0, 1 and 2, 3
            constexpr bool kPairs = kGroup == 128 && kBlocks > 1;
#pragma unroll
            for (int q = 0; q < 4; ++q) {
              uint32_t a[4];
              unpack_codes(words[q], a);
#pragma unroll
              for (int u = 0; u < NT; ++u) {
                const uint4 v = xv[i][u][q >> 1];
                const uint32_t x0 = (q & 1) ? v.z : v.x, x1 = (q & 1) ? v.w : v.y;
                if ((q == 0 && !(kPairs && (i & 1))) || (q == 2 && kGroup == 32)) mma_16816<true>(d[u], a, x0, x1);
                else mma_16816<false>(d[u], a, x0, x1);
              }
              if (q == 1 && kGroup == 32) add(sc[16 * at]);  // the first 32 of the block are a group of their own
            }
            if (!kPairs || (i & 1)) add(sc[8 * (kGroup == 32 ? 2 * at + 1 : kGroup == 64 ? at : at >> 1)]);
          }
        }
        if (j == 0 && batch + pass > 0) named_barrier_sync(2, kThreads);  // the last batch's sums have been read
#pragma unroll
        for (int u = 0; u < NT; ++u)
          *reinterpret_cast<float4*>(red + (warp * kUnits + j * NT + u) * kUnit + lane * 16) = make_float4(acc[u][0], acc[u][1], acc[u][2], acc[u][3]);
      }
      ok = named_barrier_and(1, kThreads, ok);  // a warp that gave up must not leave the others in a barrier
      if (!ok) break;
      load_next(s);  // everyone is done with this stage
      if (nb > 0) phases ^= 1u << s;
      if (++s == p.stages) s = 0;
      // sums over the warps, kUnits * 128 of them
      constexpr int kEach = kUnits * 128 / kThreads;
      const int u = (int)threadIdx.x * kEach / 128;
      if (u < n * NT) {
        float v[kEach];
#pragma unroll
        for (int e = 0; e < kEach; ++e) v[e] = 0.f;
        const float* src = reinterpret_cast<const float*>(red) + threadIdx.x * kEach;
#pragma unroll
        for (int k = 0; k < kWarps; ++k)
#pragma unroll
          for (int e = 0; e < kEach; ++e) v[e] += src[k * kUnits * (kUnit / 4) + e];
        float* dst = out + batch * kUnits * (kUnit / 4) + threadIdx.x * kEach;
#pragma unroll
        for (int e = 0; e < kEach; ++e) dst[e] = pass > 0 ? dst[e] + v[e] : v[e];
      }
    }
  }
  if (*abort_flag != 0) {  // a wait has run out: copies in flight get a bounded time to land before the block goes away
    for (int i = 0; i < 64; ++i) __nanosleep(1000);
  }
  auto join = [&]() {
    if (p.split > 1) {
      __syncwarp();
      cluster_arrive();
      cluster_wait();
    } else {
      __syncthreads();
    }
  };
  join();
  // A peer that gave up has reported it; its sums are garbage then, like every result of a call that failed.
  const int n_sums = n_tiles * NT * 128;
  for (int i = rank * kThreads + threadIdx.x; i < n_sums; i += p.split * kThreads) {
    // element e of lane (g, t) in a product: row g + 8 (e >> 1), token 2 t + (e & 1)
    const int row = i & 15, col = (i >> 4) & 7, at = i >> 7, n = at % NT;
    const uint32_t src = off_out + (uint32_t)(at * kUnit + ((row & 7) * 4 + (col >> 1)) * 16 + ((row >> 3) * 2 + (col & 1)) * 4);
    if (8 * n + col >= n_tok) continue;
    float v = 0.f;
    if (p.split > 1) {
      for (int r = 0; r < p.split; ++r) v += load_peer(mapa_shared(smem_base + src, (uint32_t)r));
    } else {
      v = *reinterpret_cast<const float*>(smem + src);
    }
    const int64_t o = (tok0 + 8 * n + col) * p.y_stride + (int64_t)mat * p.n_out + (tile0 + at / NT) * 16 + row;
    if (p.out_f32) static_cast<float*>(p.y)[o] = v;
    else static_cast<__nv_bfloat16*>(p.y)[o] = __float2bfloat16_rn(v);
  }
  if (p.split > 1) join();  // shared memory has to outlive the peers' reads
}

// ---- laying the weights out (once) ------------------------------------------------------------------------
// Scales: one thread per (matrix, row, group): s = bf16(max |w| / 7), NaN if a weight of the group is not finite.
__global__ void __launch_bounds__(256) quant4_scale_kernel(const __nv_bfloat16* __restrict__ w, int64_t n_rows, int32_t n_out, int32_t k,
                                                           int32_t group, __nv_bfloat16* __restrict__ scales) {
  const int groups = k / group;
  const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
  if (i >= n_rows * groups) return;
  const int64_t row = i / groups;
  const int gi = (int)(i - row * groups);
  const uint4* src = reinterpret_cast<const uint4*>(w + row * k + (int64_t)gi * group);
  uint32_t mx = 0u;
  for (int e = 0; e < group / 8; ++e) {
    const uint4 v = __ldg(src + e);
    mx = __vmaxu2(__vmaxu2(mx, v.x & 0x7fff7fffu), v.y & 0x7fff7fffu);
    mx = __vmaxu2(__vmaxu2(mx, v.z & 0x7fff7fffu), v.w & 0x7fff7fffu);
  }
  const uint32_t top = max(mx & 0xffffu, mx >> 16);
  const float s = top < 0x7f80u ? __fdiv_rn(__uint_as_float(top << 16), 7.0f) : NAN;
  const int64_t mat = row / n_out;
  const int r = (int)(row - mat * n_out);
  scales[((mat * (n_out >> 4) + (r >> 4)) * groups + gi) * 16 + (r & 7) * 2 + ((r >> 3) & 1)] = __float2bfloat16_rn(s);
}

__device__ __forceinline__ uint32_t quant4_code(uint32_t bits, float s) {
  // the division is exact to rounding, so a quotient on a tie is on it here too (12 bits against 24)
  const float q = s == 0.f ? 0.f : __fdiv_rn(__uint_as_float(bits << 16), s);
  return (uint32_t)(int)(rintf(fminf(fmaxf(q, -7.f), 7.f)) + 8.f);
}

// Codes: one thread per (matrix, row tile, block, lane).
__global__ void __launch_bounds__(256) quant4_code_kernel(const __nv_bfloat16* __restrict__ w, int64_t n_lanes, int32_t n_out, int32_t k,
                                                          int32_t group, const __nv_bfloat16* __restrict__ scales,
                                                          uint4* __restrict__ codes) {
  const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
  if (i >= n_lanes) return;
  const int kb = k >> 6, groups = k / group;
  const int lane = (int)(i & 31), g = lane >> 2, t = lane & 3;
  const int64_t tb = i >> 5;
  const int64_t tile = tb / kb;
  const int b = (int)(tb - tile * kb);
  const __nv_bfloat16* src = w + (tile * 16 + g) * (int64_t)k + b * 64 + 8 * t;
  uint32_t words[4];
#pragma unroll
  for (int half = 0; half < 2; ++half) {
    const int gi = (b * 64 + half * 32) / group;
    const float sa = __bfloat162float(scales[(tile * groups + gi) * 16 + g * 2]);
    const float sb = __bfloat162float(scales[(tile * groups + gi) * 16 + g * 2 + 1]);
    const uint4 va = __ldg(reinterpret_cast<const uint4*>(src + half * 32));
    const uint4 vb = __ldg(reinterpret_cast<const uint4*>(src + 8 * (int64_t)k + half * 32));
    const uint32_t xa[4] = {va.x, va.y, va.z, va.w}, xb[4] = {vb.x, vb.y, vb.z, vb.w};
#pragma unroll
    for (int s = 0; s < 2; ++s) {
      uint32_t v = 0u;
#pragma unroll
      for (int e = 0; e < 2; ++e) {  // A fragment registers: (row g, first pair), (row g + 8, first pair), then the second pair
        v |= quant4_code(xa[2 * s + e] & 0xffffu, sa) << (8 * e) | quant4_code(xa[2 * s + e] >> 16, sa) << (16 + 8 * e);
        v |= quant4_code(xb[2 * s + e] & 0xffffu, sb) << (8 * e + 4) | quant4_code(xb[2 * s + e] >> 16, sb) << (16 + 8 * e + 4);
      }
      words[2 * half + s] = v;
    }
  }
  codes[i] = make_uint4(words[0], words[1], words[2], words[3]);
}

}  // namespace

cudaError_t launch_quant4(const void* w, int32_t n_mat, int32_t n_out, int32_t k, int32_t group, void* codes, void* scales,
                          cudaStream_t stream) {
  const int64_t rows = (int64_t)n_mat * n_out, n_scale = rows * (k / group), n_lanes = rows / 16 * (k / 64) * 32;
  quant4_scale_kernel<<<(unsigned)((n_scale + 255) / 256), 256, 0, stream>>>(static_cast<const __nv_bfloat16*>(w), rows, n_out, k,
                                                                             group, static_cast<__nv_bfloat16*>(scales));
  cudaError_t e = cudaGetLastError();
  if (e != cudaSuccess) return e;
  quant4_code_kernel<<<(unsigned)((n_lanes + 255) / 256), 256, 0, stream>>>(static_cast<const __nv_bfloat16*>(w), n_lanes, n_out, k,
                                                                            group, static_cast<const __nv_bfloat16*>(scales),
                                                                            static_cast<uint4*>(codes));
  return cudaGetLastError();
}

namespace {
using Matvec4Kernel = void (*)(const Matvec4Params);
template <int NT, int kGroup>
Matvec4Kernel matvec4_pick(int blocks) {
  return blocks == 1 ? rk_matvec4_kernel<NT, kGroup, 1> : blocks == 2 ? rk_matvec4_kernel<NT, kGroup, 2> : rk_matvec4_kernel<NT, kGroup, 4>;
}
Matvec4Kernel matvec4_kernel(int nt, int group, int blocks) {
  if (nt == 1) return group == 32 ? matvec4_pick<1, 32>(blocks) : group == 64 ? matvec4_pick<1, 64>(blocks) : matvec4_pick<1, 128>(blocks);
  return group == 32 ? matvec4_pick<2, 32>(blocks) : group == 64 ? matvec4_pick<2, 64>(blocks) : matvec4_pick<2, 128>(blocks);
}
void matvec4_config(cudaLaunchConfig_t& cfg, cudaLaunchAttribute& attr, int split) {
  cfg.blockDim = dim3(kThreads);
  attr.id = cudaLaunchAttributeClusterDimension;
  attr.val.clusterDim.x = (unsigned)split;
  attr.val.clusterDim.y = attr.val.clusterDim.z = 1;
  cfg.attrs = &attr;
  cfg.numAttrs = split > 1 ? 1 : 0;
}
}  // namespace

cudaError_t matvec4_setup(int32_t* slots, int sm_count) {
  for (int nt = 1; nt <= 2; ++nt)
    for (int group = 32; group <= 128; group *= 2)
      for (int blocks = 1; blocks <= 4; blocks *= 2) {
        cudaError_t e = cudaFuncSetAttribute(matvec4_kernel(nt, group, blocks), cudaFuncAttributeMaxDynamicSharedMemorySize, kSmemBytes);
        if (e != cudaSuccess) return e;
      }
  slots[0] = 2 * sm_count;
  for (int i = 1; i < 4; ++i) {  // clusters of 1 << i thread blocks that run at the same time
    cudaLaunchConfig_t cfg = {};
    cudaLaunchAttribute attr = {};
    matvec4_config(cfg, attr, 1 << i);
    cfg.gridDim = dim3(1u << i);
    cfg.dynamicSmemBytes = kSmemBytes;
    int n = 0;
    cudaError_t e = cudaOccupancyMaxActiveClusters(&n, matvec4_kernel(2, 128, kMaxBlocks), &cfg);
    if (e != cudaSuccess) return e;
    slots[i] = n > 0 ? n : 1;
  }
  return cudaSuccess;
}

cudaError_t launch_matvec4(Matvec4Params p, const int32_t* slots, cudaStream_t stream) {
  const int tiles = p.n_out / 16, kb = p.k / 64, nt = p.n_tok <= 8 ? 1 : 2;
  const int64_t tok_blocks = (p.n_tok + 8 * nt - 1) / (8 * nt);
  // k goes over as many thread blocks as its slices of up to 2048 need, beyond eight in several passes
  int log_split = 0;
  while ((1 << log_split) < kMaxSplit && (kSliceBlocks << log_split) < kb) ++log_split;
  p.split = 1 << log_split;
  p.passes = (kb + kSliceBlocks * p.split - 1) / (kSliceBlocks * p.split);
  const int parts = p.split * p.passes;
  p.slice = ((kb + parts - 1) / parts + 1) & ~1;  // even: a group of 128 is two blocks
  const int blocks = p.slice <= kWarps ? 1 : p.slice <= 2 * kWarps ? 2 : kMaxBlocks;
  // tiles per thread block: one round of what fits the device, within the sums' space
  const int64_t all = (int64_t)p.n_mat * tiles * tok_blocks;
  int64_t run = (all + slots[log_split] - 1) / slots[log_split];
  if (run > kMaxRun / nt) run = kMaxRun / nt;
  if (run > tiles) run = tiles;
  p.runs = (tiles + (int)run - 1) / (int)run;
  p.run = (tiles + p.runs - 1) / p.runs;
  p.stage_bytes = (uint32_t)(kBatch * (p.slice * 512 + p.slice * 64 / p.group * 32));
  const int per_pass = (p.run + kBatch - 1) / kBatch, batches = p.passes * per_pass;
  p.red_bytes = (uint32_t)(kWarps * kBatch * nt * kUnit);
  p.stages = batches < kStages ? batches : kStages;
  cudaLaunchConfig_t cfg = {};
  cudaLaunchAttribute attr = {};
  matvec4_config(cfg, attr, p.split);
  cfg.gridDim = dim3((unsigned)((int64_t)p.n_mat * p.runs * p.split), (unsigned)tok_blocks);
  cfg.dynamicSmemBytes = p.stages * p.stage_bytes + p.red_bytes + (uint32_t)(per_pass * kBatch * nt * kUnit);
  cfg.stream = stream;
  return cudaLaunchKernelEx(&cfg, matvec4_kernel(nt, p.group, blocks), p);
}

}  // namespace rk
