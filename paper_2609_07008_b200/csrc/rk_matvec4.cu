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

constexpr int kWarps = 8;            // consumers; one more warp issues the copies
constexpr int kChunkBlocks = 16;     // 64-wide blocks of k per pipeline stage
constexpr uint32_t kTileBytes = kChunkBlocks * 512;        // codes of 16 output rows
constexpr uint32_t kTokBytes = kChunkBlocks * 128 + 64;    // x of one token; padded so that two rows fill the 32 banks
constexpr int kMaxStages = 4;

__device__ __forceinline__ void mma_16816(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
  asm(
      "mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
      : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
      : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}

__device__ __forceinline__ void unpack_codes(uint32_t v, uint32_t (&a)[4]) {
  const uint32_t k136 = 0x43084308u;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const uint32_t t = ((v >> (4 * i)) & 0x000f000fu) | 0x43004300u;
    const __nv_bfloat162 n = __hsub2(*reinterpret_cast<const __nv_bfloat162*>(&t), *reinterpret_cast<const __nv_bfloat162*>(&k136));
    a[i] = *reinterpret_cast<const uint32_t*>(&n);
  }
}

__device__ __forceinline__ void bulk_load(uint32_t dst, const void* src, uint32_t bytes, uint32_t bar) {
  asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];" ::"r"(dst), "l"(src),
               "r"(bytes), "r"(bar)
               : "memory");
}

// One block: RT tiles of 16 output rows, up to 8 * NT tokens.  Codes and x of 1024 k at a time come in by bulk copies, up
// to four stages ahead, which keeps tens of KB in flight per SM without holding them in registers (with plain loads in the
// consuming warps the copies of a warp were serialised by its products: 14.8 us instead of 5 for 17 MB).  The warps
// take the 64-wide blocks of a stage in turn and add their sums up in shared memory in warp order.
template <int RT, int NT>
__global__ void __launch_bounds__(kWarps * 32 + 32) rk_matvec4_kernel(const __grid_constant__ Matvec4Params p) {
  extern __shared__ __align__(128) uint8_t smem[];
  __shared__ float red[kWarps][RT * NT][128];
  __shared__ __align__(8) uint64_t bars[2 * kMaxStages];
  __shared__ int abort_word;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int g = lane >> 2, t = lane & 3;
  const int tiles = p.n_out >> 4, kb = p.k >> 6;
  const int per_mat = (tiles + RT - 1) / RT;
  const int mat = (int)(blockIdx.x / per_mat), tile0 = (int)(blockIdx.x % per_mat) * RT;
  const int64_t tok0 = (int64_t)blockIdx.y * 8 * NT;
  const int n_tok = (int)min((int64_t)8 * NT, p.n_tok - tok0);
  const int chunks = (kb + kChunkBlocks - 1) / kChunkBlocks;
  const uint32_t stage_bytes = RT * kTileBytes + (uint32_t)p.stage_toks * kTokBytes;
  const uint32_t smem_base = smem_u32(smem), bar0 = smem_u32(bars);
  auto full = [&](int s) -> uint32_t { return bar0 + 8u * s; };
  auto empty = [&](int s) -> uint32_t { return bar0 + 8u * (kMaxStages + s); };
  volatile int* abort_flag = &abort_word;
  if (threadIdx.x == 0) {
    abort_word = 0;
    for (int s = 0; s < p.stages; ++s) {
      mbar_init(full(s), 1);
      mbar_init(empty(s), kWarps);
    }
    fence_mbar_init_cluster();
  }
  __syncthreads();
  const int groups = p.k / p.group;
  float acc[RT][NT][4];
#pragma unroll
  for (int r = 0; r < RT; ++r)
#pragma unroll
    for (int n = 0; n < NT; ++n)
#pragma unroll
      for (int e = 0; e < 4; ++e) acc[r][n][e] = 0.f;

  if (warp == kWarps) {
    // ------------------------------ copies ------------------------------
    if (lane == 0) {
      const int n_t = min(RT, tiles - tile0);
      const uint4* w = p.codes + ((int64_t)mat * tiles + tile0) * kb * 32;
      const __nv_bfloat16* x = static_cast<const __nv_bfloat16*>(p.x) + tok0 * p.x_stride + (int64_t)mat * p.k;
      for (int c = 0, s = 0, phase = 0; c < chunks; ++c) {
        if (c >= p.stages &&
            !mbar_wait_bounded<false>(empty(s), (uint32_t)(phase ^ 1), p.wait_ns, abort_flag, p.status, 61, c))
          break;
        const int nb = min(kChunkBlocks, kb - c * kChunkBlocks);
        const uint32_t dst = smem_base + (uint32_t)s * stage_bytes;
        mbar_arrive_expect_tx(full(s), (uint32_t)(n_t * nb * 512 + n_tok * nb * 128));
        for (int r = 0; r < n_t; ++r)
          bulk_load(dst + r * kTileBytes, w + ((int64_t)r * kb + c * kChunkBlocks) * 32, (uint32_t)nb * 512u, full(s));
        for (int n = 0; n < n_tok; ++n)
          bulk_load(dst + RT * kTileBytes + n * kTokBytes, x + n * p.x_stride + c * kChunkBlocks * 64, (uint32_t)nb * 128u, full(s));
        if (++s == p.stages) {
          s = 0;
          phase ^= 1;
        }
      }
    }
  } else {
    // ------------------------------ products ------------------------------
    const bool g32 = p.group == 32;
    const int gshift = p.group == 128 ? 1 : 0;
    const uint32_t* sc[RT];
#pragma unroll
    for (int r = 0; r < RT; ++r)  // a tile beyond the last (odd counts) repeats the last one's scales; it is not stored
      sc[r] = p.scales + ((int64_t)mat * tiles + min(tile0 + r, tiles - 1)) * groups * 8 + g;
    bool ok = true;
    for (int c = 0, s = 0, phase = 0; c < chunks && ok; ++c) {
      // this warp's blocks of the stage: warp, warp + 8; their scales come straight from memory, ahead of the wait
      uint32_t s0[2][RT], s1[2][RT];
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const int b = c * kChunkBlocks + warp + 8 * i;
#pragma unroll
        for (int r = 0; r < RT; ++r) {
          s0[i][r] = s1[i][r] = 0u;
          if (b < kb) {
            s0[i][r] = __ldg(sc[r] + (g32 ? 2 * b : b >> gshift) * 8);
            if (g32) s1[i][r] = __ldg(sc[r] + (2 * b + 1) * 8);
          }
        }
      }
      ok = mbar_wait_bounded<false>(full(s), (uint32_t)phase, p.wait_ns, abort_flag, p.status, 62, c);
      if (!ok) break;
      const uint8_t* stage = smem + (uint32_t)s * stage_bytes;
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const int at = warp + 8 * i;
        if (c * kChunkBlocks + at >= kb) break;
        uint4 xv[NT][2];
#pragma unroll
        for (int n = 0; n < NT; ++n) {
          // a token beyond n_tok has whatever is there: its column of the product is not stored, and columns do not mix
          const int tok = min(8 * n + g, n_tok - 1);
          const uint8_t* xs = stage + RT * kTileBytes + tok * kTokBytes + at * 128 + t * 16;
          xv[n][0] = *reinterpret_cast<const uint4*>(xs);
          xv[n][1] = *reinterpret_cast<const uint4*>(xs + 64);
        }
#pragma unroll
        for (int r = 0; r < RT; ++r) {
          const uint4 wv = *reinterpret_cast<const uint4*>(stage + r * kTileBytes + at * 512 + lane * 16);
          float d[NT][4];
#pragma unroll
          for (int n = 0; n < NT; ++n)
#pragma unroll
            for (int e = 0; e < 4; ++e) d[n][e] = 0.f;
          const uint32_t words[4] = {wv.x, wv.y, wv.z, wv.w};
          auto add = [&](uint32_t sv) {
            const float lo = __uint_as_float(sv << 16), hi = __uint_as_float(sv & 0xffff0000u);
#pragma unroll
            for (int n = 0; n < NT; ++n) {
              acc[r][n][0] = fmaf(d[n][0], lo, acc[r][n][0]);
              acc[r][n][1] = fmaf(d[n][1], lo, acc[r][n][1]);
              acc[r][n][2] = fmaf(d[n][2], hi, acc[r][n][2]);
              acc[r][n][3] = fmaf(d[n][3], hi, acc[r][n][3]);
              d[n][0] = d[n][1] = d[n][2] = d[n][3] = 0.f;
            }
          };
#pragma unroll
          for (int q = 0; q < 4; ++q) {
            uint32_t a[4];
            unpack_codes(words[q], a);
#pragma unroll
            for (int n = 0; n < NT; ++n) {
              const uint4 v = xv[n][q >> 1];
              mma_16816(d[n], a, (q & 1) ? v.z : v.x, (q & 1) ? v.w : v.y);
            }
            if (q == 1 && g32) add(s0[i][r]);  // the first 32 of the block are a group of their own
          }
          add(g32 ? s1[i][r] : s0[i][r]);
        }
      }
      __syncwarp();
      if (lane == 0) mbar_arrive(empty(s));
      if (++s == p.stages) {
        s = 0;
        phase ^= 1;
      }
    }
    // accumulator e of lane (g, t): row g + 8 (e >> 1), token 2 t + (e & 1); stored as [token][row] of 8 x 16
#pragma unroll
    for (int r = 0; r < RT; ++r)
#pragma unroll
      for (int n = 0; n < NT; ++n)
#pragma unroll
        for (int e = 0; e < 4; ++e) red[warp][r * NT + n][(2 * t + (e & 1)) * 16 + g + 8 * (e >> 1)] = acc[r][n][e];
  }
  if (*abort_flag != 0) {  // a wait has run out: copies in flight get a bounded time to land before the block goes away
    for (int i = 0; i < 64; ++i) __nanosleep(1000);
  }
  __syncthreads();
  if (*abort_flag != 0) return;
  for (int i = threadIdx.x; i < RT * NT * 128; i += kWarps * 32 + 32) {
    const int rn = i >> 7, at = i & 127, r = rn / NT, n = rn - r * NT;
    float v = 0.f;
#pragma unroll
    for (int k = 0; k < kWarps; ++k) v += red[k][rn][at];
    const int64_t tok = tok0 + 8 * n + (at >> 4);
    const int tile = tile0 + r;
    if (tok >= p.n_tok || tile >= tiles) continue;
    const int64_t o = tok * p.y_stride + (int64_t)mat * p.n_out + tile * 16 + (at & 15);
    if (p.out_f32) static_cast<float*>(p.y)[o] = v;
    else static_cast<__nv_bfloat16*>(p.y)[o] = __float2bfloat16_rn(v);
  }
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

cudaError_t matvec4_setup() {
  cudaError_t e = cudaFuncSetAttribute(rk_matvec4_kernel<1, 1>, cudaFuncAttributeMaxDynamicSharedMemorySize, kMaxStages * (int)(kTileBytes + 8 * kTokBytes));
  if (e == cudaSuccess)
    e = cudaFuncSetAttribute(rk_matvec4_kernel<2, 2>, cudaFuncAttributeMaxDynamicSharedMemorySize, kMaxStages * (int)(2 * kTileBytes + 16 * kTokBytes));
  return e;
}

cudaError_t launch_matvec4(Matvec4Params p, cudaStream_t stream) {
  const int tiles = p.n_out / 16, chunks = (p.k / 64 + kChunkBlocks - 1) / kChunkBlocks;
  p.stages = chunks < kMaxStages ? chunks : kMaxStages;
  // up to eight tokens one tile per block; above that x weighs as much as the codes, and two tiles share it
  if (p.n_tok <= 8) {
    p.stage_toks = (int32_t)p.n_tok;
    rk_matvec4_kernel<1, 1><<<dim3((unsigned)(p.n_mat * tiles), 1), kWarps * 32 + 32, p.stages * (kTileBytes + p.stage_toks * kTokBytes), stream>>>(p);
  } else {
    p.stage_toks = (int32_t)(p.n_tok < 16 ? p.n_tok : 16);
    rk_matvec4_kernel<2, 2><<<dim3((unsigned)(p.n_mat * ((tiles + 1) / 2)), (unsigned)((p.n_tok + 15) / 16)), kWarps * 32 + 32,
                              p.stages * (2 * kTileBytes + p.stage_toks * kTokBytes), stream>>>(p);
  }
  return cudaGetLastError();
}

}  // namespace rk
