// Products in 8-bit integers: y[t][o] = sx[t] sw[o] sum_j X[t][j] W[o][j], codes X, W in -127 .. 127, scales in fp32.
//
// Rows (of weights and of tokens alike) are quantised by themselves: scale = fp32(max|x| / 127), code = x / scale rounded
// half to even.  The sums are exact (int32; k <= 131072 keeps |sum| < 2^31) and meet the scales once, in fp32, in the
// epilogue; rounding to bf16, where asked for, is the last step.
//
// rk_matmul8_pair_kernel: a pair of CTAs (cta_group::2) owns 256 output channels x up to 256 token rows.  The channels
// are the rows of the accumulator (M = 256) and the tokens its columns, because the number of tokens is what varies:
// N follows the rows that a tile really has, in steps of 32, down to the one or two rows an expert gets in a decode step.
// Each CTA streams its 128 channels of W and its half of the token rows in 128-byte steps of k (16 + up to 16 KB per
// stage); with N = 256 an SM draws 64 bytes per clock from L2 at the full rate of the tensor cores, below the 76 that it
// can.  Persistent: the accumulator is double buffered in tensor memory, so that the scales and stores of one tile run under
// the products of the next.  Where there are few tiles they are made smaller, or 2 or 4 pairs in a cluster share k and add
// their sums through each other's shared memory (rk_matmul8_plan; 256 x 4096 x 8192: 20.6 -> 15.4 us).
//   8192 tokens x 7168 channels x 16384: 580 to 605 us in a captured loop of ten, 3.2 to 3.3 POP/s, 0.93 to 0.97 of twice the
//   bf16 library product's measured burst rate: bounded by the tensor cores.  Called one by one for longer, with its
//   quantisation (73 us), it is 780 to 810 us, about 2.7 POP/s in the product: the rate under the power limit.
//   5 x 4096 x 8192: 11.3 us in such a loop, W's 33.6 MB in L2; 20.5 us with cold caches, of which those bytes cost 5.2 at the
//   memory's measured rate and the rest is launch, setup, first trips to memory, the join and the stores.
//
// By expert, the token rows of a tile are a gather (the tokens that chose the expert): six or seven warps, one per stage,
// copy them with 16-byte asynchronous loads into the swizzled operand layout, so that no sorted copy of the activations is made; the
// outputs go straight to the pairs' rows of y.  (TMA's gather of four rows took 72 clocks of each SM's copy engine per
// instruction, 2300 per 128 rows; a stage has 512.)
//   64 tokens, all weights used once: 143 us, 0.98 of the measured copy rate.  8192 tokens: 313 to 324 us in a captured loop of
//   ten, 291 by itself; of 313 (by removal) the gather costs 30, the first bytes of each expert's weights out of memory 62, the stores 28.
#include <cuda_bf16.h>

#include "rk_internal.h"

namespace rk {
namespace {

// ------------------------------------------------------------------------------------------------------------
// quantisation of rows
// ------------------------------------------------------------------------------------------------------------
constexpr int kQuantHeld = 4;  // 8-value chunks that a thread keeps in registers between the maximum and the codes
constexpr int kQuantRows = 8;  // rows of a thread block where a warp has a row to itself

constexpr float kQuantNear = 0.49997f;  // quotients (off by less than 1e-5) this far from a whole number are looked at again

// round(x / scale), half to even, exactly, and limited to -127 .. 127.  The quick quotient t tells the two codes; the sign of
// |x| - scale (m + 1/2), one fused product in double that is rounded once, the side of the middle between them.  Where 1 / scale
// is beyond fp32 (inv = 0), the quotient is taken in double.
__device__ __forceinline__ int quant8_code(float x, float scale, float inv) {
  const double a = fabs((double)x), m = inv == 0.f ? floor(a / (double)scale) : (double)floorf(fabsf(x * inv));
  const double r = fma(-(double)scale, m + 0.5, a);
  int c = (int)fmin(m, 127.0);
  if (c < 127 && (r > 0.0 || (r == 0.0 && (c & 1)))) ++c;
  return x < 0.f ? -c : c;
}

template <bool kVec>
__device__ __forceinline__ uint4 load_chunk(const __nv_bfloat16* row, int at, int k) {
  if constexpr (kVec) {
    if (at + 8 <= k) return __ldcs(reinterpret_cast<const uint4*>(row + at));
  }
  uint32_t v[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const uint32_t lo = at + 2 * i < k ? (uint32_t)__bfloat16_as_ushort(row[at + 2 * i]) : 0u;
    const uint32_t hi = at + 2 * i + 1 < k ? (uint32_t)__bfloat16_as_ushort(row[at + 2 * i + 1]) : 0u;
    v[i] = lo | (hi << 16);
  }
  return make_uint4(v[0], v[1], v[2], v[3]);
}
// the largest magnitude of eight bf16 values, as its 15 bits (an order of magnitudes: infinities and NaN come last)
__device__ __forceinline__ uint32_t chunk_top(const uint4& c) {
  uint32_t t = __vmaxu2(__vmaxu2(c.x & 0x7fff7fffu, c.y & 0x7fff7fffu), __vmaxu2(c.z & 0x7fff7fffu, c.w & 0x7fff7fffu));
  return max(t & 0xffffu, t >> 16);
}
// Codes of eight values.  x * inv + 1.5 * 2^23 is rounded to a whole number, half to even, whose two's complement is in the
// low byte.  `off` collects the largest |x - scale code|: the fused product is exact (a multiple of the last bit of scale, or x
// itself), so that the code is right below scale / 2.  inv is off by 2^-24 of itself, and a few values in 10^6 are found wrong.
__device__ __forceinline__ uint2 chunk_codes(const uint4& c, float scale, float inv, float& off) {
  constexpr float kMagic = 12582912.f;
  const uint32_t w[4] = {c.x, c.y, c.z, c.w};
  uint32_t y[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const float x = __uint_as_float(i & 1 ? w[i >> 1] & 0xffff0000u : w[i >> 1] << 16), r = fmaf(x, inv, kMagic);
    off = fmaxf(off, fabsf(fmaf(-scale, r - kMagic, x)));
    y[i] = __float_as_uint(r);
  }
  return make_uint2(__byte_perm(__byte_perm(y[0], y[1], 0x0040), __byte_perm(y[2], y[3], 0x0040), 0x5410),
                    __byte_perm(__byte_perm(y[4], y[5], 0x0040), __byte_perm(y[6], y[7], 0x0040), 0x5410));
}

// The values near the middle between two codes again (all values for inv = 0) of the threads `who` of the warp, each of which
// has the chunks thread, thread + step, ... of n_chunks.  A few threads' values are spread over the lanes, a thread's 32 at a
// time (2 us less than its walk over them); many threads walk side by side.
template <bool kVec>
__device__ __noinline__ void quant8_exact(unsigned who, const __nv_bfloat16* row, int k, int warp_first, int step, int n_chunks,
                                          float scale, float inv, uint8_t* codes) {
  const int lane = threadIdx.x & 31;
  auto fix = [&](int i, float x) {
    const float t = x * inv;
    if (inv == 0.f || fabsf(t - rintf(t)) >= kQuantNear) codes[i] = (uint8_t)quant8_code(x, scale, inv);
  };
  __syncwarp();
  if (__popc(who) <= 4) {
    for (; who != 0u; who &= who - 1u)
      for (int c = warp_first + __ffs(who) - 1 + (lane >> 3) * step; c < n_chunks; c += 4 * step) {
        const int i = 8 * c + (lane & 7);
        if (i < k) fix(i, __bfloat162float(row[i]));
      }
  } else if ((who >> lane) & 1u) {
    for (int c = warp_first + lane; c < n_chunks; c += step) {
      const uint4 v = load_chunk<kVec>(row, 8 * c, k);
#pragma unroll 1
      for (int i = 0; i < 8; ++i) {
        const uint32_t w = i < 4 ? (i < 2 ? v.x : v.y) : (i < 6 ? v.z : v.w);
        fix(8 * c + i, __uint_as_float(i & 1 ? w & 0xffff0000u : w << 16));
      }
    }
  }
}

// A row per thread block, or per warp (kWarp: up to 1024 values).  A row of up to 32 values per thread is read once; longer
// ones a second time out of L2.  Two bytes in, one out per value, 17
// instructions: 8192 x 16384 takes 73 to 83 us (by the data: rows with codes to correct), 0.75 to 0.85 of the copy rate; issue
// slots are 76% busy.
template <bool kVec, bool kWarp>
__global__ void __launch_bounds__(512, 3) quant8_kernel(const __nv_bfloat16* __restrict__ x, int64_t x_stride, int64_t n_rows, int k,
                                                        int k_pad, uint8_t* __restrict__ codes, float* __restrict__ scales) {
  const int64_t row = kWarp ? (int64_t)blockIdx.x * kQuantRows + (threadIdx.x >> 5) : blockIdx.x;
  if (kWarp && row >= n_rows) return;
  const __nv_bfloat16* src = x + row * x_stride;
  const int n_chunks = k_pad >> 3, nt = kWarp ? 32 : blockDim.x, tid = kWarp ? threadIdx.x & 31 : threadIdx.x;  // k_pad is a multiple of 16
  uint4 held[kQuantHeld];
  uint32_t top = 0u;
#pragma unroll
  for (int i = 0; i < kQuantHeld; ++i) {
    const int c = tid + i * nt;
    held[i] = c < n_chunks ? load_chunk<kVec>(src, 8 * c, k) : make_uint4(0u, 0u, 0u, 0u);
  }
#pragma unroll
  for (int i = 0; i < kQuantHeld; ++i) top = max(top, chunk_top(held[i]));
  for (int c = tid + kQuantHeld * nt; c < n_chunks; c += nt) top = max(top, chunk_top(load_chunk<kVec>(src, 8 * c, k)));
  top = __reduce_max_sync(0xffffffffu, top);
  if constexpr (!kWarp) {
    __shared__ uint32_t tops[16];
    if ((tid & 31) == 0) tops[tid >> 5] = top;
    __syncthreads();
    for (int w = 0; w < nt >> 5; ++w) top = max(top, tops[w]);
  }
  const bool finite = top < 0x7f80u;
  const float scale = finite ? __fdiv_rn(__uint_as_float(top << 16), 127.f) : __uint_as_float(0x7fc00000u);
  const bool blank = !finite || scale == 0.f;
  // 0 in place of the reciprocal makes codes of 0, and, for rows of tiny values, has all of them done exactly
  const float inv = blank || scale < 1e-30f ? 0.f : __fdiv_rn(1.f, scale);
  float off = !blank && inv == 0.f ? __int_as_float(0x7f800000) : 0.f;
  uint8_t* to = codes + row * k_pad;
  uint2* dst = reinterpret_cast<uint2*>(to);
#pragma unroll
  for (int i = 0; i < kQuantHeld; ++i) {
    const int c = tid + i * nt;
    if (c < n_chunks) dst[c] = finite ? chunk_codes(held[i], scale, inv, off) : make_uint2(0u, 0u);
  }
  for (int c = tid + kQuantHeld * nt; c < n_chunks; c += nt)
    dst[c] = finite ? chunk_codes(load_chunk<kVec>(src, 8 * c, k), scale, inv, off) : make_uint2(0u, 0u);
  // (with a power of two for a scale, one row in 128, the quick quotient is the quotient, and ties are many)
  const unsigned near = __ballot_sync(0xffffffffu, !blank && off >= 0.5f * scale && (inv == 0.f || (__float_as_uint(scale) & 0x7fffffu) != 0u));
  if (near != 0u) quant8_exact<kVec>(near, src, k, tid & ~31, nt, n_chunks, scale, inv, to);
  if (tid == 0) scales[row] = scale;
}

// ------------------------------------------------------------------------------------------------------------
// products
// ------------------------------------------------------------------------------------------------------------
constexpr int kThreads8 = 384;          // warp 0 loads, warp 1 issues, warps 4-11 scale and store
constexpr int kStages8 = 6;
constexpr int kStep = 128;      // bytes (= values) of k per stage
constexpr int kTileM = 256, kTileN = 256;
constexpr int kTileNFew = 192;  // by expert, few rows: smaller tiles leave room for a seventh stage
constexpr int kMaxStages8 = 7;
__host__ __device__ constexpr int stages8(bool few) { return few ? kMaxStages8 : kStages8; }
// by expert, warps 12 and up, and 2 and 3, gather token rows: one for each stage of the ring
__host__ __device__ constexpr int threads8(bool experts, bool few) { return kThreads8 + (experts ? 32 * (stages8(few) - 2) : 0); }
constexpr int kBandTok = 8;     // token tiles of a band: W streams past them together

struct Smem8 {
  static constexpr uint32_t kABytes = 128 * kStep, kBBytes = 128 * kStep;
  static constexpr uint32_t kOffBars = kMaxStages8 * (kABytes + kTileNFew / 2 * kStep);  // (the larger one of the rings)
  // full[stages], empty[stages], acc_full[2], acc_empty[2]
  static constexpr uint32_t kOffTmemPtr = kOffBars + (2 * kMaxStages8 + 4) * 8;
  static constexpr uint32_t kOffAbort = kOffTmemPtr + 8;
  static constexpr uint32_t kOffScan = kOffAbort + 8;               // by expert: a sum per warp, of the block's scan
  static constexpr int kMaxWarps = threads8(true, true) / 32;
  static constexpr uint32_t kOffTok = (kOffScan + 8 * kMaxWarps + 15) / 16 * 16;  // [2][256] TokenOut
  static constexpr uint32_t kOffFirst = kOffTok + 2 * 256 * 16;     // by expert: first tile of each, [n_mat + 1]; then row_off
  static constexpr uint32_t kBytes = kOffFirst + 2 * (kMaxExperts + 1) * 4 + 1024 + 16;
};
static_assert(Smem8::kBytes <= 227 * 1024, "shared memory");
enum { WM_EMPTY = 61, WM_FULL, WM_ACC_EMPTY, WM_ACC_FULL };

// D[tmem] (+)= A B^T in int8 -> int32, both operands in shared memory, by a CTA pair
__device__ __forceinline__ void umma_i8_pair(uint32_t tmem_d, uint64_t desc_a, uint64_t desc_b, uint32_t idesc, uint32_t accumulate) {
  asm volatile(
      "{\n\t.reg .pred p;\n\t"
      "setp.ne.b32 p, %4, 0;\n\t"
      "tcgen05.mma.cta_group::2.kind::i8 [%0], %1, %2, %3, p;\n\t}" ::"r"(tmem_d),
      "l"(desc_a), "l"(desc_b), "r"(idesc), "r"(accumulate)
      : "memory");
}
// signed 8-bit operands, both K-major, int32 sums
__device__ __forceinline__ uint32_t umma_idesc_i8(int m, int n) {
  return (2u << 4) | (1u << 7) | (1u << 10) | ((uint32_t)(n >> 3) << 17) | ((uint32_t)(m >> 4) << 24);
}
// 16 bytes from global to shared memory, or 16 zeros
__device__ __forceinline__ void copy16_async(uint32_t dst, const void* src, bool real) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(real ? 16 : 0) : "memory");
}
__device__ __forceinline__ void copies_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N>
__device__ __forceinline__ void copies_wait() {
  asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory");
}

// token rows are cut into as few tiles as they need, of equal size (a multiple of 32): a short rest would cost nearly a full
// tile's loads of W
__device__ __forceinline__ int token_tiles(int n, int most) { return (n + most - 1) / most; }
__device__ __forceinline__ int token_tile_rows(int n, int tiles) { return ((n + tiles - 1) / tiles + 31) & ~31; }

struct Tile8 {
  int mat, chan, tok, n;  // matrix, first channel, first token row (by expert: place in the list), token rows
};

struct __align__(16) TokenOut {  // an output row of a tile
  long long at;  // bytes from y, negative: not stored
  float scale;
  int pad;
};

// 32 columns of the accumulator: lane = channel, register i = token i.  `to` is y at the lane's channel.
template <class T>
__device__ __forceinline__ void store_columns(const uint32_t (&o)[32], const TokenOut* tok, uint8_t* to, float sw, bool mine) {
#pragma unroll
  for (int i = 0; i < 32; ++i) {
    const int4 raw = *reinterpret_cast<const int4*>(tok + i);
    const long long at = ((long long)raw.y << 32) | (uint32_t)raw.x;
    const float v = (float)(int)o[i] * __int_as_float(raw.z) * sw;
    if (mine && raw.y >= 0) {
      if constexpr (sizeof(T) == 4)
        *reinterpret_cast<float*>(to + at) = v;
      else
        *reinterpret_cast<__nv_bfloat16*>(to + at) = __float2bfloat16_rn(v);
    }
  }
}
// The same for bf16 where rows and channels allow 4-byte stores: neighbouring lanes trade one of two tokens, after which the
// even lane has both channels of the first and the odd lane both of the second.  `to` is y at the even lane's channel.
__device__ __forceinline__ void store_columns_paired(const uint32_t (&o)[32], const TokenOut* tok, uint8_t* to, float sw, bool mine) {
  const bool odd = threadIdx.x & 1;
#pragma unroll
  for (int i = 0; i < 32; i += 2) {
    const int4 a = *reinterpret_cast<const int4*>(tok + i), b = *reinterpret_cast<const int4*>(tok + i + 1);
    const float va = (float)(int)o[i] * __int_as_float(a.z) * sw, vb = (float)(int)o[i + 1] * __int_as_float(b.z) * sw;
    const float got = __shfl_xor_sync(0xffffffffu, odd ? va : vb, 1);
    const int hi = odd ? b.y : a.y;
    const long long at = ((long long)hi << 32) | (uint32_t)(odd ? b.x : a.x);
    const uint32_t v = odd ? pack_bf16(got, vb) : pack_bf16(va, got);
    if (mine && hi >= 0) *reinterpret_cast<uint32_t*>(to + at) = v;
  }
}

// kSplit > 1: that many pairs of a cluster share the k of one tile (a cluster has one tile then), and a CTA joins the sums of its
// share of the token columns out of the others' shared memory.
// kFew (by expert): tiles of up to 192 token rows in a ring of seven stages, in place of 256 and six.
template <bool kExperts, bool kFew, int kSplit>
__global__ void __launch_bounds__(threads8(kExperts, kFew), 1) rk_matmul8_pair_kernel(const __grid_constant__ Matmul8Params p) {
  using S = Smem8;
  constexpr int kStages = stages8(kFew), kMost = kFew ? kTileNFew : kTileN;
  const int most = kExperts ? kMost : p.tile_rows;  // token rows of a tile
  constexpr uint32_t kStageBytes = S::kABytes + (uint32_t)(kMost / 2 * kStep);
  static_assert(kStages * kStageBytes <= S::kOffBars, "ring");
  static_assert(!kExperts || S::kOffScan + 8 * (threads8(kExperts, kFew) / 32) <= S::kOffTok, "scan");
  extern __shared__ uint8_t smem_raw[];
  const uint32_t smem_base = (smem_u32(smem_raw) + 1023u) & ~1023u;
  uint8_t* smem = smem_raw + (smem_base - smem_u32(smem_raw));
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const uint32_t cluster_rank = cluster_ctarank(), crank = cluster_rank & 1u, lead = cluster_rank & ~1u;  // place in the pair; the pair's leader
  const int pair = (int)blockIdx.x / (2 * kSplit), n_pairs = (int)gridDim.x / (2 * kSplit);
  auto full_bar = [&](int s) -> uint32_t { return smem_base + S::kOffBars + 8u * s; };
  auto empty_bar = [&](int s) -> uint32_t { return smem_base + S::kOffBars + 8u * (kStages + s); };
  auto acc_full_bar = [&](int b) -> uint32_t { return smem_base + S::kOffBars + 8u * (2 * kStages + b); };
  auto acc_empty_bar = [&](int b) -> uint32_t { return smem_base + S::kOffBars + 8u * (2 * kStages + 2 + b); };
  volatile int* abort_flag = reinterpret_cast<volatile int*>(smem + S::kOffAbort);
  volatile uint32_t* tmem_ptr_smem = reinterpret_cast<volatile uint32_t*>(smem + S::kOffTmemPtr);
  int* first = reinterpret_cast<int*>(smem + S::kOffFirst);
  int* offs = first + kMaxExperts + 1;
  const uint64_t limit = p.wait_ns;
  const int n_chan = (p.n_out + kTileM - 1) / kTileM;
  const int all_chunks = (p.k_pad + kStep - 1) / kStep;
  const int k_first = kSplit > 1 ? all_chunks * (int)(cluster_rank >> 1) / kSplit : 0;  // in steps of k
  const int k_chunks = kSplit > 1 ? all_chunks * (int)((cluster_rank >> 1) + 1) / kSplit - k_first : all_chunks;

  if (threadIdx.x == 0) {
    *abort_flag = 0;
    for (int s = 0; s < kStages; ++s) {
      // leader's: one arrival (its own expect_tx) + the bytes of both CTAs, and both CTAs' gather warp of the stage
      mbar_init(full_bar(s), kExperts ? 1 + 2 : 1);
      mbar_init(empty_bar(s), 1);  // each CTA's: the pair's commit arrives on both
    }
    for (int b = 0; b < 2; ++b) {
      mbar_init(acc_full_bar(b), 1);    // each CTA's: the pair's commit arrives on both
      mbar_init(acc_empty_bar(b), 16);  // leader's: the eight epilogue warps of both CTAs
    }
    fence_mbar_init_cluster();
  }
  if (warp == 0) {
    __syncwarp();
    tmem_alloc<2>(smem_base + S::kOffTmemPtr, 512);
    tmem_relinquish<2>();
  }
  int n_tiles;
  if constexpr (kExperts) {
    // the list's bounds, made safe: an expert's rows lie inside the list and behind the previous expert's
    long long* scan = reinterpret_cast<long long*>(smem + S::kOffScan);
    for (int e = threadIdx.x; e <= p.n_mat; e += blockDim.x) offs[e] = p.row_off[e];
    __syncthreads();
    long long base = 0;
    for (int e0 = 0; e0 < p.n_mat; e0 += blockDim.x) {
      const int e = e0 + (int)threadIdx.x;
      long long tiles = 0;
      if (e < p.n_mat) {
        const int lo = offs[e], hi = offs[e + 1];
        if (lo >= 0 && lo <= hi && hi <= p.n_tok)
          tiles = (long long)token_tiles(hi - lo, kMost) * n_chan;
        else if (blockIdx.x == 0)
          report_status(p.status, 4 /*RK_ERR_ROWS*/, RK_CHK_EXPERT_OFF, e);
      }
      long long sum = tiles;
      for (int d = 1; d < 32; d <<= 1) {
        const long long v = __shfl_up_sync(0xffffffffu, sum, d);
        if (lane >= d) sum += v;
      }
      if (lane == 31) scan[warp] = sum;
      __syncthreads();
      long long before = base;
      for (int w = 0; w < (int)blockDim.x / 32; ++w) {
        if (w < warp) before += scan[w];
        base += scan[w];
      }
      if (e < p.n_mat) first[e] = (int)(before + sum - tiles);
      __syncthreads();
    }
    if (threadIdx.x == 0) first[p.n_mat] = (int)base;
    // bounds that fall and rise again may name more rows than the list has; what 32 bits cannot count is left alone
    n_tiles = base <= (1 << 30) ? (int)base : 0;
    if (base > (1 << 30) && blockIdx.x == 0 && threadIdx.x == 0) report_status(p.status, 4 /*RK_ERR_ROWS*/, RK_CHK_EXPERT_OFF, p.n_mat);
  } else {
    n_tiles = n_chan * token_tiles(p.n_tok, most);
  }
  // Tile t of the pair's sequence.  `e` walks up the experts as t grows.
  auto tile_at = [&](int t, int& e) -> Tile8 {
    Tile8 r;
    if constexpr (kExperts) {
      while (t >= first[e + 1]) ++e;
      const int i = t - first[e], tt = i / n_chan;
      const int n = offs[e + 1] - offs[e], rows = token_tile_rows(n, token_tiles(n, kMost));
      r.mat = e;
      r.chan = (i - tt * n_chan) * kTileM;
      r.tok = offs[e] + tt * rows;
      r.n = min(rows, offs[e + 1] - r.tok);
    } else {
      const int n_tok_tiles = token_tiles(p.n_tok, most), rows = token_tile_rows(p.n_tok, n_tok_tiles), per_band = kBandTok * n_chan;
      const int band = t / per_band, here = min(kBandTok, n_tok_tiles - band * kBandTok), rem = t - band * per_band;
      const int cb = rem / here;
      r.mat = 0;
      r.chan = cb * kTileM;
      r.tok = (band * kBandTok + rem - cb * here) * rows;
      r.n = min(rows, p.n_tok - r.tok);
    }
    return r;
  };
  tc_fence_before_sync();
  __syncthreads();
  __syncwarp();
  cluster_arrive();
  cluster_wait();
  tc_fence_after_sync();
  const uint32_t tmem_base = *tmem_ptr_smem;

  if (warp == 0) {
    // ---- loads: this CTA's 128 channels and its half of the token rows; bytes are counted on the leader's barrier ----
    if (lane == 0) {
      tma_prefetch_desc(&p.tm_w);
      if (!kExperts) tma_prefetch_desc(&p.tm_x);
    }
    uint32_t it = 0, s = 0, turn = 0;  // uses of stages; the stage of this one, and its place among the stage's uses (mod 2)
    int e = 0;
    bool ok = true;
    const uint32_t bytes = 2u * (S::kABytes + (kExperts ? 0u : (uint32_t)(most / 2 * kStep)));
    const uint64_t once_policy = l2_policy_evict_first();  // (64 tokens: 149 -> 142 us)
    for (int t = pair; t < n_tiles && ok; t += n_pairs) {
      const Tile8 tile = tile_at(t, e);
      const int half = ((tile.n + 31) >> 5) << 4;  // token rows of this CTA, a multiple of 16
      const int w_row = tile.mat * p.n_out + tile.chan + (int)crank * 128;
      const bool once = kExperts && offs[tile.mat + 1] - offs[tile.mat] == tile.n;  // no other tile reads these weights
      for (int kc = 0; kc < k_chunks && ok; ++kc, ++it) {
        if (it >= (uint32_t)kStages) ok = mbar_wait_bounded<false>(empty_bar(s), turn ^ 1u, limit, abort_flag, p.status, WM_EMPTY, t);
        ok = __all_sync(0xffffffffu, ok);
        if (!ok) break;
        const uint32_t full_remote = mapa_shared(full_bar(s), lead);
        const uint32_t a_dst = smem_base + s * kStageBytes;
        if (elect_one()) {
          if (crank == 0) mbar_arrive_expect_tx(full_bar(s), bytes);
          if (!p.starve) {  // (the timeout tests: announced and never sent)
            if (once)
              tma_load_2d_pair_hint(a_dst, &p.tm_w, full_remote, (k_first + kc) * kStep, w_row, once_policy);
            else
              tma_load_2d_pair(a_dst, &p.tm_w, full_remote, (k_first + kc) * kStep, w_row);
          }
          if constexpr (!kExperts) tma_load_2d_pair(a_dst + S::kABytes, &p.tm_x, full_remote, (k_first + kc) * kStep, tile.tok + (int)crank * half);
        }
        __syncwarp();
        if (++s == (uint32_t)kStages) {
          s = 0;
          turn ^= 1u;
        }
      }
    }
    for (uint32_t back = 1; back <= (uint32_t)kStages && ok; ++back) {
      if (it >= back) {
        const uint32_t u = it - back;
        ok = mbar_wait_bounded<false>(empty_bar(u % kStages), (u / kStages) & 1u, limit, abort_flag, p.status, WM_EMPTY, -1);
        ok = __all_sync(0xffffffffu, ok);
      }
    }
  } else if (warp == 1) {
    // ---- products (leader CTA only) ----
    if (crank == 0) {
      uint32_t s = 0, turn = 0, tile_i = 0;
      int e = 0;
      bool ok = true;
      for (int t = pair; t < n_tiles && ok; t += n_pairs, ++tile_i) {
        const Tile8 tile = tile_at(t, e);
        const uint32_t idesc = umma_idesc_i8(kTileM, ((tile.n + 31) >> 5) << 5);
        const uint32_t b = tile_i & 1u;
        if (tile_i >= 2) {
          ok = mbar_wait_bounded<true>(acc_empty_bar(b), ((tile_i >> 1) & 1u) ^ 1u, limit, abort_flag, p.status, WM_ACC_EMPTY, t);
          ok = __all_sync(0xffffffffu, ok);
          if (!ok) break;
          tc_fence_after_sync();
        }
        const uint32_t acc = tmem_base + b * kTileN;
        for (int kc = 0; kc < k_chunks && ok; ++kc) {
          ok = mbar_wait_bounded<false>(full_bar(s), turn, limit, abort_flag, p.status, WM_FULL, t);
          ok = __all_sync(0xffffffffu, ok);
          if (!ok) break;
          const uint32_t a_addr = smem_base + s * kStageBytes;
          if (elect_one()) {
            const uint64_t da = umma_desc_sw128(a_addr, 16, 1024), db = umma_desc_sw128(a_addr + S::kABytes, 16, 1024);
#pragma unroll
            for (int k = 0; k < 4; ++k)
              umma_i8_pair(acc, da + (uint64_t)(2 * k), db + (uint64_t)(2 * k), idesc, (kc > 0 || k > 0) ? 1u : 0u);
            umma_commit_2_mc(empty_bar(s), (uint16_t)(3u << lead));
            if (kc == k_chunks - 1) umma_commit_2_mc(acc_full_bar(b), (uint16_t)(3u << lead));
          }
          __syncwarp();
          if (++s == (uint32_t)kStages) {
            s = 0;
            turn ^= 1u;
          }
        }
      }
    }
  } else if (kExperts && (warp >= 12 || warp == 2 || warp == 3)) {
    // ---- gather (by expert): a warp fills one stage of the ring over and over, so that all of them may be under way.  Four rows
    // per instruction, eight lanes to a row of 128 bytes ----
    const uint32_t s = warp >= 12 ? warp - 12 : warp + kStages - 4;
    const int sub = lane >> 3, chunk = lane & 7;
    const uint32_t dst = smem_base + s * kStageBytes + S::kABytes;
    const uint32_t full_remote = mapa_shared(full_bar(s), lead);
    int e = 0, t = pair, known = -1, half = 0, kc = (int)s;
    uint32_t from[kMost / 8];  // this lane's rows of the half, in units of 16 bytes from x
    for (uint32_t use = 0;; ++use, kc += kStages) {
      for (; kc >= k_chunks; kc -= k_chunks) t += n_pairs;
      if (t >= n_tiles) break;
      if (t != known) {
        const Tile8 tile = tile_at(t, e);
        known = t;
        half = ((tile.n + 31) >> 5) << 4;
        uint32_t row[(kMost + 63) / 64];  // lane l has rows l, l + 32, ...; places behind the last repeat it (their sums are not stored)
#pragma unroll
        for (int j = 0; j < (kMost + 63) / 64; ++j) {
          const int pr = p.rows[tile.tok + min((int)crank * half + 32 * j + lane, tile.n - 1)];
          row[j] = ((unsigned)pr < (unsigned)p.n_tok ? (unsigned)pr / (unsigned)p.per : 0u) * (uint32_t)(p.k_pad >> 4);
        }
        // rows x k_pad / 16 stays below 2^32
#pragma unroll
        for (int i = 0; i < kMost / 8; ++i) from[i] = __shfl_sync(0xffffffffu, row[i >> 3], ((4 * i) & 31) + sub) + chunk;
      }
      bool ok = use == 0 || mbar_wait_bounded<false>(empty_bar(s), (use & 1u) ^ 1u, limit, abort_flag, p.status, WM_EMPTY, t);
      ok = __all_sync(0xffffffffu, ok);
      if (!ok) break;
      const bool real = kc * kStep + 16 * chunk < p.k_pad;
      const uint8_t* src = p.x + (real ? kc * kStep : 0);
#pragma unroll
      for (int i = 0; i < kMost / 8; ++i)
        if (4 * i < half) copy16_async(dst + sw128_offset(4 * i + sub, chunk), src + (uint64_t)from[i] * 16, real);
      copies_commit();
      copies_wait<0>();
      fence_proxy_async_smem();
      __syncwarp();
      if (lane == 0) mbar_arrive_remote(full_remote);
    }
  } else if (warp >= 4) {
    // ---- scales and stores: lane = channel, columns = token rows; the two groups of four warps take 32 columns in turn ----
    const int group = (warp - 4) >> 2, quad = warp & 3;
    const uint32_t lane_base = (uint32_t)(quad * 32) << 16;
    const uint32_t acc_empty_remote = mapa_shared(acc_empty_bar(0), lead);
    TokenOut* toks = reinterpret_cast<TokenOut*>(smem + S::kOffTok);
    uint32_t tile_i = 0;
    int e = 0;
    bool ok = true;
    for (int t = pair; t < n_tiles && ok; t += n_pairs, ++tile_i) {
      const Tile8 tile = tile_at(t, e);
      const uint32_t b = tile_i & 1u;
      {  // scale and output row of every token row of the tile (two sets: the other one may still be in use)
        const int i = (int)threadIdx.x - 128;
        float sc = 0.f;
        int row = -1;
        if (i < tile.n) {
          if constexpr (kExperts) {
            const int pr = p.rows[tile.tok + i];
            if ((unsigned)pr < (unsigned)p.n_tok) {
              row = pr;
              sc = p.sx[(unsigned)pr / (unsigned)p.per];
            } else {
              report_status(p.status, 4 /*RK_ERR_ROWS*/, RK_CHK_EXPERT_ROW, pr);
            }
          } else {
            row = tile.tok + i;
            sc = p.sx[row];
          }
        }
        TokenOut out;
        out.at = row < 0 ? -1 : (long long)row * p.y_stride * (p.out_f32 ? 4 : 2);
        out.scale = sc;
        out.pad = 0;
        toks[256 * b + i] = out;
      }
      const int chan = tile.chan + (int)crank * 128 + quad * 32 + lane;
      const bool mine = chan < p.n_out;
      const float sw = mine ? p.sw[(int64_t)tile.mat * p.n_out + chan] : 0.f;
      ok = mbar_wait_bounded<false>(acc_full_bar(b), (tile_i >> 1) & 1u, limit, abort_flag, p.status, WM_ACC_FULL, t);
      ok = named_barrier_and(1, 256, ok);
      if (!ok) break;
      tc_fence_after_sync();
      for (int c0 = 32 * group; c0 < tile.n; c0 += 64) {
        uint32_t o[32];
        __syncwarp();  // (lanes beyond the last channel store nothing)
        tmem_ld_x32(tmem_base + lane_base + b * kTileN + c0, o);
        tmem_wait_ld();
        if constexpr (kSplit > 1) {  // into the ring, whose products are done: [token][channel]
          uint32_t* part = reinterpret_cast<uint32_t*>(smem) + c0 * 128 + quad * 32 + lane;
#pragma unroll
          for (int i = 0; i < 32; ++i) part[i * 128] = o[i];
          continue;
        }
        if (p.out_f32)
          store_columns<float>(o, toks + 256 * b + c0, static_cast<uint8_t*>(p.y) + (int64_t)chan * 4, sw, mine);
        else if (p.paired)
          store_columns_paired(o, toks + 256 * b + c0, static_cast<uint8_t*>(p.y) + (int64_t)(chan & ~1) * 2, sw, mine);
        else
          store_columns<__nv_bfloat16>(o, toks + 256 * b + c0, static_cast<uint8_t*>(p.y) + (int64_t)chan * 2, sw, mine);
      }
      tc_fence_before_sync();
      __syncwarp();
      if (lane == 0) mbar_arrive_remote(acc_empty_remote + 8u * b);
    }
  }
  if (*abort_flag != 0) {
    for (int i = 0; i < 64; ++i) __nanosleep(1000);
  }
  if constexpr (kSplit > 1) {
    __syncwarp();
    cluster_arrive();
    cluster_wait();  // all partial sums are in shared memory
    if (warp >= 4) {
      int e = 0;
      const Tile8 tile = tile_at(pair, e);
      const int part = (((tile.n + 31) >> 5) << 5) / kSplit;  // token columns of this CTA: a multiple of 8
      const int begin = (int)(cluster_rank >> 1) * part, end = min(begin + part, tile.n);
      const int quad = warp & 3, chan = tile.chan + (int)crank * 128 + quad * 32 + lane;
      const bool mine = chan < p.n_out;
      const float sw = mine ? p.sw[chan] : 0.f;
      const TokenOut* toks = reinterpret_cast<const TokenOut*>(smem + S::kOffTok);
      constexpr int kCols = 4;  // columns at a time: all their loads (a trip to another SM each) are under way together
      for (int c = begin + kCols * ((warp - 4) >> 2); c < end; c += 2 * kCols) {
        int v[kSplit][kCols];
        const uint32_t at = smem_base + (uint32_t)(c * 128 + quad * 32 + lane) * 4u;
#pragma unroll
        for (int r = 0; r < kSplit; ++r) {
          const uint32_t from = mapa_shared(at, 2 * r + crank);
#pragma unroll
          for (int i = 0; i < kCols; ++i) asm volatile("ld.shared::cluster.s32 %0, [%1];" : "=r"(v[r][i]) : "r"(from + 512u * i));
        }
#pragma unroll
        for (int i = 0; i < kCols; ++i) {
          int sum = v[0][i];
#pragma unroll
          for (int r = 1; r < kSplit; ++r) sum += v[r][i];
          const TokenOut out = toks[c + i];
          const float f = (float)sum * out.scale * sw;
          if (!mine || out.at < 0) continue;
          if (p.out_f32)
            *reinterpret_cast<float*>(static_cast<uint8_t*>(p.y) + out.at + (int64_t)chan * 4) = f;
          else
            *reinterpret_cast<__nv_bfloat16*>(static_cast<uint8_t*>(p.y) + out.at + (int64_t)chan * 2) = __float2bfloat16_rn(f);
        }
      }
    }
  }
  __syncwarp();
  tc_fence_before_sync();
  __syncthreads();
  __syncwarp();
  cluster_arrive();
  cluster_wait();
  if (warp == 0) {
    __syncwarp();
    tmem_dealloc<2>(tmem_base, 512);
  }
}

cudaLaunchConfig_t pair_config(int n_blocks, int n_threads, int cluster, cudaLaunchAttribute* attr, cudaStream_t stream) {
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(n_blocks);
  cfg.blockDim = dim3(n_threads);
  cfg.dynamicSmemBytes = Smem8::kBytes;
  cfg.stream = stream;
  attr->id = cudaLaunchAttributeClusterDimension;
  attr->val.clusterDim.x = cluster;
  attr->val.clusterDim.y = attr->val.clusterDim.z = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  return cfg;
}

}  // namespace

cudaError_t matmul8_setup(int32_t* split_slots) {
  cudaError_t e = cudaSuccess;
  for (auto kernel : {rk_matmul8_pair_kernel<false, false, 1>, rk_matmul8_pair_kernel<true, false, 1>, rk_matmul8_pair_kernel<true, true, 1>,
                      rk_matmul8_pair_kernel<false, false, 2>, rk_matmul8_pair_kernel<false, false, 4>})
    if (e == cudaSuccess) e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)Smem8::kBytes);
  for (int i = 0; i < 2 && e == cudaSuccess; ++i) {
    cudaLaunchAttribute attr;
    const cudaLaunchConfig_t cfg = pair_config(4 << i, kThreads8, 4 << i, &attr, nullptr);
    int n = 0;
    const cudaError_t asked = i == 0 ? cudaOccupancyMaxActiveClusters(&n, rk_matmul8_pair_kernel<false, false, 2>, &cfg)
                                     : cudaOccupancyMaxActiveClusters(&n, rk_matmul8_pair_kernel<false, false, 4>, &cfg);
    split_slots[i] = asked == cudaSuccess ? n : 0;  // 0: a device without room for such a cluster, whose products do not share k
    if (asked != cudaSuccess) cudaGetLastError();
  }
  return e;
}

cudaError_t launch_quant8(const void* x, int64_t x_stride, int64_t n_rows, int32_t k, void* codes, float* scales, cudaStream_t stream) {
  const int k_pad = (k + 15) / 16 * 16, want = (k_pad / 8 + kQuantHeld - 1) / kQuantHeld;
  const bool vec = (reinterpret_cast<uintptr_t>(x) & 15u) == 0 && x_stride % 8 == 0;
  const __nv_bfloat16* src = static_cast<const __nv_bfloat16*>(x);
  uint8_t* dst = static_cast<uint8_t*>(codes);
  if (want <= 32) {
    auto kernel = vec ? quant8_kernel<true, true> : quant8_kernel<false, true>;
    kernel<<<(unsigned)((n_rows + kQuantRows - 1) / kQuantRows), 32 * kQuantRows, 0, stream>>>(src, x_stride, n_rows, k, k_pad, dst, scales);
  } else {
    int nt = 64;
    while (nt < want && nt < 512) nt *= 2;
    auto kernel = vec ? quant8_kernel<true, false> : quant8_kernel<false, false>;
    kernel<<<(unsigned)n_rows, nt, 0, stream>>>(src, x_stride, n_rows, k, k_pad, dst, scales);
  }
  return cudaGetLastError();
}

// Few tiles: smaller ones, or k shared by the pairs of a cluster, put more SMs to work.  Clocks of a pair, measured: a step
// of k takes 2 N where the tensor cores set the pace and no less than 350, a token row's stores 14, the join 2000 + 10 N.
extern "C" void rk_matmul8_plan(int64_t n_out, int64_t n_tok, int32_t k_pad, int32_t sm_count, const int32_t* split_slots, int32_t* tile_rows,
                                int32_t* split) {
  const int64_t n_chan = (n_out + kTileM - 1) / kTileM;
  const int k_chunks = (k_pad + kStep - 1) / kStep;
  double best = 1e30;
  for (int most = kTileN; most >= 32; most /= 2) {
    const int64_t n = n_chan * ((n_tok + most - 1) / most);
    for (int s = 1; s <= 4; s *= 2) {
      const int64_t slots = s == 1 ? (sm_count < 2 ? 1 : sm_count / 2) : split_slots[s / 4];
      if (slots < 1) continue;
      const int64_t rounds = (n + slots - 1) / slots;
      if (s > 1 && (rounds > 1 || k_chunks < 4 * s)) continue;
      const double step = 2.1 * most > 350.0 ? 2.1 * most : 350.0;
      const double clocks = (double)rounds * ((k_chunks + s - 1) / s) * step + 14.0 * most + (s > 1 ? 2000.0 + 10.0 * most : 0.0);
      if (clocks < 0.97 * best) {  // (the larger tile where it makes no difference)
        best = clocks;
        *tile_rows = most;
        *split = s;
      }
    }
  }
}

cudaError_t launch_matmul8(Matmul8Params p, int sm_count, cudaStream_t stream) {
  p.paired = !p.out_f32 && (reinterpret_cast<uintptr_t>(p.y) & 3u) == 0 && p.y_stride % 2 == 0 && p.n_out % 2 == 0;
  const int64_t n_chan = (p.n_out + kTileM - 1) / kTileM;
  // by expert the number of tiles is known on the device only: at most one part-filled tile per expert more than full ones
  // Tiles of 256 rows where experts have more than 128 on average (at 192 an expert of 200 or 400 rows costs a tile more:
  // 8192 tokens, 384 rows on average, 8% less time), the deeper ring where their weights' bytes count (64 tokens: 154 -> 149)
  const bool few = p.rows != nullptr && p.n_tok <= 128 * (int64_t)p.n_mat;
  const int most = few ? kTileNFew : kTileN;
  const int64_t tok_tiles = (p.n_tok + most - 1) / most + (p.rows ? (p.n_mat < p.n_tok ? p.n_mat : p.n_tok) : 0);
  int64_t tiles = n_chan * tok_tiles;
  cudaLaunchAttribute attr;
  if (!p.rows) {
    tiles = n_chan * ((p.n_tok + p.tile_rows - 1) / p.tile_rows);
    if (p.split > 1) {
      const cudaLaunchConfig_t cfg = pair_config((int)tiles * 2 * p.split, kThreads8, 2 * p.split, &attr, stream);
      return p.split == 4 ? cudaLaunchKernelEx(&cfg, rk_matmul8_pair_kernel<false, false, 4>, p) : cudaLaunchKernelEx(&cfg, rk_matmul8_pair_kernel<false, false, 2>, p);
    }
  }
  const int n_pairs = (int)(tiles < sm_count / 2 ? tiles : sm_count / 2);
  const cudaLaunchConfig_t cfg = pair_config(2 * n_pairs, threads8(p.rows != nullptr, few), 2, &attr, stream);
  if (!p.rows) return cudaLaunchKernelEx(&cfg, rk_matmul8_pair_kernel<false, false, 1>, p);
  return few ? cudaLaunchKernelEx(&cfg, rk_matmul8_pair_kernel<true, true, 1>, p) : cudaLaunchKernelEx(&cfg, rk_matmul8_pair_kernel<true, false, 1>, p);
}

}  // namespace rk
