// Absorbed-MLA attention of single tokens (or a few drafted ones) over the 4-bit paged latent cache:
//   per document segment i:  q_i = R(-delta_i) q;   S = q_i K_i^T;   O = softmax over all segments' keys, times C.
//
// A decode step has few query rows (q_len * heads of one sequence) and many keys, so the products are issued with
// the KEYS in the M = 128 dimension of the tensor cores and the query rows in N = 16, 32 or 64:
//   S^T[128 keys x N]   = K[128 x 576] Q^T          9 chunks of 64 dims, A K-major, B K-major
//   O^T[512 dims x N]  += C^T[512 x 128] P^T        4 tiles of 128 dims, A MN-major, B MN-major
// With the rows in M a 64-row tile would run the tensor cores at half rate (M = 64) and 16 rows at an eighth.  The
// same shared-memory tile (128 keys x 64 dims per 16 KB chunk, 128-byte swizzle) is the K-major A operand of the
// scores and the MN-major A operand of the values.
//
// Dequantisation happens between the HBM load and the shared-memory store: 256 threads, two per key, hold the next
// tile's 13 16-byte units each in registers while this tile computes (53 KB in flight per SM) and write the bf16
// values n * s, which are exact.  One tile (144 KB) and the queries (72 KB) fill the shared memory, so the tile is
// refilled chunk pair by chunk pair as the value products release it; the scores' products of the next tile follow
// behind.  P^T (16 KB) shares the space of the rope chunk, which only the scores read.
//
// Statistics: running maximum per query row in shared memory, raised only when a tile exceeds it by more than 2^8
// (then O^T is rescaled in tensor memory, columns = rows of the query); sums per (key lane, row) in registers in
// fp32, added up over the lanes once per row tile.  P is rounded to bf16 for the tensor cores (relative 2^-9 per
// key, averaged by the sum); the rotated query rope is rounded to bf16 like in the online step.
//
// Work: the plan lists every (sequence, row tile, key tile) in order and gives each CTA an equal run of them.  A
// row tile whose keys several CTAs share leaves normalised fp32 partial results and their log-sum-exp, which a
// second kernel joins in CTA order (no atomics: results do not depend on timing).
//
// Warps (576 threads): 0 issues the MMAs, 1 loads the queries (TMA) and turns their rope part, 2-9 load and
// dequantise keys, 10-17 softmax, correction and epilogue.
#include <cuda_bf16.h>

#include "rk_internal.h"

namespace rk {
namespace {

constexpr int kThreads = 576;
constexpr uint32_t kKChunk = 16384;  // 128 keys x 64 dims bf16
constexpr uint32_t kQChunk = 8192;   // up to 64 rows x 64 dims bf16

constexpr uint32_t kOffQ = 0;                        // 8 latent chunks, then the turned rope chunk
constexpr uint32_t kOffK = 9 * kQChunk;              // 8 latent chunks, then the rope chunk / P^T
constexpr uint32_t kOffP = kOffK + 8 * kKChunk;
constexpr uint32_t kOffBars = kOffK + 9 * kKChunk;
enum { B_QFULL = 0, B_QROPE = 1, B_KFULL = 2 /*5*/, B_SFULL = 7, B_PREADY = 8, B_PVDONE = 9 /*4*/, B_COUNT = 13 };
constexpr uint32_t kOffTmem = kOffBars + B_COUNT * 8;
constexpr uint32_t kOffAbort = kOffTmem + 4;
constexpr uint32_t kOffMax = kOffBars + 128;         // float [64]: running maximum of each row, base-2 units
constexpr uint32_t kOffPos = kOffMax + 256;          // int [64]: request position of each row (-1: no row)
constexpr uint32_t kOffRed = kOffPos + 256;          // float [4][64]: per lane quarter
constexpr uint32_t kOffAlpha = kOffRed + 1024;       // float [64]: factor of the last raise of a row's maximum
constexpr uint32_t kSmemUsed = kOffAlpha + 256;
constexpr uint32_t kSmemBytes = kSmemUsed + 1024;    // alignment slack

constexpr uint32_t kColS = 256;      // O^T takes 4 x N columns from 0
constexpr float kNoMax = -1e30f;     // "no key seen yet": finite, so that differences stay defined

enum { W_QFULL = 41, W_QROPE, W_KFULL, W_SFULL, W_PREADY, W_PVDONE };

// Walks one CTA's run of key tiles.  A "group" is the part of one (sequence, row tile) that this CTA owns.
struct Cursor {
  const DecodeAttnParams& p;
  int left;             // tiles this CTA still has to do, the current group's included
  int b, rt, tile;      // sequence, row tile, first key tile of the group within the sequence
  int n_b, tile0, cnt;  // key tiles of the sequence, its first record, tiles of the group
  __device__ Cursor(const DecodeAttnParams& p_) : p(p_) {
    const int4 s = p.cta_start[blockIdx.x];
    const long long w0 = (long long)blockIdx.x * p.header->chunk;
    const long long w1 = (long long)p.header->n_tiles * p.n_row_tiles;
    const long long rest = w1 - w0;
    left = s.w == 0 || rest <= 0 ? 0 : (int)(rest < p.header->chunk ? rest : p.header->chunk);
    b = s.x;
    rt = s.y;
    tile = s.z;
    cnt = 0;
  }
  // makes the next group current; false when the run is done
  __device__ bool next() {
    if (cnt > 0) {
      left -= cnt;
      tile += cnt;
      if (tile == n_b) {
        tile = 0;
        if (++rt == p.n_row_tiles) {
          rt = 0;
          ++b;
        }
      }
    }
    if (left <= 0) return false;
    while (true) {
      tile0 = p.seq_tile[b];
      n_b = p.seq_tile[b + 1] - tile0;
      if (n_b > 0) break;
      ++b;  // a sequence that sees no key has no tiles; the joining kernel writes its rows
    }
    cnt = n_b - tile < left ? n_b - tile : left;
    return true;
  }
  __device__ int record(int k) const { return tile0 + tile + k; }
  __device__ bool whole() const { return cnt == n_b; }
};

template <int N>
__device__ __forceinline__ void tmem_ld(uint32_t a, uint32_t* r) {
  if constexpr (N == 8) tmem_ld_x8(a, r);
  else if constexpr (N == 16) tmem_ld_x16(a, r);
  else tmem_ld_x32(a, r);
}
__device__ __forceinline__ float fast_exp2(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}

// One key's share of a tile in one of its two threads: chunks h, h + 2, h + 4, h + 6 of the latent (two units each),
// the scale unit h and rope units 4 h .. 4 h + 3.
struct KeyRegs {
  uint4 code[8];
  uint4 scale;
  uint4 rope[4];
};

}  // namespace

template <int kRows>
__global__ void __launch_bounds__(kThreads, 1) rk_decode_attn_kernel(const __grid_constant__ DecodeAttnParams p) {
  extern __shared__ uint8_t smem_raw[];
  const uint32_t smem_base = (smem_u32(smem_raw) + 1023u) & ~1023u;
  uint8_t* smem = smem_raw + (smem_base - smem_u32(smem_raw));
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  auto bar = [&](int i) -> uint32_t { return smem_base + kOffBars + 8u * i; };
  volatile int* abort_flag = reinterpret_cast<volatile int*>(smem + kOffAbort);
  volatile uint32_t* tmem_ptr = reinterpret_cast<volatile uint32_t*>(smem + kOffTmem);
  const uint64_t limit = p.wait_ns;

  {  // the plan has to be the one of this call's shape, heads and pool
    const DecodePlanHeader* h = p.header;
    if (h->magic != kDecodePlanMagic || h->n_seqs != p.n_seqs || h->q_len != p.q_len || h->n_items != p.n_items ||
        h->max_tiles != p.max_tiles || h->n_heads != p.n_heads || h->n_pages != p.n_pages) {
      if (threadIdx.x == 0) report_status(p.status, 3 /*RK_ERR_LAYOUT*/, RK_CHK_PLAN_MATCH, h->magic);
      return;
    }
    if (p.cta_start[blockIdx.x].w == 0) return;  // no work for this CTA
  }
  if (threadIdx.x == 0) {
    *abort_flag = 0;
    mbar_init(bar(B_QFULL), 1);
    mbar_init(bar(B_QROPE), 1);
    for (int i = 0; i < 5; ++i) mbar_init(bar(B_KFULL + i), 8);
    mbar_init(bar(B_SFULL), 1);
    mbar_init(bar(B_PREADY), 8);
    for (int i = 0; i < 4; ++i) mbar_init(bar(B_PVDONE + i), 1);
    fence_mbar_init_cluster();
  }
  if (warp == 0) {
    __syncwarp();
    tmem_alloc<1>(smem_base + kOffTmem, 512);
    tmem_relinquish<1>();
  }
  tc_fence_before_sync();
  __syncthreads();
  tc_fence_after_sync();
  const uint32_t tmem = *tmem_ptr;
  const int rows_per_seq = p.q_len * p.n_heads;

  if (warp == 0) {
    // ------------------------------ MMA issue (whole warp loops, one elected lane issues) ----------------------
    constexpr uint32_t id_qk = umma_idesc_bf16(128, kRows, 0, 0);
    constexpr uint32_t id_pv = umma_idesc_bf16(128, kRows, 1, 1);
    uint32_t t = 0, groups = 0;  // tiles and groups done so far: their parities are the barriers' phases
    bool ok = true;
    for (Cursor c(p); ok && c.next(); ++groups) {
      ok = mbar_wait_bounded<false>(bar(B_QFULL), groups & 1u, limit, abort_flag, p.status, W_QFULL, (int)groups);
      for (int k = 0; ok && k < c.cnt; ++k, ++t) {
        for (int m = 0; ok && m < 4; ++m) {  // scores: chunk pairs in the order they are filled
          ok = mbar_wait_bounded<false>(bar(B_KFULL + m), t & 1u, limit, abort_flag, p.status, W_KFULL, m);
          if (!ok) break;
          if (elect_one()) {
            const uint64_t da = umma_desc_sw128(smem_base + kOffK + 2 * m * kKChunk, 16, 1024);
            const uint64_t db = umma_desc_sw128(smem_base + kOffQ + 2 * m * kQChunk, 16, 1024);
#pragma unroll
            for (int s = 0; s < 8; ++s)
              umma_f16<1>(tmem + kColS, da + (uint64_t)(((s >> 2) * kKChunk + (s & 3) * 32) >> 4),
                          db + (uint64_t)(((s >> 2) * kQChunk + (s & 3) * 32) >> 4), id_qk, (m > 0 || s > 0) ? 1u : 0u);
          }
          __syncwarp();
        }
        ok = ok && mbar_wait_bounded<false>(bar(B_KFULL + 4), t & 1u, limit, abort_flag, p.status, W_KFULL, 4) &&
             mbar_wait_bounded<false>(bar(B_QROPE), t & 1u, limit, abort_flag, p.status, W_QROPE, k);
        if (!ok) break;
        if (elect_one()) {
          const uint64_t da = umma_desc_sw128(smem_base + kOffK + 8 * kKChunk, 16, 1024);
          const uint64_t db = umma_desc_sw128(smem_base + kOffQ + 8 * kQChunk, 16, 1024);
#pragma unroll
          for (int s = 0; s < 4; ++s) umma_f16<1>(tmem + kColS, da + (uint64_t)(2 * s), db + (uint64_t)(2 * s), id_qk, 1u);
          umma_commit_1(bar(B_SFULL));
        }
        __syncwarp();
        ok = mbar_wait_bounded<false>(bar(B_PREADY), t & 1u, limit, abort_flag, p.status, W_PREADY, k);
        if (!ok) break;
        tc_fence_after_sync();
        if (elect_one()) {
          const uint64_t db = umma_desc_sw128(smem_base + kOffP, 16, 1024);
#pragma unroll 1
          for (int m = 0; m < 4; ++m) {  // 128 dims each: two 64-dim chunks, 16 KB apart
            const uint64_t da = umma_desc_sw128(smem_base + kOffK + 2 * m * kKChunk, kKChunk, 1024);
#pragma unroll
            for (int s = 0; s < 8; ++s)
              umma_f16<1>(tmem + (uint32_t)(m * kRows), da + (uint64_t)((s * 2048) >> 4), db + (uint64_t)((s * 2048) >> 4), id_pv,
                          (k > 0 || s > 0) ? 1u : 0u);
            umma_commit_1(bar(B_PVDONE + m));
          }
        }
        __syncwarp();
      }
    }
  } else if (warp == 1) {
    // ------------------------------ queries: latent chunks by TMA, rope chunk turned by R(-delta) -------------
    uint32_t t = 0, groups = 0;
    bool ok = true;
    const int rc = lane & 7;
    for (Cursor c(p); ok && c.next(); ++groups) {
      // the previous group's scores are done with the query chunks (its last tile's S is complete)
      if (t > 0) ok = mbar_wait_bounded<false>(bar(B_SFULL), (t - 1) & 1u, limit, abort_flag, p.status, W_SFULL, (int)t);
      if (!ok) break;
      const int row0 = c.b * rows_per_seq + c.rt * kRows;
      if (elect_one()) {
        mbar_arrive_expect_tx(bar(B_QFULL), 8 * kRows * 128);
        for (int d = 0; d < 8; ++d) tma_load_2d(smem_base + kOffQ + d * kQChunk, &p.tm_q, bar(B_QFULL), d * 64, row0);
      }
      __syncwarp();
      int valid = rows_per_seq - c.rt * kRows;
      if (valid > kRows) valid = kRows;
      int delta = -1;
      for (int k = 0; ok && k < c.cnt; ++k, ++t) {
        const int d = p.tiles[c.record(k)].delta;
        if (k > 0) ok = mbar_wait_bounded<false>(bar(B_SFULL), (t - 1) & 1u, limit, abort_flag, p.status, W_SFULL, (int)t);
        if (!ok) break;
        if (d != delta) {
          delta = d;
          float cs[4], sn[4];
#pragma unroll
          for (int e = 0; e < 4; ++e) rope_cos_sin(p.rope, d, 4 * rc + e, cs[e], sn[e]);
          const __nv_bfloat16* src = static_cast<const __nv_bfloat16*>(p.q) + (int64_t)row0 * kDQK + kDLatent + rc * 8;
#pragma unroll 4
          for (int r = lane >> 3; r < kRows; r += 4) {
            uint4 v = make_uint4(0, 0, 0, 0);
            if (r < valid) v = *reinterpret_cast<const uint4*>(src + (int64_t)r * kDQK);
            const uint32_t in[4] = {v.x, v.y, v.z, v.w};
            uint32_t o[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              const float x0 = __uint_as_float(in[e] << 16), x1 = __uint_as_float(in[e] & 0xffff0000u);
              o[e] = pack_bf16(x0 * cs[e] + x1 * sn[e], x1 * cs[e] - x0 * sn[e]);
            }
            *reinterpret_cast<uint4*>(smem + kOffQ + 8 * kQChunk + sw128_offset((uint32_t)r, (uint32_t)rc)) =
                make_uint4(o[0], o[1], o[2], o[3]);
          }
          fence_proxy_async_smem();
        }
        __syncwarp();
        if (lane == 0) mbar_arrive(bar(B_QROPE));
      }
    }
  } else if (warp < 10) {
    // ------------------------------ keys: HBM -> registers (4-bit) -> shared memory (bf16) --------------------
    const int kw = warp - 2;
    const int row = 32 * (kw & 3) + lane, h = kw >> 2;
    const uint32_t xr = (uint32_t)(row & 7);
    KeyRegs kr;
    const uint8_t* src = nullptr;  // this key's first unit in the tile being loaded, null for a row that is not there
    auto open = [&](int rec) {
      const int4 v = *reinterpret_cast<const int4*>(&p.tiles[rec]);
      const int page = row < 64 ? v.x : v.y;
      src = row < v.w ? p.pages + (int64_t)page * kCache4PageBytes + (row & 63) * 16 : nullptr;
    };
    // rows that are not there become zeros (code 8): their scores are masked, and 0 * 0 adds nothing to O
    auto load_pair = [&](int m) {
      const uint32_t z = 0x88888888u;
      kr.code[2 * m] = kr.code[2 * m + 1] = make_uint4(z, z, z, z);
      if (src != nullptr) {
        kr.code[2 * m] = __ldg(reinterpret_cast<const uint4*>(src + (4 * m + 2 * h) * 1024));
        kr.code[2 * m + 1] = __ldg(reinterpret_cast<const uint4*>(src + (4 * m + 2 * h + 1) * 1024));
      }
    };
    auto load_scale = [&]() -> uint4 {
      return src != nullptr ? __ldg(reinterpret_cast<const uint4*>(src + (16 + h) * 1024)) : make_uint4(0, 0, 0, 0);
    };
    auto load_rope = [&]() {
#pragma unroll
      for (int e = 0; e < 4; ++e)
        kr.rope[e] = src != nullptr ? __ldg(reinterpret_cast<const uint4*>(src + (18 + 4 * h + e) * 1024)) : make_uint4(0, 0, 0, 0);
    };
    uint32_t t = 0;
    bool ok = true;
    Cursor c(p);
    bool more = c.next();
    int k = 0;
    if (more) {
      open(c.record(0));
#pragma unroll
      for (int m = 0; m < 4; ++m) load_pair(m);
      kr.scale = load_scale();
      load_rope();
    }
    while (ok && more) {
      // the record after this one: its loads go out piece by piece as this tile's registers become free
      if (++k == c.cnt) {
        more = c.next();
        k = 0;
      }
      if (more) open(c.record(k));
      else src = nullptr;
      const uint4 next_scale = load_scale();
      const uint32_t sw[4] = {kr.scale.x, kr.scale.y, kr.scale.z, kr.scale.w};
#pragma unroll
      for (int m = 0; m < 4; ++m) {
        if (t > 0) ok = mbar_wait_bounded<false>(bar(B_PVDONE + m), (t - 1) & 1u, limit, abort_flag, p.status, W_PVDONE, m);
        if (!ok) break;
        uint8_t* dst = smem + kOffK + (2 * m + h) * kKChunk + row * 128;
#pragma unroll
        for (int u = 0; u < 2; ++u) {
          const uint4 v = kr.code[2 * m + u];
          const uint32_t s0 = cache4_scale((sw[m] >> (16 * u)) & 255u), s1 = cache4_scale((sw[m] >> (16 * u + 8)) & 255u);
          *reinterpret_cast<uint4*>(dst + (((4u * u + 0u) ^ xr) << 4)) = cache4_dequant(v.x, s0);
          *reinterpret_cast<uint4*>(dst + (((4u * u + 1u) ^ xr) << 4)) = cache4_dequant(v.y, s0);
          *reinterpret_cast<uint4*>(dst + (((4u * u + 2u) ^ xr) << 4)) = cache4_dequant(v.z, s1);
          *reinterpret_cast<uint4*>(dst + (((4u * u + 3u) ^ xr) << 4)) = cache4_dequant(v.w, s1);
        }
        if (more) load_pair(m);
        fence_proxy_async_smem();
        __syncwarp();
        if (lane == 0) mbar_arrive(bar(B_KFULL + m));
      }
      if (!ok) break;
      // the rope chunk's space held P^T of the previous tile: every value product has completed (waited for above)
      uint8_t* dst = smem + kOffK + 8 * kKChunk + row * 128;
#pragma unroll
      for (int e = 0; e < 4; ++e) *reinterpret_cast<uint4*>(dst + (((4u * h + e) ^ xr) << 4)) = kr.rope[e];
      if (more) load_rope();
      kr.scale = next_scale;
      fence_proxy_async_smem();
      __syncwarp();
      if (lane == 0) mbar_arrive(bar(B_KFULL + 4));
      ++t;
    }
  } else {
    // ------------------------------ softmax, correction, epilogue ---------------------------------------------
    // Thread = one key of the tile (TMEM lane) and half of the query rows (columns).
    constexpr int NC = kRows / 2;
    const int q = warp & 3;            // TMEM lane quarter
    const int ch = (warp - 10) >> 2;   // column half
    const int key = 32 * q + lane;
    const int c0 = ch * NC;
    const uint32_t lane_base = (uint32_t)(32 * q) << 16;
    const uint32_t t_s = tmem + lane_base + kColS + (uint32_t)c0;
    const uint32_t t_o = tmem + lane_base + (uint32_t)c0;
    float* s_max = reinterpret_cast<float*>(smem + kOffMax);
    int* s_pos = reinterpret_cast<int*>(smem + kOffPos);
    float* s_red = reinterpret_cast<float*>(smem + kOffRed);
    float* s_alpha = reinterpret_cast<float*>(smem + kOffAlpha);
    const int tid = threadIdx.x - 320;
    const float scale = p.scale_log2;
    uint32_t t = 0;
    bool ok = true;
    for (Cursor c(p); ok && c.next();) {
      // s_max, s_pos: every warp is done with the previous group (the barrier in its epilogue)
      int pmin = 0x7fffffff;
      for (int i = 0; i < p.q_len; ++i) pmin = min(pmin, p.pos[c.b * p.q_len + i]);
      if (tid < kRows) {
        const int r = c.rt * kRows + tid;
        s_max[tid] = kNoMax;
        s_pos[tid] = r < rows_per_seq ? p.pos[c.b * p.q_len + r / p.n_heads] : -1;
      }
      named_barrier_sync(1, 256);
      float l[NC];
#pragma unroll
      for (int i = 0; i < NC; ++i) l[i] = 0.f;
      for (int k = 0; ok && k < c.cnt; ++k, ++t) {
        const int4 rec = *reinterpret_cast<const int4*>(&p.tiles[c.record(k)]);
        const bool full = rec.w == kDecodeKeys && pmin - rec.z + 1 >= kDecodeKeys;  // no key of the tile is masked
        ok = mbar_wait_bounded<false>(bar(B_SFULL), t & 1u, limit, abort_flag, p.status, W_SFULL, k);
        // a warp that gave up must not leave the others in a named barrier: the vote below ends them together
        if (ok) tc_fence_after_sync();
        uint32_t s[NC];
        float top = -INFINITY;
        if (ok) {
          tmem_ld<NC>(t_s, s);
          tmem_wait_ld();
          if (!full) {
#pragma unroll
            for (int i = 0; i < NC; ++i)
              if (key >= rec.w || rec.z + key > s_pos[c0 + i]) s[i] = 0xff800000u;
          }
#pragma unroll
          for (int i = 0; i < NC; i += 4) {
            const float4 mx = *reinterpret_cast<const float4*>(s_max + c0 + i);
            top = fmaxf(fmaxf(top, fmaf(__uint_as_float(s[i]), scale, -mx.x)), fmaf(__uint_as_float(s[i + 1]), scale, -mx.y));
            top = fmaxf(fmaxf(top, fmaf(__uint_as_float(s[i + 2]), scale, -mx.z)), fmaf(__uint_as_float(s[i + 3]), scale, -mx.w));
          }
        }
        ok = named_barrier_and(2, 256, ok);
        if (!ok) break;
        if (named_barrier_or(1, 256, top > 8.f)) {
          // some row's maximum grows by more than 2^8 (always so for the first visible keys): exact maxima of the tile
#pragma unroll
          for (int i = 0; i < NC; ++i) {
            float v = __uint_as_float(s[i]) * scale;
#pragma unroll
            for (int o = 16; o > 0; o >>= 1) v = fmaxf(v, __shfl_xor_sync(0xffffffffu, v, o));
            if (lane == 0) s_red[q * 64 + c0 + i] = v;
          }
          named_barrier_sync(1, 256);
          if (tid < kRows) {
            const float v = fmaxf(fmaxf(s_red[tid], s_red[64 + tid]), fmaxf(s_red[128 + tid], s_red[192 + tid]));
            const float old = s_max[tid];
            const bool raise = v > old + 8.f;
            s_alpha[tid] = raise ? fast_exp2(old - v) : 1.f;
            if (raise) s_max[tid] = v;
          }
          named_barrier_sync(1, 256);
#pragma unroll
          for (int i = 0; i < NC; ++i) l[i] *= s_alpha[c0 + i];
          if (k > 0) {  // S of this tile is complete, so every value product before it is too
#pragma unroll 1
            for (int m = 0; m < 4; ++m) {
#pragma unroll 1
              for (int i0 = 0; i0 < NC; i0 += 8) {
                uint32_t o[8];
                tmem_ld_x8(t_o + (uint32_t)(m * kRows + i0), o);
                tmem_wait_ld();
#pragma unroll
                for (int i = 0; i < 8; ++i) o[i] = __float_as_uint(__uint_as_float(o[i]) * s_alpha[c0 + i0 + i]);
                tmem_st_x8(t_o + (uint32_t)(m * kRows + i0), o);
              }
            }
            tmem_wait_st();
          }
        }
        uint32_t pk[NC / 2];
#pragma unroll
        for (int i = 0; i < NC; i += 4) {
          const float4 mx = *reinterpret_cast<const float4*>(s_max + c0 + i);
          const float p0 = fast_exp2(fmaf(__uint_as_float(s[i]), scale, -mx.x));
          const float p1 = fast_exp2(fmaf(__uint_as_float(s[i + 1]), scale, -mx.y));
          const float p2 = fast_exp2(fmaf(__uint_as_float(s[i + 2]), scale, -mx.z));
          const float p3 = fast_exp2(fmaf(__uint_as_float(s[i + 3]), scale, -mx.w));
          l[i] += p0;
          l[i + 1] += p1;
          l[i + 2] += p2;
          l[i + 3] += p3;
          pk[i / 2] = pack_bf16(p0, p1);
          pk[i / 2 + 1] = pack_bf16(p2, p3);
        }
        // P^T, one 128-byte row per key, query rows contiguous; the rope chunk it replaces has been read (S is complete)
        uint8_t* dst = smem + kOffP + key * 128;
#pragma unroll
        for (int i = 0; i < NC / 8; ++i)
          *reinterpret_cast<uint4*>(dst + ((((uint32_t)(c0 / 8 + i)) ^ (uint32_t)(key & 7)) << 4)) =
              make_uint4(pk[4 * i], pk[4 * i + 1], pk[4 * i + 2], pk[4 * i + 3]);
        fence_proxy_async_smem();
        tc_fence_before_sync();
        __syncwarp();
        if (lane == 0) mbar_arrive(bar(B_PREADY));
      }
      if (!ok) break;
      // ---- epilogue of the group: sums over the key lanes, then O^T / l ----
#pragma unroll
      for (int i = 0; i < NC; ++i) {
        float v = l[i];
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
        if (lane == 0) s_red[q * 64 + c0 + i] = v;
      }
      ok = mbar_wait_bounded<false>(bar(B_PVDONE + 3), (t - 1) & 1u, limit, abort_flag, p.status, W_PVDONE, 4);
      ok = named_barrier_and(2, 256, ok);
      if (!ok) break;
      tc_fence_after_sync();
      const bool whole = c.whole();
      const int slot = 2 * blockIdx.x + (c.tile > 0 ? 0 : 1);
      const int valid = min(rows_per_seq - c.rt * kRows, kRows);
      const int64_t row0 = (int64_t)c.b * rows_per_seq + c.rt * kRows;
#pragma unroll
      for (int i = 0; i < NC; ++i) {
        const int col = c0 + i;
        const float tot = (s_red[col] + s_red[64 + col]) + (s_red[128 + col] + s_red[192 + col]);
        l[i] = tot;
      }
      if (lane == 0 && q == 0) {
#pragma unroll
        for (int i = 0; i < NC; ++i) {
          const int col = c0 + i;
          // tot > 0 or NaN: a NaN score makes its row NaN, a row without visible keys has the sum 0
          const float lse2 = l[i] == 0.f ? -INFINITY : s_max[col] + log2f(l[i]);
          if (!whole) p.part_lse[(int64_t)slot * 64 + col] = lse2;
          else if (col < valid) p.lse[row0 + col] = lse2 * 0.69314718055994530942f;
        }
      }
#pragma unroll
      for (int i = 0; i < NC; ++i) l[i] = l[i] == 0.f ? 0.f : 1.f / l[i];
#pragma unroll 1
      for (int m = 0; m < 4; ++m) {
        uint32_t o[NC];
        tmem_ld<NC>(t_o + (uint32_t)(m * kRows), o);
        tmem_wait_ld();
        const int dim = 128 * m + key;
        if (whole) {
          __nv_bfloat16* out = static_cast<__nv_bfloat16*>(p.O) + row0 * kDLatent + dim;
#pragma unroll
          for (int i = 0; i < NC; ++i)
            if (c0 + i < valid) out[(int64_t)(c0 + i) * kDLatent] = __float2bfloat16_rn(__uint_as_float(o[i]) * l[i]);
        } else {
          float* out = p.part_o + ((int64_t)slot * 64) * kDLatent + dim;
#pragma unroll
          for (int i = 0; i < NC; ++i)
            if (c0 + i < valid) out[(int64_t)(c0 + i) * kDLatent] = __uint_as_float(o[i]) * l[i];
        }
      }
      tc_fence_before_sync();
      named_barrier_sync(1, 256);  // s_red, s_max and s_pos may be overwritten from here on
    }
  }

  // ------------------------------ teardown -------------------------------------------------------------------
  // after a wait has expired: copies and products in flight get a bounded time to finish
  if (*abort_flag != 0) {
    for (int i = 0; i < 64; ++i) __nanosleep(1000);
  }
  __syncwarp();
  tc_fence_before_sync();
  __syncthreads();
  if (warp == 0) {
    __syncwarp();
    tmem_dealloc<1>(tmem, 512);
  }
}

// Joins the partial results of row tiles whose keys several CTAs share, in CTA order: lse = log2 sum 2^lse_j,
// O = sum 2^(lse_j - lse) O_j.  One block per query row; four groups of 128 threads take every fourth part, 16 bytes
// of the row each, so that a row shared by all CTAs has four times eight loads in flight.  Rows of sequences that see
// nothing get O = 0, lse = -inf; rows that one CTA finished alone are already written.
__global__ void __launch_bounds__(512) rk_decode_join_kernel(const __grid_constant__ DecodeAttnParams p, int row_tile) {
  const DecodePlanHeader* h = p.header;
  if (h->magic != kDecodePlanMagic || h->n_seqs != p.n_seqs || h->q_len != p.q_len || h->n_items != p.n_items ||
      h->max_tiles != p.max_tiles || h->n_heads != p.n_heads || h->n_pages != p.n_pages)
    return;  // reported by the attention kernel
  const int rows_per_seq = p.q_len * p.n_heads;
  const int64_t row = blockIdx.x;
  const int b = (int)(row / rows_per_seq), r = (int)(row - (int64_t)b * rows_per_seq);
  const int rt = r / row_tile, col = r - rt * row_tile;
  const int tile0 = p.seq_tile[b], n_b = p.seq_tile[b + 1] - tile0;
  const int part = threadIdx.x >> 7, d4 = threadIdx.x & 127;
  __nv_bfloat16* out = static_cast<__nv_bfloat16*>(p.O) + row * kDLatent + d4 * 4;
  if (n_b == 0) {
    if (part == 0) *reinterpret_cast<uint2*>(out) = make_uint2(0u, 0u);
    if (threadIdx.x == 0) p.lse[row] = -INFINITY;
    return;
  }
  const long long x = (long long)tile0 * p.n_row_tiles + (long long)rt * n_b, y = x + n_b;
  const int ca = (int)(x / h->chunk), cb = (int)((y - 1) / h->chunk);
  if (ca == cb) return;
  // a part is in slot 1 of the CTA that starts the row tile, in slot 0 of the ones that go on with it
  auto slot = [&](int cta) -> int64_t { return (int64_t)2 * cta + (cta == ca ? 1 : 0); };
  float mx = -INFINITY;
  bool nan = false;
  for (int i = ca; i <= cb; ++i) {
    const float v = __ldg(p.part_lse + slot(i) * 64 + col);
    mx = fmaxf(mx, v);
    nan |= v != v;
  }
  const float base = mx == -INFINITY ? 0.f : mx;
  float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
  float tot = 0.f;
#pragma unroll 8
  for (int i = ca + part; i <= cb; i += 4) {
    const float w = exp2f(__ldg(p.part_lse + slot(i) * 64 + col) - base);
    const float4 v = __ldg(reinterpret_cast<const float4*>(p.part_o + (slot(i) * 64 + col) * kDLatent) + d4);
    tot += w;
    if (w != 0.f) {
      acc.x = fmaf(w, v.x, acc.x);
      acc.y = fmaf(w, v.y, acc.y);
      acc.z = fmaf(w, v.z, acc.z);
      acc.w = fmaf(w, v.w, acc.w);
    }
  }
  __shared__ float4 s_acc[3][128];
  __shared__ float s_tot[4];
  if (part > 0) s_acc[part - 1][d4] = acc;
  if (d4 == 0) s_tot[part] = tot;
  __syncthreads();
  if (part > 0) return;
  const float all = (s_tot[0] + s_tot[1]) + (s_tot[2] + s_tot[3]);
  const float inv = all == 0.f ? 0.f : 1.f / all;
#pragma unroll
  for (int i = 0; i < 3; ++i) {
    const float4 v = s_acc[i][d4];
    acc.x += v.x;
    acc.y += v.y;
    acc.z += v.z;
    acc.w += v.w;
  }
  *reinterpret_cast<uint2*>(out) = make_uint2(pack_bf16(acc.x * inv, acc.y * inv), pack_bf16(acc.z * inv, acc.w * inv));
  if (threadIdx.x == 0) p.lse[row] = nan ? NAN : (all == 0.f ? -INFINITY : (base + log2f(all)) * 0.69314718055994530942f);
}

int decode_row_tile(int rows_per_seq) { return rows_per_seq <= 16 ? 16 : (rows_per_seq <= 32 ? 32 : 64); }

cudaError_t decode_attn_setup() {
  cudaError_t e = cudaFuncSetAttribute(rk_decode_attn_kernel<16>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)kSmemBytes);
  if (e == cudaSuccess) e = cudaFuncSetAttribute(rk_decode_attn_kernel<32>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)kSmemBytes);
  if (e == cudaSuccess) e = cudaFuncSetAttribute(rk_decode_attn_kernel<64>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)kSmemBytes);
  return e;
}

cudaError_t launch_decode_attn(const DecodeAttnParams& p, int row_tile, cudaStream_t stream) {
  const dim3 grid((unsigned)p.n_ctas);
  if (row_tile == 16) rk_decode_attn_kernel<16><<<grid, kThreads, kSmemBytes, stream>>>(p);
  else if (row_tile == 32) rk_decode_attn_kernel<32><<<grid, kThreads, kSmemBytes, stream>>>(p);
  else rk_decode_attn_kernel<64><<<grid, kThreads, kSmemBytes, stream>>>(p);
  cudaError_t e = cudaGetLastError();
  if (e != cudaSuccess) return e;
  const int64_t rows = (int64_t)p.n_seqs * p.q_len * p.n_heads;
  rk_decode_join_kernel<<<(unsigned)rows, 512, 0, stream>>>(p, row_tile);
  return cudaGetLastError();
}

}  // namespace rk
