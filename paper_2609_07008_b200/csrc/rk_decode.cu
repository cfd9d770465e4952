// Absorbed-MLA attention of single tokens (or a few drafted ones) over the 4-bit paged latent cache:
//   per document segment i:  q_i = R(-delta_i) q;   S = q_i K_i^T;   O = softmax over all segments' keys, times C.
//
// A decode step has few query rows (q_len * heads of one sequence) and many keys, so the products are issued with
// the KEYS in the M = 128 dimension of the tensor cores and the query rows in N = 16, 32 or 64:
//   S^T[128 keys x N]   = K[128 x 576] Q^T          9 chunks of 64 dims, A K-major, B K-major
//   O^T[512 dims x N]  += C^T[512 x 128] P^T        4 tiles of 128 dims, A MN-major, B MN-major
// With the rows in M a 64-row tile would run the tensor cores at half rate (M = 64) and 16 rows at an eighth.
//
// Dequantisation happens between the HBM load and the operands: 256 threads, two per key, hold the next tile's codes and
// scales in registers (37 KB in flight per SM) and turn them into the bf16 values n * s, which are exact.  They go into
// tensor memory as the A operand of the scores (a lane is a key; 128 dims per slot, two slots); the softmax warps copy them
// from there into shared memory as the A operand of the values (128 keys x 64 dims per 16 KB chunk, 128-byte swizzle).  The
// keys' rope chunk is bf16 in the pages, whose units of 64 rows x 16 bytes are the unswizzled K-major operand as they are:
// it is copied into its place by bulk copies, into the space that P^T takes over once the scores are done.
// An M = 128, N = 64 product takes 33 clk with the keys in tensor memory and 49 with both operands in shared memory
// (6 KB at 128 B/clk): 3000 clk of products per tile.
// One tile's values (128 KB), the queries (80 KB) and P^T (16 KB) fill the shared memory, so the value chunks are
// refilled pair by pair as the products release them.  The scores do not wait for that: the keys of the next pair
// are already in tensor memory, and the products of the next tile's first half run under this tile's softmax.
//
// What bounds it: a tile takes some 5000 clk, of which the tensor core works 3000 (37 % of the kernel's cycles with start
// and end), the ALUs 42 % and the issue slots 46 %.  The rest is the chain from tile to tile: value products -> free chunks
// -> copied values and free key slots -> last scores -> softmax -> value products, each step at the speed that eight warps
// get beside the others.  Measured: 64 requests with 64 heads over 440k visible rows 101 us, one request over 262144 rows
// 62 us (112 MB of pages in: 1.8 TB/s), 16 requests with two tokens of 128 heads 218 us (694 TFLOP/s), 8 tiles 15 us.
// Rows that do not fill their row tile are slower, see write_p: one request over 262144 rows 64 us with 24 heads, 54 with 32, 78
// with 48, 61 with 64, 133 with 72, 104 with 128.
// Tried and slower: the keys through shared memory only (more operand traffic, 1.1x), the key warps writing the values
// (they then wait for the value products, 1.07x), four key warps of twice the registers (1.25x), the register split of
// setmaxnreg (its small share spilled, 1.03x to 1.8x), unrolled copies and products (instruction cache, 1.03x to 1.15x).
//
// Statistics: running maximum per query row in shared memory, raised only when a tile exceeds it by more than 2^8
// (then O^T is rescaled in tensor memory, columns = rows of the query); sums per (key lane, row) in registers in
// fp32, added up over the lanes once per row tile.  P is rounded to bf16 for the tensor cores (at most 2^-8 of each
// key's, averaged by the sum); the turned query rope goes in as two bf16 parts, high and low (2^-16 together):
// the log-sum-exp is an fp32 output, and one part alone moves a logit by 1e-3.  A key with a NaN scale has finite values
// and a NaN flag beside its tile, which the softmax turns into a NaN score: rows whose mask leaves the key out stay clean.
//
// Work: the plan lists every (sequence, row tile, key tile) in order and gives each CTA an equal run of them.  A
// row tile whose keys several CTAs share leaves normalised fp32 partial results and their log-sum-exp, which a
// second kernel joins in CTA order (no atomics: results do not depend on timing).
//
// Warps (640 threads): 0 issues the MMAs, 1 and 3 load the queries (TMA) and turn their rope part, 2 loads the keys' rope
// part, 4-11 load and dequantise keys, 12-19 softmax, correction and epilogue.
#include <cuda_bf16.h>

#include <type_traits>

#include "../../include/rk.h"
#include "rk_internal.h"

namespace rk {
namespace {

constexpr int kThreads = 640;      // x 96 registers: shared memory takes nearly all of L1, so a spilled register in a loop comes back from L2
constexpr int kKeyWarps = 8, kKeyWarp0 = 4, kSoftWarp0 = kKeyWarp0 + kKeyWarps;
constexpr int kSoftWarps = 8, kSoftmax = 32 * kSoftWarps;
constexpr uint32_t kKChunk = 16384;  // 128 keys x 64 dims bf16
constexpr uint32_t kQChunk = 8192;   // up to 64 rows x 64 dims bf16

constexpr uint32_t kOffQ = 0;                        // 8 latent chunks, then the turned rope chunk: high and low parts
constexpr uint32_t kOffV = 10 * kQChunk;             // 8 latent chunks of the keys
constexpr uint32_t kOffP = kOffV + 8 * kKChunk;      // rope chunk of the keys until the scores are done, then P^T
constexpr uint32_t kOffBars = kOffP + kKChunk;
// every one of them has one phase per tile (B_QFULL: per group)
enum { B_QFULL = 0, B_QROPE = 1, B_KROPE = 2, B_KFULL = 3 /*4*/, B_KFREE = 7 /*4*/, B_SFULL = 11, B_PREADY = 12, B_PVDONE = 13 /*4*/,
       B_COUNT = 17 };
constexpr uint32_t kOffTmem = kOffBars + B_COUNT * 8;
constexpr uint32_t kOffAbort = kOffTmem + 4;
constexpr uint32_t kOffFlag = kOffTmem + 8;          // int: 1 + the last tile some row's maximum has to be raised for
constexpr uint32_t kOffMax = kOffBars + 160;         // float [64]: running maximum of each row, base-2 units
constexpr uint32_t kOffPos = kOffMax + 256;          // int [64]: request position of each row (-1: no row)
constexpr uint32_t kOffRed = kOffPos + 256;          // float [4][64]: per lane quarter
constexpr uint32_t kOffAlpha = kOffRed + 1024;       // float [64]: factor of the last raise of a row's maximum
constexpr uint32_t kOffNan = kOffAlpha + 256;         // uint8 [2][2][128]: tile parity, half of the key's groups, key: a scale is NaN
constexpr uint32_t kOffGroup = kOffNan + 512;         // int [8]: the softmax warps' group, see there
constexpr uint32_t kSmemUsed = kOffGroup + 32;
constexpr uint32_t kSmemBytes = kSmemUsed;

// tensor memory columns: O^T takes 4 x N from 0; two score buffers; two slots of 128 dims of the keys (bf16 pairs)
constexpr uint32_t kColS = 256, kColK = 384;
constexpr float kNoMax = -1e30f;     // "no key seen yet": finite, so that differences stay defined

enum { W_QFULL = 41, W_QROPE, W_KROPE, W_KFULL, W_KFREE, W_SFULL, W_PREADY, W_PVDONE };

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
  // put away in shared memory and taken from there
  __device__ Cursor(const DecodeAttnParams& p_, const volatile int* at)
      : p(p_), left(at[0]), b(at[1]), rt(at[2]), tile(at[3]), n_b(at[5]), tile0(at[6]), cnt(at[4]) {}
  __device__ void store(volatile int* at) const {
    at[0] = left;
    at[1] = b;
    at[2] = rt;
    at[3] = tile;
    at[4] = cnt;
    at[5] = n_b;
    at[6] = tile0;
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
};

__device__ __forceinline__ float fast_exp2(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}

// Column results over the lanes of a warp: lane i gets column i mod N of the N (8, 16 or 32) that every lane holds.  Each exchange
// halves the columns a lane holds, N - 1 of them in all where a reduction per column takes 5 N.
template <int N, typename Op>
__device__ __forceinline__ float over_lanes(float (&x)[N], int lane, Op op) {
#pragma unroll
  for (int w = N / 2; w >= 1; w /= 2) {
    const bool upper = (lane & w) != 0;
#pragma unroll
    for (int i = 0; i < w; ++i) {
      const float keep = upper ? x[i + w] : x[i], give = upper ? x[i] : x[i + w];
      x[i] = op(keep, __shfl_xor_sync(0xffffffffu, give, w));
    }
  }
#pragma unroll
  for (int w = N; w < 32; w *= 2) x[0] = op(x[0], __shfl_xor_sync(0xffffffffu, x[0], w));
  return x[0];
}

__device__ __forceinline__ void prefetch_page(const uint8_t* page) {
  asm volatile("cp.async.bulk.prefetch.L2.global [%0], %1;" ::"l"(page), "r"((uint32_t)kCache4PageBytes) : "memory");
}

// Shared-memory operand descriptors as their low words (start address and leading byte offset); the high word, stride
// 1024 bytes, version 1 and 128-byte swizzle, is the same for every operand here.
constexpr uint32_t kDescHi = (1024u >> 4) | (1u << 14) | (2u << 29);
__device__ __forceinline__ uint32_t desc_lo(uint32_t addr, uint32_t lbo) { return ((addr & 0x3FFFFu) >> 4) | ((lbo >> 4) << 16); }
// the keys' rope chunk as it is in the pages: 8 rows x 16 bytes contiguous, the next 8 rows 128 bytes on, no swizzle
constexpr uint32_t kDescHiPlain = (128u >> 4) | (1u << 14);
__device__ __forceinline__ void mma_ss(uint32_t d, uint32_t a, uint32_t a_hi, uint32_t b, uint32_t idesc, uint32_t accumulate) {
  asm volatile(
      "{\n\t.reg .pred p;\n\t.reg .b64 da, db;\n\t"
      "mov.b64 da, {%1, %6};\n\tmov.b64 db, {%2, %5};\n\t"
      "setp.ne.b32 p, %4, 0;\n\t"
      "tcgen05.mma.cta_group::1.kind::f16 [%0], da, db, %3, p;\n\t}"
      ::"r"(d), "r"(a), "r"(b), "r"(idesc), "r"(accumulate), "r"(kDescHi), "r"(a_hi)
      : "memory");
}
__device__ __forceinline__ void mma_ts(uint32_t d, uint32_t a_tmem, uint32_t b, uint32_t idesc, uint32_t accumulate) {
  asm volatile(
      "{\n\t.reg .pred p;\n\t.reg .b64 db;\n\t"
      "mov.b64 db, {%2, %5};\n\t"
      "setp.ne.b32 p, %4, 0;\n\t"
      "tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], db, %3, p;\n\t}"
      ::"r"(d), "r"(a_tmem), "r"(b), "r"(idesc), "r"(accumulate), "r"(kDescHi)
      : "memory");
}

__device__ __forceinline__ void bulk_load(uint32_t dst, const void* src, uint32_t bytes, uint32_t bar) {
  asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];" ::"r"(dst), "l"(src),
               "r"(bytes), "r"(bar)
               : "memory");
}
__device__ __forceinline__ uint32_t globaltimer_lo() {
  uint32_t t;
  asm volatile("mov.u32 %0, %globaltimer_lo;" : "=r"(t));
  return t;
}
__device__ __forceinline__ uint32_t load_shared(uint32_t at) {
  uint32_t v;
  asm volatile("ld.volatile.shared.u32 %0, [%1];" : "=r"(v) : "r"(at) : "memory");
  return v;
}
__device__ __forceinline__ void load_shared4(float* r, uint32_t at) {
  asm volatile("ld.shared.v4.f32 {%0, %1, %2, %3}, [%4];" : "=f"(r[0]), "=f"(r[1]), "=f"(r[2]), "=f"(r[3]) : "r"(at) : "memory");
}
__device__ __forceinline__ void store_shared4(uint32_t at, const uint32_t* r) {
  asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(at), "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]) : "memory");
}
__device__ __forceinline__ void store_shared(uint32_t at, uint32_t v) {
  asm volatile("st.volatile.shared.u32 [%0], %1;" ::"r"(at), "r"(v) : "memory");
}
__device__ __forceinline__ void put(uint32_t* r, const uint4& v) {
  r[0] = v.x;
  r[1] = v.y;
  r[2] = v.z;
  r[3] = v.w;
}

}  // namespace

// kStarve: test instantiation in which the signals of one kind of barrier (p.starve) are withheld, so that whoever waits for them gives
// up.  Nothing is withheld that memory accesses depend on.
template <int kRows, bool kStarve>
__global__ void __launch_bounds__(kThreads, 1) rk_decode_attn_kernel(const __grid_constant__ DecodeAttnParams p) {
  extern __shared__ __align__(1024) uint8_t smem[];
  const uint32_t smem_base = smem_u32(smem);
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  auto bar = [&](int i) -> uint32_t { return smem_base + kOffBars + 8u * i; };
  auto fed = [&](int what) -> bool { return !kStarve || p.starve != what; };
  volatile uint32_t* tmem_ptr = reinterpret_cast<volatile uint32_t*>(smem + kOffTmem);
  // Bounded wait of a whole warp on one of the barriers, kept short: it is inlined two dozen times, and the kernel's loops have
  // to stay in the instruction cache.  The word at kOffAbort is the tag of the first wait that ran out (reported once, at the
  // end), after which everyone gives up.  The lanes look at the barrier, the word and the clock one by one, so the warp votes:
  // it goes on together or gives up together, as what follows a wait are operations of all its lanes.  The votes cost 2 % (64
  // requests 98.7 -> 100.8 us); fewer of them, with the roles going on to the end of a tile on unfinished data, won 1 % back.
  auto wait = [&](int b, uint32_t parity, int where) -> bool {
    const uint32_t at = smem_base + kOffBars + 8u * (uint32_t)b;
    uint32_t t0 = 0u;
    bool done = true;
#pragma unroll 1
    for (uint32_t n = 1; !mbar_try_wait(at, parity); ++n) {
      if ((n & 63u) != 0u) continue;
      const uint32_t now = globaltimer_lo();
      if (n == 64u) t0 = now;
      const bool late = now - t0 > p.wait_ns;
      done = !late && load_shared(smem_base + kOffAbort) == 0u;
      if (late) store_shared(smem_base + kOffAbort, (uint32_t)where);
      if (!done) break;
    }
    return __all_sync(0xffffffffu, done);
  };

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
    store_shared(smem_base + kOffAbort, 0u);
    mbar_init(bar(B_QFULL), 1);
    mbar_init(bar(B_QROPE), 2);
    mbar_init(bar(B_KROPE), 1);
    for (int i = 0; i < 4; ++i) {
      mbar_init(bar(B_KFULL + i), kKeyWarps);
      mbar_init(bar(B_KFREE + i), 1 + kSoftWarps);
      mbar_init(bar(B_PVDONE + i), 1);
    }
    mbar_init(bar(B_SFULL), 1);
    mbar_init(bar(B_PREADY), 1);
    *reinterpret_cast<volatile int*>(smem + kOffFlag) = 0;
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
  // All 512 columns are this block's, so they start at 0; a constant keeps the MMA operands out of vector registers.
  constexpr uint32_t tmem = 0u;
  if (*tmem_ptr != tmem || (smem_base & 1023u) != 0u) {  // cannot happen; nothing has been started yet
    if (threadIdx.x == 0) report_status(p.status, 8 /*RK_ERR_CUDA*/, RK_CHK_PLAN_MATCH, (int)*tmem_ptr);
    __syncthreads();
    if (warp == 0) tmem_dealloc<1>(*tmem_ptr, 512);
    return;
  }
  const int rows_per_seq = p.q_len * p.n_heads;

  if (warp == 0) {
    // ------------------------------ MMA issue (whole warp loops, one elected lane issues) ----------------------
    // Scores of a tile come in five pieces: four times 128 dims as the keys reach tensor memory, then rope.  The first two
    // run under the softmax of the tile before, the rest behind its value products.  The order is fixed and the products come in
    // long batches: the tensor core's queue holds only a few products, so whatever this warp does between two batches beyond some
    // 150 clocks leaves it idle.  And everything is kept small: with the pieces and their descriptors unrolled the role spilled, and
    // every reload cost the tensor core an L2 latency.
    constexpr uint32_t id_qk = umma_idesc_bf16(128, kRows, 0, 0);
    constexpr uint32_t id_pv = umma_idesc_bf16(128, kRows, 1, 1);
    uint32_t t = 0, groups = 0;  // tiles and groups so far: their parities are the barriers' phases
    bool ok = true;
    // 128 dims of tile tq, slot i & 1.  The reduction turns the loop's counters into uniform values for the compiler, as the
    // products' operands have to be.
    auto piece = [&](int i, uint32_t tq) {
      ok = ok && wait(B_KFULL + i, tq & 1u, W_KFULL);
      if (!ok) return;
      tc_fence_after_sync();
      const uint32_t w = __reduce_max_sync(0xffffffffu, (uint32_t)i | ((tq & 1u) << 3)), iu = w & 3u;
      const uint32_t ts = tmem + kColS + (w >> 3) * 64u, tk = tmem + kColK + (iu & 1u) * 64u;
      const uint32_t db = desc_lo(smem_base + kOffQ, 16) + 2u * iu * (kQChunk >> 4);
      if (elect_one()) {
#pragma unroll
        for (int s = 0; s < 8; ++s)
          mma_ts(ts, tk + 8u * s, db + (uint32_t)(((s >> 2) * kQChunk + (s & 3) * 32) >> 4), id_qk, s > 0 ? 1u : iu);
        if (fed(RK_STARVE_KEYS_FREE)) umma_commit_1(bar(B_KFREE) + 8u * iu);
      }
      __syncwarp();
    };
    for (Cursor c(p); ok && c.next(); ++groups) {
      ok = wait(B_QFULL, groups & 1u, W_QFULL);
#pragma unroll 1
      for (int k = -1; ok && k < c.cnt; ++k) {
        if (k >= 0) {  // what is left of this tile's scores
#pragma unroll 1
          for (int i = 2; i < 4; ++i) piece(i, t);
          ok = ok && wait(B_QROPE, t & 1u, W_QROPE) && wait(B_KROPE, t & 1u, W_KROPE);
          if (!ok) break;
          tc_fence_after_sync();
          const uint32_t ts = tmem + kColS + __reduce_max_sync(0xffffffffu, t & 1u) * 64u;
          if (elect_one()) {
            const uint32_t da = desc_lo(smem_base + kOffP, 2048), db = desc_lo(smem_base + kOffQ + 8 * kQChunk, 16);
#pragma unroll
            for (int s = 0; s < 8; ++s)  // the same 64 dims of the keys against the high and the low part of the turned queries
              mma_ss(ts, da + (uint32_t)(((s & 3) * 4096) >> 4), kDescHiPlain, db + (uint32_t)(((s >> 2) * kQChunk + (s & 3) * 32) >> 4), id_qk, 1u);
            if (fed(RK_STARVE_SCORES)) umma_commit_1(bar(B_SFULL));
          }
          __syncwarp();
        }
        if (k + 1 < c.cnt) {  // the first half of the next tile's (the next group has other queries)
#pragma unroll 1
          for (int i = 0; i < 2; ++i) piece(i, k < 0 ? t : t + 1u);
        }
        if (k < 0) continue;
        ok = ok && wait(B_PREADY, t & 1u, W_PREADY);
        if (!ok) break;
        tc_fence_after_sync();
        if (elect_one()) {
          const uint32_t db = desc_lo(smem_base + kOffP, 16);
          uint32_t da = desc_lo(smem_base + kOffV, kKChunk);
#pragma unroll 1
          for (int m = 0; m < 4; ++m, da += (2 * kKChunk) >> 4) {  // 128 dims each: two 64-dim chunks, 16 KB apart
#pragma unroll
            for (int s = 0; s < 8; ++s)
              mma_ss(tmem + (uint32_t)(m * kRows), da + (uint32_t)((s * 2048) >> 4), kDescHi, db + (uint32_t)((s * 2048) >> 4), id_pv,
                     s > 0 ? 1u : (uint32_t)k);
            if (fed(RK_STARVE_VALUES)) umma_commit_1(bar(B_PVDONE) + 8u * (uint32_t)m);
          }
        }
        __syncwarp();
        ++t;
      }
    }
  } else if (warp == 1 || warp == 3) {
    // ------------------------------ queries: latent chunks by TMA, rope chunk turned by R(-delta) -------------
    // Two warps, eight rows apiece in turn; the rope parts stay in registers for the group, so that a new segment costs
    // arithmetic and no loads (from memory row by row, a new segment held the scores up for 10000 clk).
    uint32_t t = 0, groups = 0;
    bool ok = true;
    const int rc = lane & 7, r_first = (lane >> 3) + (warp == 3 ? 4 : 0);
    for (Cursor c(p); ok && c.next(); ++groups) {
      const int row0 = c.b * rows_per_seq + c.rt * kRows;
      const int valid = min(rows_per_seq - c.rt * kRows, kRows);
      int d = __ldg(&p.tiles[c.record(0)].delta);
      uint4 raw[kRows / 8];
      {
        const __nv_bfloat16* src = static_cast<const __nv_bfloat16*>(p.q) + ((int64_t)row0 + r_first) * kDQK + kDLatent + rc * 8;
#pragma unroll
        for (int i = 0; i < kRows / 8; ++i)
          raw[i] = r_first + 8 * i < valid ? __ldg(reinterpret_cast<const uint4*>(src + (int64_t)(8 * i) * kDQK)) : make_uint4(0, 0, 0, 0);
      }
      // the previous group's scores are done with the query chunks (its last tile's S is complete)
      if (t > 0) ok = wait(B_SFULL, (t - 1) & 1u, W_SFULL);
      if (!ok) break;
      if (warp == 1 && fed(RK_STARVE_QUERIES) && elect_one()) {
        mbar_arrive_expect_tx(bar(B_QFULL), 8 * kRows * 128);
        for (int d = 0; d < 8; ++d) tma_load_2d(smem_base + kOffQ + d * kQChunk, &p.tm_q, bar(B_QFULL), d * 64, row0);
      }
      __syncwarp();
      int delta = -1;
      for (int k = 0; ok && k < c.cnt; ++k, ++t) {
        if (k > 0) d = __ldg(&p.tiles[c.record(k)].delta);
        if (k > 0) ok = wait(B_SFULL, (t - 1) & 1u, W_SFULL);
        if (!ok) break;
        if (d != delta) {
          delta = d;
          float cos_of, sin_of, cs[4], sn[4];  // each lane one of the 32 angles, then this lane's four
          rope_cos_sin(p.rope, d, lane, cos_of, sin_of);
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            cs[e] = __shfl_sync(0xffffffffu, cos_of, 4 * rc + e);
            sn[e] = __shfl_sync(0xffffffffu, sin_of, 4 * rc + e);
          }
          uint8_t* dst = smem + kOffQ + 8 * kQChunk + sw128_offset((uint32_t)r_first, (uint32_t)rc);
#pragma unroll 1
          for (int i = 0; i < kRows / 8; ++i, dst += 1024) {  // the rows go round in the registers: one copy of the code
            const uint4 now = raw[0];
#pragma unroll
            for (int n = 0; n + 1 < kRows / 8; ++n) raw[n] = raw[n + 1];
            raw[kRows / 8 - 1] = now;
            const uint32_t in[4] = {now.x, now.y, now.z, now.w};
            uint32_t o[4], lo[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              const float x0 = __uint_as_float(in[e] << 16), x1 = __uint_as_float(in[e] & 0xffff0000u);
              const float y0 = x0 * cs[e] + x1 * sn[e], y1 = x1 * cs[e] - x0 * sn[e];
              o[e] = pack_bf16(y0, y1);
              lo[e] = pack_bf16(y0 - __uint_as_float(o[e] << 16), y1 - __uint_as_float(o[e] & 0xffff0000u));
            }
            *reinterpret_cast<uint4*>(dst) = make_uint4(o[0], o[1], o[2], o[3]);
            *reinterpret_cast<uint4*>(dst + kQChunk) = make_uint4(lo[0], lo[1], lo[2], lo[3]);
          }
          fence_proxy_async_smem();
        }
        __syncwarp();
        if (lane == 0 && fed(RK_STARVE_QUERY_ROPE)) mbar_arrive(bar(B_QROPE));
      }
    }
  } else if (warp == 2) {
    // ------------------------------ keys' rope chunk: straight into the operand's place -----------------------
    // A page holds 64 rows x 16 bytes per unit, which is the unswizzled K-major operand: 1 KB copies of a unit of a page.
    uint32_t t = 0;
    bool ok = true;
    for (Cursor c(p); ok && c.next();) {
      for (int k = 0; k < c.cnt; ++k, ++t) {
        if (k + 2 < c.cnt && lane < 2) {  // pages of the tile after next into L2, where its loads will find them
          const int4 v = *reinterpret_cast<const int4*>(&p.tiles[c.record(k + 2)]);
          if (v.w > 64 * lane + 32) prefetch_page(p.pages + (int64_t)(lane == 0 ? v.x : v.y) * kCache4PageBytes);
        }
        const int4 v = __ldg(reinterpret_cast<const int4*>(&p.tiles[c.record(k)]));
        const uint32_t page0 = __reduce_max_sync(0xffffffffu, (uint32_t)v.x), page1 = __reduce_max_sync(0xffffffffu, (uint32_t)v.y);
        const uint32_t both = __reduce_max_sync(0xffffffffu, v.w > 64 ? 1u : 0u);  // uniform, as the copies' operands have to be
        const uint8_t* src0 = p.pages + (int64_t)page0 * kCache4PageBytes + 18 * 1024;
        const uint8_t* src1 = p.pages + (int64_t)page1 * kCache4PageBytes + 18 * 1024;
        if (t > 0) ok = wait(B_PVDONE + 3, (t - 1) & 1u, W_PVDONE);  // P^T of the last tile has been read
        if (!ok) break;
        // rows that are not there keep what is in their place: their scores are masked
        if (fed(RK_STARVE_LOADS) && elect_one()) {
          mbar_arrive_expect_tx(bar(B_KROPE), both != 0u ? 16384u : 8192u);
#pragma unroll
          for (int u = 0; u < 8; ++u) bulk_load(smem_base + kOffP + u * 2048, src0 + u * 1024, 1024u, bar(B_KROPE));
          if (both != 0u) {
#pragma unroll
            for (int u = 0; u < 8; ++u) bulk_load(smem_base + kOffP + u * 2048 + 1024, src1 + u * 1024, 1024u, bar(B_KROPE));
          }
        }
        __syncwarp();
      }
    }
  } else if (warp < kSoftWarp0) {
    // ------------------------------ keys: HBM -> registers (4-bit) -> tensor memory (bf16) --------------------
    // Two threads per key: thread h has chunk 2 m + h (64 dims, two units) of every 128 dims m and the scale unit h (one word per
    // chunk).
    const int h = (warp - kKeyWarp0) >> 2;
    const int row = 32 * (warp & 3) + lane;  // a warp reaches the tensor memory lanes of its quarter
    const uint32_t t_k = tmem + ((uint32_t)(32 * (warp & 3)) << 16) + kColK + 32u * h;
    uint32_t code[32], scl[4];
    const uint8_t* src = p.pages;  // this key's first unit in the tile being loaded
    // A row behind the last key of its tile is read like any other (its page is in the pool): whatever it holds becomes finite
    // values, its scores are masked, and 0 times a value adds nothing to O.
    auto load_pair = [&](int m) {
#pragma unroll
      for (int e = 0; e < 2; ++e) put(code + 8 * m + 4 * e, __ldg(reinterpret_cast<const uint4*>(src + h * 2048 + (4 * m + e) * 1024)));
    };
    auto load_scale = [&]() { put(scl, __ldg(reinterpret_cast<const uint4*>(src + h * 1024 + 16 * 1024))); };
    uint32_t t = 0;
    bool ok = true;
    Cursor c(p);
    bool more = c.next();
    int k = 0;
    int page = 0;  // of the tile after the one in registers, fetched a tile ahead
    auto fetch = [&]() {  // moves the cursor on and fetches that record
      if (++k >= c.cnt) {
        more = c.next();
        k = 0;
      }
      if (more) {
        page = __ldg(&p.tiles[c.record(k)].page0 + (row >> 6));
      }
    };
    auto open = [&]() { src = p.pages + (int64_t)page * kCache4PageBytes + (row & 63) * 16; };
    bool here = more;  // there is a tile in registers
    if (more) {
      k = -1;
      fetch();
      open();
#pragma unroll
      for (int m = 0; m < 4; ++m) load_pair(m);
      load_scale();
      fetch();
    }
    while (here) {
      const bool next = more;
      if (next) open();
      // A group whose scale is NaN (byte 255) makes the key's scores NaN, and with them every output that sees the key; the values
      // stay numbers, so that rows that do not see it are untouched.
      const bool nan = (cache4_nan_bytes(scl[0]) | cache4_nan_bytes(scl[1]) | cache4_nan_bytes(scl[2]) | cache4_nan_bytes(scl[3])) != 0u;
#pragma unroll
      for (int m = 0; m < 4; ++m) {
        uint32_t v[32];  // 64 dims of this key
        {
          uint32_t s2[4];
          cache4_scale_quad(scl[m], s2);
#pragma unroll
          for (int g = 0; g < 4; ++g) {
            const uint32_t o2 = cache4_offset(s2[g]);
            put(v + 8 * g, cache4_dequant(code[8 * m + 2 * g], s2[g], o2));
            put(v + 8 * g + 4, cache4_dequant(code[8 * m + 2 * g + 1], s2[g], o2));
          }
        }
        // the next tile's loads go out as the registers become free: they have a whole tile's time to arrive
        if (next) {
          load_pair(m);
          if (m == 3) {
            load_scale();
            fetch();
          }
        }
        // the slot may be overwritten once its last content has been multiplied and copied
        ok = m >= 2 ? wait(B_KFREE + m - 2, t & 1u, W_KFREE) : (t == 0 || wait(B_KFREE + m + 2, (t - 1u) & 1u, W_KFREE));
        if (!ok) break;
        tc_fence_after_sync();
        if (m == 0) smem[kOffNan + (t & 1u) * 256u + (uint32_t)(h * 128 + row)] = nan ? 1 : 0;
        tmem_st_x32(t_k + (m & 1) * 64u, v);
        tmem_wait_st();
        tc_fence_before_sync();
        __syncwarp();
        if (lane == 0 && fed(RK_STARVE_KEYS)) mbar_arrive(bar(B_KFULL + m));
      }
      if (!ok) break;
      ++t;
      here = next;
    }
  } else {
    // ------------------------------ softmax, correction, epilogue ---------------------------------------------
    // Thread = one key of the tile (TMEM lane) and half of the query rows (columns).
    constexpr int NC = kRows / 2;
    const int q = warp & 3;            // TMEM lane quarter
    const int c0 = ((warp - kSoftWarp0) >> 2) * NC;
    const int key = 32 * q + lane;
    const uint32_t lane_base = (uint32_t)(32 * q) << 16;
    const uint32_t t_s0 = tmem + lane_base + kColS + (uint32_t)c0;
    const uint32_t t_o = tmem + lane_base + (uint32_t)c0;
    float* s_max = reinterpret_cast<float*>(smem + kOffMax);
    int* s_pos = reinterpret_cast<int*>(smem + kOffPos);
    float* s_red = reinterpret_cast<float*>(smem + kOffRed);
    float* s_alpha = reinterpret_cast<float*>(smem + kOffAlpha);
    volatile int* s_flag = reinterpret_cast<volatile int*>(smem + kOffFlag);
    const int tid = threadIdx.x - 32 * kSoftWarp0;
    const uint32_t max_at = smem_base + kOffMax + 4u * c0;
    uint32_t t = 0;
    bool ok = true;
    // The values of tile tv: copied from tensor memory, where the key warps put them for the scores, into shared memory,
    // chunk pair by chunk pair as the previous tile's products release the space.  Here and not in the key warps, which
    // thereby never wait for the value products; the softmax warps have nothing else to do while those run.
    auto copy_values = [&](uint32_t tv) -> bool {
      const uint32_t v_row = smem_base + kOffV + (c0 ? 1 : 0) * kKChunk + key * 128 + ((key & 7) << 4);
#pragma unroll 1
      for (int m = 0; m < 4; ++m) {
        if (!wait(B_KFULL + m, tv & 1u, W_KFULL)) return false;
        tc_fence_after_sync();
        uint32_t v[32];
        __syncwarp();
        tmem_ld_x32(tmem + lane_base + kColK + (m & 1) * 64u + (c0 ? 32u : 0u), v);
        tmem_wait_ld();
        tc_fence_before_sync();
        __syncwarp();
        if (lane == 0) mbar_arrive(bar(B_KFREE + m));
        if (tv > 0 && !wait(B_PVDONE + m, (tv - 1) & 1u, W_PVDONE)) return false;
#pragma unroll
        for (int e = 0; e < 8; ++e)
          store_shared4((v_row + 2 * m * kKChunk) ^ (e << 4), v + 4 * e);  // rows are 128 bytes apart and aligned
      }
      return true;
    };
    // The cursor lives in shared memory, moved on by one thread, as the registers are full: tiles left, sequence, row tile, first
    // tile, its tiles, the sequence's tiles, its first record; the last word says that there is a group.
    volatile int* s_group = reinterpret_cast<volatile int*>(smem + kOffGroup);
    if (tid == 0) {
      Cursor c(p);
      s_group[7] = c.next();
      c.store(s_group);
    }
    named_barrier_sync(1, kSoftmax);
    while (ok && s_group[7] != 0) {
      // s_max, s_pos: every warp is done with the previous group (the barrier in its epilogue)
      int pmin = 0x7fffffff;
      for (int i = 0; i < p.q_len; ++i) pmin = min(pmin, p.pos[s_group[1] * p.q_len + i]);
      if (tid < kRows) {
        const int r = s_group[2] * kRows + tid;
        s_max[tid] = kNoMax;
        s_pos[tid] = r < rows_per_seq ? p.pos[s_group[1] * p.q_len + r / p.n_heads] : -1;
      }
      const int cnt = s_group[4];
      const DecodeTile* rec_at = p.tiles + (s_group[6] + s_group[3]);
      named_barrier_sync(1, kSoftmax);
      float l[NC];
#pragma unroll
      for (int i = 0; i < NC; ++i) l[i] = 0.f;
      int2 ahead = *reinterpret_cast<const int2*>(&rec_at->base);  // first key position and keys of a tile, fetched a tile ahead
      for (int k = 0; ok && k < cnt; ++k, ++t) {
        const int2 rec = ahead;
        const bool full = rec.y == kDecodeKeys && pmin - rec.x + 1 >= kDecodeKeys;  // no key of the tile is masked
        const uint32_t t_s = t_s0 + (t & 1u) * 64u;
        // p = 2^(score - max), eight rows at a time: added to the sums and written as P^T, one 128-byte row per key,
        // query rows contiguous.  `masked`: with masks, and with the sums corrected after a raise (see below).  Returns the largest
        // exponent.
        auto write_p = [&](auto masked, bool raised, float scale) -> float {
          constexpr bool kMasked = decltype(masked)::value;
          const int at = key < rec.y ? rec.x + key : 0x7fffffff;
          const float add = raised && k > 0 ? 0.f : 1.f;
          float top = 0.f;
          const uint32_t dst = smem_base + kOffP + key * 128 + (((c0 / 8) ^ (key & 7)) << 4);
#pragma unroll
          for (int i = 0; i < NC; i += 8) {
            uint32_t s[8], pk[4];
            tmem_ld_x8(t_s + (uint32_t)i, s);
            tmem_wait_ld();
#pragma unroll
            for (int j = 0; j < 8; j += 4) {
              float mx[4], al[4] = {1.f, 1.f, 1.f, 1.f}, pv[4];
              int4 last = make_int4(0, 0, 0, 0);
              load_shared4(mx, max_at + 4u * (i + j));
              if constexpr (kMasked) {
                if (raised) load_shared4(al, max_at + (kOffAlpha - kOffMax) + 4u * (i + j));
                last = *reinterpret_cast<const int4*>(s_pos + c0 + i + j);
              }
              const int lasts[4] = {last.x, last.y, last.z, last.w};
#pragma unroll
              for (int n = 0; n < 4; ++n) {
                float e = fmaf(__uint_as_float(s[j + n]), scale, -mx[n]);
                if (kMasked && at > lasts[n]) e = -INFINITY;
                pv[n] = fast_exp2(e);
                if constexpr (!kMasked) l[i + j + n] += pv[n];
                else {
                  const float old = l[i + j + n];  // a NaN in it stays, see below
                  l[i + j + n] = al[n] < 1e-27f && old == old ? pv[n] : fmaf(old, al[n], add * pv[n]);
                }
              }
              top = fmaxf(top, fmaxf(fmaxf(pv[0], pv[1]), fmaxf(pv[2], pv[3])));
              pk[j / 2] = pack_bf16(pv[0], pv[1]);
              pk[j / 2 + 1] = pack_bf16(pv[2], pv[3]);
            }
            store_shared4(dst ^ (uint32_t)((i / 8) << 4), pk);  // c0 / 8 and i / 8 have no bits in common
          }
          fence_proxy_async_smem();
          return top;
        };
        ok = copy_values(t);
        if (k + 1 < cnt) ahead = *reinterpret_cast<const int2*>(&(++rec_at)->base);
        ok = ok && wait(B_SFULL, t & 1u, W_SFULL);
        tc_fence_after_sync();
        const uint8_t* s_nan = smem + kOffNan + (t & 1u) * 256u + key;
        const float scale = s_nan[0] | s_nan[128] ? NAN : p.scale_log2;
        // First try with the maxima as they are (S of this tile is complete, so P^T of the previous one has been read).
        // A warp that finds an exponent above 8, or that gave up waiting, raises the flag; everyone sees it behind
        // the barrier.  Not tried for the first tile of a group, which has no maxima yet.  A column without a query row never gets
        // one: unmasked, its p are infinite (nobody reads them), and every full tile of a short row tile is gone over twice.
        float top = INFINITY;
        if (k > 0 && ok) top = full ? write_p(std::false_type(), false, scale) : write_p(std::true_type(), false, scale);
        if (top > 256.f) *s_flag = (int)t + 1;
        tc_fence_before_sync();
        named_barrier_sync(1, kSoftmax);
        if (*s_flag == (int)t + 1) {
          ok = named_barrier_and(2, kSoftmax, ok);  // a warp that gave up must not leave the others in a barrier
          if (!ok) break;
          // exact maxima of the tile; a row's maximum is raised where the tile exceeds it by more than 2^8
          {
            const int at = key < rec.y ? rec.x + key : 0x7fffffff;
            float v[NC];
#pragma unroll
            for (int i = 0; i < NC; i += 8) tmem_ld_x8(t_s + (uint32_t)i, reinterpret_cast<uint32_t*>(v) + i);
            tmem_wait_ld();
#pragma unroll
            for (int i = 0; i < NC; i += 4) {
              const int4 last = *reinterpret_cast<const int4*>(s_pos + c0 + i);
              v[i] = at > last.x ? -INFINITY : v[i] * scale;
              v[i + 1] = at > last.y ? -INFINITY : v[i + 1] * scale;
              v[i + 2] = at > last.z ? -INFINITY : v[i + 2] * scale;
              v[i + 3] = at > last.w ? -INFINITY : v[i + 3] * scale;
            }
            const float top_of = over_lanes(v, lane, [](float a, float b) { return fmaxf(a, b); });  // leaves NaN out
            if (lane < NC) s_red[q * 64 + c0 + lane] = top_of;
          }
          named_barrier_sync(1, kSoftmax);
          bool raise = false;
          if (tid < kRows) {
            const float v = fmaxf(fmaxf(s_red[tid], s_red[64 + tid]), fmaxf(s_red[128 + tid], s_red[192 + tid]));
            const float old = s_max[tid];
            raise = v > old + 8.f;
            s_alpha[tid] = raise ? fast_exp2(old - v) : 1.f;
            if (raise) s_max[tid] = v;
          }
          if (named_barrier_or(1, kSoftmax, raise) && k > 0) {  // S of this tile is complete, so every value product before it is too
#pragma unroll 1
            for (int i0 = 0; i0 < 4 * NC; i0 += 8) {
              const uint32_t col = (uint32_t)(i0 / NC * kRows + i0 % NC);
              uint32_t o[8];
              tmem_ld_x8(t_o + col, o);
              tmem_wait_ld();
#pragma unroll
              for (int i = 0; i < 8; ++i) o[i] = __float_as_uint(__uint_as_float(o[i]) * s_alpha[c0 + i0 % NC + i]);
              tmem_st_x8(t_o + col, o);
            }
            tmem_wait_st();
          }
          // Where the first try was made, the sums already hold this tile's p against the old maximum, and the factor makes
          // them right for the new one; otherwise this tile's p are added here.
          // Where the maximum rose by more than 2^90 (or there was none) they may have overflowed: there, what was
          // summed up before is below 2^-60 of the new sum and is dropped - unless it is a NaN, which is the row's for good: the
          // first tiles of a row may hold nothing but NaN scores, which leave the maximum where it was.
          write_p(std::true_type(), true, scale);
          tc_fence_before_sync();
          named_barrier_sync(1, kSoftmax);
        }
        if (tid == 0 && fed(RK_STARVE_WEIGHTS)) mbar_arrive(bar(B_PREADY));
      }
      if (!ok) break;
      // ---- epilogue of the group: sums over the key lanes, then O^T / l ----
      ok = wait(B_PVDONE + 3, (t - 1) & 1u, W_PVDONE);
      ok = named_barrier_and(2, kSoftmax, ok);
      if (!ok) break;
      tc_fence_after_sync();
      const float sum_of = over_lanes(l, lane, [](float a, float b) { return a + b; });
      if (lane < NC) s_red[q * 64 + c0 + lane] = sum_of;
      named_barrier_sync(1, kSoftmax);
      const int first_row = s_group[2] * kRows;
      const bool whole = s_group[4] == s_group[5];
      const int slot = 2 * blockIdx.x + (s_group[3] > 0 ? 0 : 1);
      const int valid = min(rows_per_seq - first_row, kRows);
      const int64_t row0 = (int64_t)s_group[1] * rows_per_seq + first_row;
      if (tid < kRows) {
        // a NaN score makes its row NaN; a row without visible keys has the sum 0
        const float tot = (s_red[tid] + s_red[64 + tid]) + (s_red[128 + tid] + s_red[192 + tid]);
        const float lse2 = tot == 0.f ? -INFINITY : s_max[tid] + log2f(tot);
        s_alpha[tid] = tot == 0.f ? 0.f : 1.f / tot;
        if (!whole) p.part_lse[(int64_t)slot * 64 + tid] = lse2;
        else if (tid < valid) p.lse[row0 + tid] = lse2 * 0.69314718055994530942f;
      }
      named_barrier_sync(1, kSoftmax);
      constexpr int kCols = NC;
#pragma unroll 1
      for (int m = 0; m < 4; ++m) {  // 128 dims each
        const int r = c0;
        uint32_t o[kCols];
        if constexpr (kCols == 8) tmem_ld_x8(t_o + (uint32_t)(m * kRows), o);
        else if constexpr (kCols == 16) tmem_ld_x16(t_o + (uint32_t)(m * kRows), o);
        else tmem_ld_x32(t_o + (uint32_t)(m * kRows), o);
        tmem_wait_ld();
        const int dim = 128 * m + key;
        if (whole) {
          __nv_bfloat16* out = static_cast<__nv_bfloat16*>(p.O) + (row0 + r) * kDLatent + dim;
#pragma unroll
          for (int i = 0; i < kCols; ++i)
            if (r + i < valid) out[i * kDLatent] = __float2bfloat16_rn(__uint_as_float(o[i]) * s_alpha[r + i]);
        } else {
          float* out = p.part_o + ((int64_t)slot * 64 + r) * kDLatent + dim;
#pragma unroll
          for (int i = 0; i < kCols; ++i)
            if (r + i < valid) out[i * kDLatent] = __uint_as_float(o[i]) * s_alpha[r + i];
        }
      }
      tc_fence_before_sync();
      named_barrier_sync(1, kSoftmax);  // s_group, s_red, s_max and s_pos may be overwritten from here on
      if (tid == 0) {
        Cursor c(p, s_group);
        s_group[7] = c.next();
        c.store(s_group);
      }
      named_barrier_sync(1, kSoftmax);
    }
  }

  // ------------------------------ teardown -------------------------------------------------------------------
  __syncwarp();
  tc_fence_before_sync();
  __syncthreads();
  // Looked at once every role is done: the epilogue's wait can run out after the other roles have left.  Copies and products in
  // flight then get a bounded time to finish.
  if (load_shared(smem_base + kOffAbort) != 0u) {
    if (threadIdx.x == 0) report_timeout(p.status, (int)load_shared(smem_base + kOffAbort), 0);
    for (int i = 0; i < 64; ++i) __nanosleep(1000);
  }
  if (warp == 0) {
    __syncwarp();
    tmem_dealloc<1>(tmem, 512);
  }
}

// Joins the partial results of row tiles whose keys several CTAs share, in CTA order: lse = log2 sum 2^lse_j,
// O = sum 2^(lse_j - lse) O_j.  The plan lists those row tiles (at most one per CTA) with a running count of work units,
// which the blocks take in turn.  Few parts (a batch: two or three): a unit is 16 rows, one per warp.  Many parts (one
// long request: up to one per CTA): a unit is half a row; eight groups of 64 threads take every eighth part, 16 bytes
// each, so that the 2 KB rows of many parts are in flight at once.  Rows of sequences that see nothing get O = 0,
// lse = -inf; rows that one CTA finished alone are already written.
constexpr int kJoinThreads = 512;
__global__ void __launch_bounds__(kJoinThreads) rk_decode_join_kernel(const __grid_constant__ DecodeAttnParams p, int row_tile) {
  const DecodePlanHeader* h = p.header;
  if (h->magic != kDecodePlanMagic || h->n_seqs != p.n_seqs || h->q_len != p.q_len || h->n_items != p.n_items ||
      h->max_tiles != p.max_tiles || h->n_heads != p.n_heads || h->n_pages != p.n_pages)
    return;  // reported by the attention kernel
  __shared__ float s_w[kDecodeMaxCtas];
  __shared__ float4 s_acc[7][64];
  __shared__ float s_red[32];
  const int rows_per_seq = p.q_len * p.n_heads;
  const int tid = threadIdx.x, lane = tid & 31;
  for (int b = blockIdx.x; b < p.n_seqs; b += gridDim.x) {
    if (p.seq_tile[b + 1] != p.seq_tile[b]) continue;
    uint4* out = reinterpret_cast<uint4*>(static_cast<__nv_bfloat16*>(p.O) + (int64_t)b * rows_per_seq * kDLatent);
    for (int i = tid; i < rows_per_seq * (kDLatent / 8); i += kJoinThreads) out[i] = make_uint4(0, 0, 0, 0);
    for (int i = tid; i < rows_per_seq; i += kJoinThreads) p.lse[(int64_t)b * rows_per_seq + i] = -INFINITY;
  }
  const int n_joins = h->n_joins;
  const int n_units = n_joins > 0 ? p.joins[n_joins - 1].w : 0;
  for (int unit = blockIdx.x; unit < n_units; unit += gridDim.x) {
    int lo = 0, hi = n_joins - 1;  // first join whose running count exceeds the unit
    while (lo < hi) {
      const int mid = (lo + hi) >> 1;
      if (p.joins[mid].w > unit) hi = mid; else lo = mid + 1;
    }
    const int4 j = p.joins[lo];  // (sequence, row tile), first CTA, parts, units so far
    const int n = j.z, at = unit - (lo > 0 ? p.joins[lo - 1].w : 0), b = j.x / p.n_row_tiles, rt = j.x - b * p.n_row_tiles;
    // a part is in slot 1 of the CTA that starts the row tile, in slot 0 of the ones that go on with it
    auto slot = [&](int i) -> int64_t { return (int64_t)2 * (j.y + i) + (i == 0 ? 1 : 0); };
    if (n <= kJoinFewParts) {
      const int col = 16 * at + (tid >> 5), r = rt * row_tile + col;
      if (r < rows_per_seq) {
        const int64_t row = (int64_t)b * rows_per_seq + r;
        const float mine = lane < n ? __ldg(p.part_lse + slot(lane) * 64 + col) : -INFINITY;
        float mx = mine;
        for (int o = 16; o > 0; o >>= 1) mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, o));
        const float base = mx == -INFINITY ? 0.f : mx;
        const float w = lane < n ? exp2f(mine - base) : 0.f;  // a NaN stays one; an empty part has the weight 0
        float sum = w;
        for (int o = 16; o > 0; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
        const float inv = sum == 0.f ? 0.f : 1.f / sum;
        float4 acc[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) acc[e] = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 2
        for (int i = 0; i < n; ++i) {
          const float wi = __shfl_sync(0xffffffffu, w, i);
          const float4* src = reinterpret_cast<const float4*>(p.part_o + (slot(i) * 64 + col) * kDLatent) + lane;
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const float4 v = __ldg(src + 32 * e);
            acc[e].x = fmaf(wi, v.x, acc[e].x);
            acc[e].y = fmaf(wi, v.y, acc[e].y);
            acc[e].z = fmaf(wi, v.z, acc[e].z);
            acc[e].w = fmaf(wi, v.w, acc[e].w);
          }
        }
        uint2* out = reinterpret_cast<uint2*>(static_cast<__nv_bfloat16*>(p.O) + row * kDLatent) + lane;
#pragma unroll
        for (int e = 0; e < 4; ++e) out[32 * e] = make_uint2(pack_bf16(acc[e].x * inv, acc[e].y * inv), pack_bf16(acc[e].z * inv, acc[e].w * inv));
        if (lane == 0) p.lse[row] = sum == 0.f ? -INFINITY : (base + log2f(sum)) * 0.69314718055994530942f;
      }
      continue;
    }
    const int col = at >> 1, half = at & 1, r = rt * row_tile + col;
    if (r >= rows_per_seq) continue;
    const int part = tid >> 6, d4 = tid & 63;
    const int64_t row = (int64_t)b * rows_per_seq + r;
    const float mine = tid < n ? __ldg(p.part_lse + slot(tid) * 64 + col) : -INFINITY;
    float mx = mine, sum = 0.f;
    for (int o = 16; o > 0; o >>= 1) mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, o));
    if (lane == 0) s_red[tid >> 5] = mx;
    __syncthreads();
    mx = s_red[0];
    for (int i = 1; i < kJoinThreads / 32; ++i) mx = fmaxf(mx, s_red[i]);
    const float base = mx == -INFINITY ? 0.f : mx;
    const float w = tid < n ? exp2f(mine - base) : 0.f;
    if (tid < n) s_w[tid] = w;
    sum = w;
    for (int o = 16; o > 0; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
    if (lane == 0) s_red[16 + (tid >> 5)] = sum;
    __syncthreads();
    sum = s_red[16];
    for (int i = 1; i < kJoinThreads / 32; ++i) sum += s_red[16 + i];
    float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 8
    for (int i = part; i < n; i += 8) {
      const float wi = s_w[i];
      const float4 v = __ldg(reinterpret_cast<const float4*>(p.part_o + (slot(i) * 64 + col) * kDLatent + half * 256) + d4);
      acc.x = fmaf(wi, v.x, acc.x);
      acc.y = fmaf(wi, v.y, acc.y);
      acc.z = fmaf(wi, v.z, acc.z);
      acc.w = fmaf(wi, v.w, acc.w);
    }
    if (part > 0) s_acc[part - 1][d4] = acc;
    __syncthreads();
    if (part == 0) {
#pragma unroll
      for (int i = 0; i < 7; ++i) {
        const float4 v = s_acc[i][d4];
        acc.x += v.x;
        acc.y += v.y;
        acc.z += v.z;
        acc.w += v.w;
      }
      const float inv = sum == 0.f ? 0.f : 1.f / sum;
      __nv_bfloat16* out = static_cast<__nv_bfloat16*>(p.O) + row * kDLatent + half * 256 + d4 * 4;
      *reinterpret_cast<uint2*>(out) = make_uint2(pack_bf16(acc.x * inv, acc.y * inv), pack_bf16(acc.z * inv, acc.w * inv));
      if (tid == 0 && half == 0) p.lse[row] = sum == 0.f ? -INFINITY : (base + log2f(sum)) * 0.69314718055994530942f;
    }
    __syncthreads();
  }
}

int decode_row_tile(int rows_per_seq) { return rows_per_seq <= 16 ? 16 : (rows_per_seq <= 32 ? 32 : 64); }

namespace {
using DecodeKernel = void (*)(const DecodeAttnParams);
DecodeKernel decode_kernel(int row_tile, bool starve) {
  if (row_tile == 16) return starve ? rk_decode_attn_kernel<16, true> : rk_decode_attn_kernel<16, false>;
  if (row_tile == 32) return starve ? rk_decode_attn_kernel<32, true> : rk_decode_attn_kernel<32, false>;
  return starve ? rk_decode_attn_kernel<64, true> : rk_decode_attn_kernel<64, false>;
}
}  // namespace

cudaError_t decode_attn_setup() {
  cudaError_t e = cudaSuccess;
  for (int row_tile = 16; row_tile <= 64 && e == cudaSuccess; row_tile *= 2)
    e = cudaFuncSetAttribute(decode_kernel(row_tile, false), cudaFuncAttributeMaxDynamicSharedMemorySize, (int)kSmemBytes);
  return e;
}

cudaError_t launch_decode_attn(const DecodeAttnParams& p, int row_tile, cudaStream_t stream) {
  const dim3 grid((unsigned)p.n_ctas);
  const DecodeKernel kernel = decode_kernel(row_tile, p.starve != 0);
  if (p.starve != 0) {  // set up here, so that creating a context does not load the test's instantiations
    cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)kSmemBytes);
    if (e != cudaSuccess) return e;
  }
  kernel<<<grid, kThreads, kSmemBytes, stream>>>(p);
  cudaError_t e = cudaGetLastError();
  if (e != cudaSuccess) return e;
  rk_decode_join_kernel<<<(unsigned)(2 * p.n_ctas), kJoinThreads, 0, stream>>>(p, row_tile);
  return cudaGetLastError();
}

}  // namespace rk
