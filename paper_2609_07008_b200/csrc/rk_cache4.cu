// The 4-bit paged latent cache of the decode step: appending new rows (key rotation and quantisation on the
// way), reading rows back as the packed bf16 stream of the online step, and the plan that the single-token
// attention over the cache (rk_decode.cu) walks.
//
// A cached row is 416 bytes instead of 1152: 512 latent dims as 4-bit codes n in -7..7 (stored as n + 8) with one
// 8-bit scale per 16 dims, and the 64 rope dims in bf16 (the rotated key is what positions hang on).  A scale has
// four significant bits, a code three, so every value n * s has seven and IS a bf16 number: the attention's tensor
// cores take it without a further rounding.  Pages hold 64 rows, unit-major: 26 units of 16 bytes, each a
// contiguous 1 KB block of 64 rows, so that a warp whose lanes are rows reads 512 contiguous bytes per load.
#include <cuda_bf16.h>
#include <math.h>

#include "rk_internal.h"

namespace rk {
namespace {

constexpr int kRowsPerBlock = 32;                 // rows staged per block: 8 warps x 4 rows
constexpr int kUnitStride = kRowsPerBlock * 16 + 16;  // padded: the lanes of a warp write 16 different units

// Largest s in [0, n) with off[s] <= i, found by all lanes of a warp together, 32 probes per round: two dependent
// loads for up to 1024 segments where a binary search takes ten.
__device__ __forceinline__ int warp_find_segment(const int32_t* __restrict__ off, int n, int i) {
  const int lane = threadIdx.x & 31;
  int lo = 0, len = n;  // the answer is in [lo, lo + len)
  while (len > 1) {
    const int step = (len + 31) >> 5;
    const int at = lo + lane * step;
    const bool le = at < lo + len && __ldg(off + at) <= i;
    const unsigned b = __ballot_sync(0xffffffffu, le);
    const int k = b == 0u ? 0 : 31 - __clz((int)b);
    const int end = lo + len;
    lo += k * step;
    len = min(step, end - lo);
  }
  return lo;
}

// Byte addresses in the pages of up to 32 consecutive rows of a ragged batch (the last off[s+1] - off[s] rows of every segment
// s), one per lane of the calling warp, and the rows' indexes in their segments; -1 for no row.  Rows beyond off[n_segs] are no
// rows of the batch and are skipped silently; whatever the tables say is bounds checked, a bad entry is reported and its row
// skipped.  The segments of the first and the last row are found by the warp together; mostly they are the same.
__device__ __forceinline__ int64_t row_addresses(const Cache4Table& t, const int32_t* __restrict__ off, int64_t row0, int64_t n_rows,
                                                 int64_t n_pages, DeviceStatus* st, int* index_in_segment) {
  *index_in_segment = 0;
  if (t.n_segs == 0) return -1;
  const int64_t last = min(min(row0 + 31, n_rows - 1), (int64_t)__ldg(off + t.n_segs) - 1);
  if (row0 > last) return -1;
  int s = warp_find_segment(off, t.n_segs, (int)row0), hi = warp_find_segment(off, t.n_segs, (int)last);
  const int64_t i = row0 + (threadIdx.x & 31);
  if (i > last) return -1;
  while (s < hi) {
    const int mid = (s + hi + 1) >> 1;
    if (__ldg(off + mid) <= i) s = mid;
    else hi = mid - 1;
  }
  const int o0 = __ldg(off + s), o1 = __ldg(off + s + 1), len = __ldg(t.seg_len + s);
  const int p0 = __ldg(t.page_off + s), p1 = __ldg(t.page_off + s + 1);
  const long long j = (long long)len - ((long long)o1 - o0) + (i - o0);
  const long long pi = (long long)p0 + (j >> 6);
  if (i < o0 || j < 0 || j >= len || p0 < 0 || pi >= p1 || pi >= t.n_listed) {
    report_status(st, 4 /*RK_ERR_ROWS*/, RK_CHK_CACHE_ROW, (int)i);
    return -1;
  }
  const int page = __ldg(t.page_ids + pi);
  if (page < 0 || page >= n_pages) {
    report_status(st, 4 /*RK_ERR_ROWS*/, RK_CHK_CACHE_PAGE, page);
    return -1;
  }
  *index_in_segment = (int)j;
  return (int64_t)page * kCache4PageBytes + (j & 63) * 16;
}

// 32 rows per block.  Lane g of a warp owns scale group g of a row (16 dims, 32 contiguous bytes), so the group's
// maximum never leaves the lane.  The finished units are staged in shared memory and leave with the row index
// running fastest: consecutive rows of a page are consecutive 16-byte pieces.
// Rounding: with approximate reciprocals a quotient may sit a hair beside a tie.  No quotient of an 8-bit and a 4-bit
// significand lies closer than 2^-9 to a half-integer without being one, so rounding it to multiples of 2^-11 (adding 6144)
// restores exact ties, and the result is round-half-even of the true quotient.  Likewise max / 7 lies no closer than
// 2^-11 of itself to the middle between two scales without being on it, so 12 of its 24 bits are kept before it is rounded to 4.
// Bound by HBM (1152 bytes in, 416 out per row).  Measured: 64 documents of 1025 to 4096 rows (170k rows) in 44 us
// before their read back, 55 us from cold, issue slots 63 % busy; the floor at 6.5 TB/s is 41 us.  64 single rows: 5 us, start to end of
// a chain of dependent loads (segment, page list, page).
__global__ void __launch_bounds__(256) cache4_append_kernel(uint8_t* __restrict__ pages, int64_t n_pages, Cache4Table tab,
                                                            const __nv_bfloat16* __restrict__ c, int64_t c_stride,
                                                            const __nv_bfloat16* __restrict__ kr, int64_t r_stride,
                                                            const int32_t* __restrict__ new_off, int64_t n_new,
                                                            RopeTurns rope, DeviceStatus* status) {
  __shared__ __align__(16) uint8_t stage[kCache4Units * kUnitStride];
  __shared__ int64_t addr[kRowsPerBlock];
  __shared__ int index[kRowsPerBlock];
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int64_t row0 = (int64_t)blockIdx.x * kRowsPerBlock + warp * 4;
  // all loads of the warp's four rows first; the first warp's search runs under them
  uint4 x[4][2];
#pragma unroll
  for (int r = 0; r < 4; ++r) {
    x[r][0] = x[r][1] = make_uint4(0, 0, 0, 0);
    if (row0 + r < n_new) {
      const uint4* src = reinterpret_cast<const uint4*>(c + (row0 + r) * c_stride + lane * 16);
      x[r][0] = __ldcs(src);
      x[r][1] = __ldcs(src + 1);
    }
  }
  const int rr = lane >> 3, rc = lane & 7;  // rope: lane covers 8 dims of one of the four rows
  uint4 xr = make_uint4(0, 0, 0, 0);
  if (row0 + rr < n_new) xr = __ldcs(reinterpret_cast<const uint4*>(kr + (row0 + rr) * r_stride + rc * 8));
  if (warp == 0) {
    int j;
    addr[lane] = row_addresses(tab, new_off, row0, n_new, n_pages, status, &j);
    index[lane] = j;
  }
#pragma unroll
  for (int r = 0; r < 4; ++r) {
    const uint32_t w[8] = {x[r][0].x, x[r][0].y, x[r][0].z, x[r][0].w, x[r][1].x, x[r][1].y, x[r][1].z, x[r][1].w};
    uint32_t mx = 0u;  // two 15-bit magnitudes at a time: bf16 orders like its bits
#pragma unroll
    for (int e = 0; e < 8; ++e) mx = __vmaxu2(mx, w[e] & 0x7fff7fffu);
    const uint32_t top = max(mx & 0xffffu, mx >> 16);
    const bool finite = top < 0x7f80u;
    uint32_t u = (__float_as_uint(__uint_as_float(top << 16) * (1.0f / 7.0f)) + 0x800u) & ~0xfffu;
    u += 0x7ffffu + ((u >> 20) & 1u);  // round to four significant bits, ties to even
    int code = (int)(u >> 20) - (107 << 3);
    code = finite ? min(max(code, 0), 254) : 255;
    const float inv = __fdividef(1.0f, __uint_as_float((uint32_t)(code + (107 << 3)) << 20));
    float y[16];  // 6144 + x / s
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      y[2 * e] = __fmaf_rn(__uint_as_float(w[e] << 16), inv, 6144.0f);
      y[2 * e + 1] = __fmaf_rn(__uint_as_float(w[e] & 0xffff0000u), inv, 6144.0f);
    }
    // max|c| / scale is at most 7 * 17 / 16 and rounds to 7, unless the scale was limited or the group is NaN
    if (__any_sync(0xffffffffu, code >= 254)) {
#pragma unroll
      for (int e = 0; e < 16; ++e) y[e] = fminf(fmaxf(y[e], 6144.0f - 7.0f), 6144.0f + 7.0f);
    }
    // The float bits of 1.5 * 2^23 + 8 + n are 0x4b400008 + n: eight of them, shifted and summed modulo 2^32, are the
    // packed codes plus a constant.  That keeps the packing on the multiply-add pipe.
    uint2 out = make_uint2(0u, 0u);
#pragma unroll
    for (int e = 0; e < 16; ++e) {
      const float q = __fadd_rn(y[e], 12582920.0f - 6144.0f);
      const uint32_t at = 1u << (4 * ((e & 7) >> 1) + 16 * (e & 1));
      (e < 8 ? out.x : out.y) += (__float_as_uint(q)) * at;
    }
    // 0x4b400000 times the sum of the eight place values
    const uint32_t bias = (uint32_t)(0x4b400000ull * 0x11111111ull);
    out.x -= bias;
    out.y -= bias;
    const int row = warp * 4 + r;
    *reinterpret_cast<uint2*>(stage + (lane >> 1) * kUnitStride + row * 16 + (lane & 1) * 8) = out;
    stage[(16 + ((lane >> 2) & 1)) * kUnitStride + row * 16 + 4 * (lane >> 3) + (lane & 3)] = (uint8_t)code;
  }
  __syncthreads();
  {  // R(j): the stored key is in the position-zero frame of its segment
    const uint32_t in[4] = {xr.x, xr.y, xr.z, xr.w};
    uint32_t o[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      float cs, sn;
      rope_cos_sin(rope, index[warp * 4 + rr], 4 * rc + e, cs, sn);
      const float x0 = __uint_as_float(in[e] << 16), x1 = __uint_as_float(in[e] & 0xffff0000u);
      o[e] = pack_bf16(x0 * cs - x1 * sn, x0 * sn + x1 * cs);
    }
    *reinterpret_cast<uint4*>(stage + (18 + rc) * kUnitStride + (warp * 4 + rr) * 16) = make_uint4(o[0], o[1], o[2], o[3]);
  }
  __syncthreads();
  for (int idx = threadIdx.x; idx < kCache4Units * kRowsPerBlock; idx += 256) {
    const int unit = idx >> 5, row = idx & 31;
    const int64_t a = addr[row];
    if (a >= 0) *reinterpret_cast<uint4*>(pages + a + unit * 1024) = *reinterpret_cast<const uint4*>(stage + unit * kUnitStride + row * 16);
  }
}

// The way back: 32 rows per block.  Units come in with the row index running fastest; then a warp writes a row at a time,
// 16-byte pieces of eight values with the column running fastest (a 32-bit word holds the codes of one piece), so that
// every lane's places in a row are fixed.  Bound by HBM: 262144 rows (109 MB in, 302 out) in 68 us, 92 % of the
// measured copy rate.
__global__ void __launch_bounds__(256) cache4_read_kernel(const uint8_t* __restrict__ pages, int64_t n_pages, Cache4Table tab,
                                                          const int32_t* __restrict__ row_off, int64_t n_rows,
                                                          __nv_bfloat16* __restrict__ kv, DeviceStatus* status) {
  __shared__ __align__(16) uint8_t stage[kCache4Units * kUnitStride];
  __shared__ int64_t addr[kRowsPerBlock];
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int64_t row0 = (int64_t)blockIdx.x * kRowsPerBlock;
  if (warp == 0) {
    int j;
    addr[lane] = row_addresses(tab, row_off, row0, n_rows, n_pages, status, &j);
  }
  __syncthreads();
  {
    const int64_t a = addr[lane];  // unit = warp + 8 i, row = lane
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int unit = warp + 8 * i;
      if (unit < kCache4Units && a >= 0)
        *reinterpret_cast<uint4*>(stage + unit * kUnitStride + lane * 16) = __ldcs(reinterpret_cast<const uint4*>(pages + a + unit * 1024));
    }
  }
  __syncthreads();
  // latent piece q of a row: word q & 3 of unit q >> 2, scale group q >> 1; this lane has pieces lane and lane + 32
  const uint8_t* code_at = stage + (lane >> 2) * kUnitStride + (lane & 3) * 4;
  const int g = lane >> 1;
  const uint8_t* scale_at = stage + (16 + ((g >> 2) & 1)) * kUnitStride + 4 * (g >> 3) + (g & 3);
#pragma unroll
  for (int r = 0; r < 4; ++r) {
    const int row = warp * 4 + r;
    if (addr[row] < 0) continue;
    uint4* dst = reinterpret_cast<uint4*>(kv + (row0 + row) * kDQK) + lane;
#pragma unroll
    for (int half = 0; half < 2; ++half) {
      const uint32_t v = *reinterpret_cast<const uint32_t*>(code_at + row * 16 + half * 8 * kUnitStride);
      const uint32_t s = cache4_scale(scale_at[row * 16 + half * 8]);
      __stcs(dst + 32 * half, cache4_dequant(v, s, cache4_offset(s)));
    }
  }
  const int row = warp * 4 + (lane >> 3);  // rope: eight pieces of each of the four rows
  if (addr[row] >= 0)
    __stcs(reinterpret_cast<uint4*>(kv + (row0 + row) * kDQK) + 64 + (lane & 7),
           *reinterpret_cast<const uint4*>(stage + (18 + (lane & 7)) * kUnitStride + row * 16));
}

// ---- plan -------------------------------------------------------------------------------------------------
// Pass 1 (one block): key tiles of every item (a segment in a sequence) and their running sum.
constexpr int kPlanThreads = 1024;

__global__ void __launch_bounds__(kPlanThreads) decode_plan_scan_kernel(DecodePlanArgs a) {
  __shared__ int warp_sums[32];
  __shared__ long long carry;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  if (tid == 0) carry = 0;
  // Every key lies at 0 or above and below 2^30: a later position sees all there is, a negative one nothing, whichever it is.
  // With both ends limited the sums, differences and comparisons behind stay inside 32 bits.
  for (int i = tid; i < a.n_seqs * a.q_len; i += kPlanThreads) a.pos_out[i] = max(min(a.q_pos[i], 1 << 30), -1);
  __syncthreads();
  for (int base = 0; base < a.n_items; base += kPlanThreads) {
    const int i = base + tid;
    int n = 0;
    if (i < a.n_items) {
      int lo = 0, hi = a.n_seqs - 1;  // largest b with seq_off[b] <= i
      while (lo < hi) {
        const int mid = (lo + hi + 1) >> 1;
        if (__ldg(a.seq_off + mid) <= i) lo = mid; else hi = mid - 1;
      }
      const bool listed = __ldg(a.seq_off + lo) <= i && i < __ldg(a.seq_off + lo + 1);
      const int seg = a.item_seg[i];
      if (seg < 0 || seg >= a.tab.n_segs) {
        if (listed) report_status(a.status, 4, RK_CHK_PLAN_ITEM, i);
      } else if (listed) {
        int pmax = -1;
        for (int t = 0; t < a.q_len; ++t) pmax = max(pmax, a.q_pos[lo * a.q_len + t]);
        const int delta = a.item_delta[i], len = a.tab.seg_len[seg];
        const int p0 = a.tab.page_off[seg], p1 = a.tab.page_off[seg + 1];
        long long seen = (long long)pmax - delta + 1;
        seen = seen < 0 ? 0 : (seen < len ? seen : len);
        const long long np = (seen + 63) >> 6;
        // a pool without pages has no row to see (and no page that a tile with a bad entry could stand on)
        if (delta < 0 || len < 0 || p0 < 0 || (seen > 0 && (p0 + np > p1 || p0 + np > a.tab.n_listed || a.n_pages == 0)) ||
            (long long)delta + len > (1ll << 30)) {
          report_status(a.status, 4, RK_CHK_PLAN_ITEM, i);
        } else {
          // one tile more than fits is as good as any larger number, and keeps the block's sum inside 32 bits
          n = (int)min((seen + 127) >> 7, (long long)a.max_tiles + 1);
        }
      }
    }
    int v = n;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const int y = __shfl_up_sync(0xffffffffu, v, o);
      if (lane >= o) v += y;
    }
    if (lane == 31) warp_sums[warp] = v;
    __syncthreads();
    if (warp == 0) {
      int s = warp_sums[lane];
#pragma unroll
      for (int o = 1; o < 32; o <<= 1) {
        const int y = __shfl_up_sync(0xffffffffu, s, o);
        if (lane >= o) s += y;
      }
      warp_sums[lane] = s;
    }
    __syncthreads();
    const long long before = carry + (warp ? warp_sums[warp - 1] : 0) + v - n;
    if (i < a.n_items) a.item_tile[i] = (int)(before < 0x7fffffff ? before : 0x7fffffff);
    __syncthreads();
    if (tid == kPlanThreads - 1) carry = before + n;
    __syncthreads();
  }
  const long long total = carry;
  const bool fits = total <= a.max_tiles;
  if (tid == 0) {
    if (!fits) report_status(a.status, 6 /*RK_ERR_WORKSPACE*/, RK_CHK_PLAN_ITEM, (int)total);
    a.item_tile[a.n_items] = fits ? (int)total : 0;
    DecodePlanHeader h = {};
    h.magic = kDecodePlanMagic;
    h.n_seqs = a.n_seqs;
    h.q_len = a.q_len;
    h.n_items = a.n_items;
    h.max_tiles = a.max_tiles;
    h.n_heads = a.n_heads;
    h.n_pages = a.n_pages;
    h.n_tiles = fits ? (int)total : 0;
    const long long work = (long long)h.n_tiles * a.n_row_tiles;
    h.chunk = (int)((work + a.n_ctas - 1) / a.n_ctas);
    if (h.chunk < 1) h.chunk = 1;
    *a.header = h;
  }
  __syncthreads();
  for (int b = tid; b <= a.n_seqs; b += kPlanThreads) {
    const int at = a.seq_off[b];
    const bool ok = at >= 0 && at <= a.n_items && (b == 0 || at >= a.seq_off[b - 1]);
    if (!ok) report_status(a.status, 4, RK_CHK_PLAN_ITEM, b);
    // a malformed list makes an empty plan: the running sum below must never decrease
    if (!ok) a.header->n_tiles = 0;
  }
  __syncthreads();
  __threadfence_block();
  const bool empty = *(volatile int*)&a.header->n_tiles == 0;
  for (int b = tid; b <= a.n_seqs; b += kPlanThreads) a.seq_tile[b] = empty ? 0 : a.item_tile[a.seq_off[b]];
  __syncthreads();
  // where every CTA of the attention starts, and which row tiles start in a CTA and go on in the next
  const int chunk = a.header->chunk;
  const long long work = empty ? 0 : (long long)total * a.n_row_tiles;
  auto locate = [&](long long w, int* first) -> int4 {  // (sequence, row tile, key tile) of work item w
    int lo = 0, hi = a.n_seqs - 1;  // largest b with n_row_tiles * seq_tile[b] <= w
    while (lo < hi) {
      const int mid = (lo + hi + 1) >> 1;
      if ((long long)a.seq_tile[mid] * a.n_row_tiles <= w) lo = mid; else hi = mid - 1;
    }
    const int n_b = a.seq_tile[lo + 1] - a.seq_tile[lo];
    const long long rest = w - (long long)a.seq_tile[lo] * a.n_row_tiles;
    *first = n_b;
    return make_int4(lo, (int)(rest / n_b), (int)(rest % n_b), 1);
  };
  int4 join = make_int4(0, 0, 0, 0);
  bool is_join = false;
  if (tid < a.n_ctas) {
    const long long w = (long long)tid * chunk, last = min(w + chunk, work) - 1;
    int n_b;
    a.cta_start[tid] = w < work ? locate(w, &n_b) : make_int4(0, 0, 0, 0);
    if (w < work) {
      const int4 e = locate(last, &n_b);
      const long long begin = last - e.z, end = begin + n_b;  // the row tile that holds this CTA's last key tile
      is_join = begin >= w && end > last + 1;
      if (is_join) {
        const int parts = (int)((end - 1) / chunk) - tid + 1;
        join = make_int4(e.x * a.n_row_tiles + e.y, tid, parts, parts <= kJoinFewParts ? (a.row_tile + 15) / 16 : 2 * a.row_tile);
      }
    }
  }
  // compacted in CTA order, the work units summed up on the way
  const unsigned ballot = __ballot_sync(0xffffffffu, is_join);
  int units = is_join ? join.w : 0;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const int y = __shfl_up_sync(0xffffffffu, units, o);
    if (lane >= o) units += y;
  }
  __shared__ int warp_units[32];
  __syncthreads();
  if (lane == 31) {
    warp_sums[warp] = __popc(ballot);
    warp_units[warp] = units;
  }
  __syncthreads();
  int at = __popc(ballot & ((1u << lane) - 1u)), n_joins = 0;
  for (int i = 0; i < 32; ++i) {
    if (i < warp) {
      at += warp_sums[i];
      units += warp_units[i];
    }
    n_joins += warp_sums[i];
  }
  if (is_join) {
    join.w = units;
    a.joins[at] = join;
  }
  if (tid == 0) a.header->n_joins = n_joins;
}

// Pass 2: one thread per key tile.
__global__ void __launch_bounds__(256) decode_plan_fill_kernel(DecodePlanArgs a) {
  const int t = blockIdx.x * 256 + threadIdx.x;
  const int n_tiles = a.header->n_tiles;
  if (t >= n_tiles) return;
  int lo = 0, hi = a.n_items - 1;  // largest i with item_tile[i] <= t: the last of equal entries owns the tile
  while (lo < hi) {
    const int mid = (lo + hi + 1) >> 1;
    if (a.item_tile[mid] <= t) lo = mid; else hi = mid - 1;
  }
  int b = 0, bh = a.n_seqs - 1;
  while (b < bh) {
    const int mid = (b + bh + 1) >> 1;
    if (a.seq_off[mid] <= lo) b = mid; else bh = mid - 1;
  }
  int pmax = -1;
  for (int k = 0; k < a.q_len; ++k) pmax = max(pmax, a.pos_out[b * a.q_len + k]);
  const int seg = a.item_seg[lo], delta = a.item_delta[lo];
  const int j0 = (t - a.item_tile[lo]) * kDecodeKeys;
  const int seen = min(a.tab.seg_len[seg], pmax - delta + 1);
  const int n = min(seen - j0, kDecodeKeys);
  const int p0 = a.tab.page_off[seg] + (j0 >> 6);
  DecodeTile rec;
  rec.page0 = a.tab.page_ids[p0];
  rec.page1 = n > 64 ? a.tab.page_ids[p0 + 1] : rec.page0;
  rec.base = delta + j0;
  rec.n = n;
  if (rec.page0 < 0 || rec.page0 >= a.n_pages || rec.page1 < 0 || rec.page1 >= a.n_pages) {
    report_status(a.status, 4, RK_CHK_CACHE_PAGE, (rec.page0 < 0 || rec.page0 >= a.n_pages) ? rec.page0 : rec.page1);
    rec.page0 = rec.page1 = rec.n = 0;  // no row of the tile is read; its keys count as unseen
  }
  rec.delta = delta;
  rec.pad[0] = rec.pad[1] = rec.pad[2] = 0;
  a.tiles[t] = rec;
}

}  // namespace

cudaError_t launch_cache4_append(void* pages, int64_t n_pages, const Cache4Table& tab, const void* c, int64_t c_stride,
                                 const void* k_rope, int64_t r_stride, const int32_t* new_off, int64_t n_new,
                                 const RopeTurns& rope, DeviceStatus* status, cudaStream_t stream) {
  const int64_t blocks = (n_new + kRowsPerBlock - 1) / kRowsPerBlock;
  cache4_append_kernel<<<(unsigned)blocks, 256, 0, stream>>>(static_cast<uint8_t*>(pages), n_pages, tab,
                                                             static_cast<const __nv_bfloat16*>(c), c_stride,
                                                             static_cast<const __nv_bfloat16*>(k_rope), r_stride, new_off, n_new,
                                                             rope, status);
  return cudaGetLastError();
}

cudaError_t launch_cache4_read(const void* pages, int64_t n_pages, const Cache4Table& tab, const int32_t* row_off, int64_t n_rows,
                               void* kv, DeviceStatus* status, cudaStream_t stream) {
  const int64_t blocks = (n_rows + kRowsPerBlock - 1) / kRowsPerBlock;
  cache4_read_kernel<<<(unsigned)blocks, 256, 0, stream>>>(static_cast<const uint8_t*>(pages), n_pages, tab, row_off, n_rows,
                                                           static_cast<__nv_bfloat16*>(kv), status);
  return cudaGetLastError();
}

cudaError_t launch_decode_plan(const DecodePlanArgs& a, cudaStream_t stream) {
  decode_plan_scan_kernel<<<1, kPlanThreads, 0, stream>>>(a);
  cudaError_t e = cudaGetLastError();
  if (e != cudaSuccess) return e;
  if (a.max_tiles == 0) return cudaSuccess;
  decode_plan_fill_kernel<<<(unsigned)((a.max_tiles + 255) / 256), 256, 0, stream>>>(a);
  return cudaGetLastError();
}

}  // namespace rk
