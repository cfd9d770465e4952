// Internal declarations shared by the host layer and the kernel launchers (not part of the ABI).
#pragma once
#include <cuda.h>
#include <cuda_runtime.h>
#include <stdint.h>

#include "rk_ptx.cuh"

namespace rk {

constexpr int kDLatent = 512;
constexpr int kDRope = 64;
constexpr int kDQK = 576;
constexpr int kDV = 128;
constexpr int kGroup = 8;

// ---- attention -----------------------------------------------------------------------
constexpr int kAttnRowsPerCta = 64;    // query rows (token x head pairs) per CTA
constexpr int kAttnRowsPerPair = 128;  // per CTA pair (one UMMA M=128 across two SMs)
constexpr int kAttnKeysPerTile = 256;  // keys per UMMA N

struct AttnWorkItem {
  int32_t tile;    // flattened-row tile index (128 rows each)
  int32_t maxpos;  // largest request position among the tile's rows
};

struct AttnParams {
  CUtensorMap tm_q;   // [n_flat][576] bf16, box 64 cols x 64 rows, 128B swizzle
  CUtensorMap tm_kv;  // [T][576] bf16, box 64 cols x 128 rows, 128B swizzle
  const int32_t* row_pos;    // [T] request position of each packed row
  const int32_t* rowmap;     // [n_tok] token slot -> packed row, or nullptr (identity)
  const int32_t* seg_off;    // [S+1]
  const int32_t* seg_delta;  // [S]
  const float2* seg_cs;      // [S][32] (cos, sin)(delta_i * theta_j)
  const AttnWorkItem* work;  // [n_tiles] cost-descending
  void* O;                   // bf16 [n_flat][512] (output-phase instantiation: [n_flat][576])
  float* lse;                // [n_flat]
  DeviceStatus* status;
  unsigned long long wait_ns;
  int32_t n_segs;
  int32_t n_tiles;
  int32_t n_flat;  // tokens * heads_per_token
  int32_t hpt;     // heads per token in this pass (G or L)
  int32_t n_pairs;
  float scale_log2;  // sm_scale * log2(e)
  int32_t isolated;  // 1: a row sees only its own segment (documents built alone, Algorithm 1)
  int32_t row_base;  // packed row of token slot 0 when rowmap is null
  int32_t n_rows_total;  // T: bound of every packed-row index (read by the bounds-checked build)
  double rope_turns[32];  // theta_j / (2 pi), j = 0..31 (used by the output-phase instantiation only)
};

cudaError_t launch_attention(const AttnParams& p, int n_pairs, bool value_phase, bool starve_loads, cudaStream_t stream);
cudaError_t attention_setup();  // sets the dynamic shared memory attribute once
int attention_max_pairs(int sm_count);

// ---- batched GEMM  C[M,N] = A[M,K] * B[N,K]^T  (bf16 in, fp32 accumulate, bf16 out) ----------
struct GemmBatch {
  int32_t a_col0;   // column offset of this batch's A block
  int32_t b_row0;   // row offset of this batch's B block
  int32_t b_col0;   // column offset of this batch's B block
  int32_t b_skip;   // K index at which a 128-column hole starts in B (or a huge value)
  int32_t c_col0;   // column offset of this batch's C block
  int32_t pad[3];
};

struct GemmParams {
  CUtensorMap tm_a;  // [M rows][a_cols] box 64 x 128
  CUtensorMap tm_b;  // [b_rows][b_cols] box 64 x BN (64 x 128 for the CTA-pair kernel)
  CUtensorMap tm_c;  // [M rows][ldc] box 64 x 128 (epilogue stores)
  void* C;
  const GemmBatch* batches;
  DeviceStatus* status;
  unsigned long long wait_ns;
  int64_t ldc;  // elements
  int32_t M, N, K;
  int32_t n_batches;
};

cudaError_t launch_gemm(const GemmParams& p, int bn, int sm_count, cudaStream_t stream);
cudaError_t gemm_setup();
// single-batch launches with N a multiple of 256 run on CTA pairs; their B tensor map needs a 128-row box
bool gemm_uses_pairs(int M, int N, int n_batches);

// fused sliced first projection of the Global heads: o = O_g W_uv^T stays on chip, z_on_g = o W_a[slice]^T
struct FusedProjParams {
  CUtensorMap tm_a;   // O_g  [M][G * ow]      box 64 x 128
  CUtensorMap tm_b1;  // W_uv [H * 128][ow]    box 64 x 128
  CUtensorMap tm_b2;  // W_a  [G * r_o][1024]  box 64 x 128
  CUtensorMap tm_c;   // z_on_g [M][G * r_o]   box 64 x 128 (stores)
  const GemmBatch* batches_uv;  // per group: a_col0 = g * ow, b_row0 = Global head * 128
  const GemmBatch* batches_wa;  // per group: b_row0 = g * r_o, b_col0 = 128 * slot of the Global head, c_col0 = g * r_o
  DeviceStatus* status;
  unsigned long long wait_ns;
  int32_t M, n_groups, K1, o_rank;
};
cudaError_t launch_proj_fused(const FusedProjParams& p, int sm_count, cudaStream_t stream);
cudaError_t proj_fused_setup();

// ---- streaming kernels -----------------------------------------------------------------------
constexpr int kMergeMaxParts = 4096;  // the merge keeps 8 warps x n_parts weights in shared memory (128 KB at most)
cudaError_t stream_setup();          // raises the merge kernels' dynamic shared memory limit once
cudaError_t launch_relocate(const void* q_rope, int64_t n_rows, int32_t n_heads, int64_t row_stride,
                            int64_t head_stride, const float2* seg_cs, int32_t seg_begin, int32_t seg_end,
                            void* out, int sm_count, cudaStream_t stream);
cudaError_t launch_merge(int32_t n_parts, int64_t n_rh, const void* O_part, int32_t part_dtype,
                         const float* lse_part, void* O, float* lse, int sm_count, cudaStream_t stream);
cudaError_t launch_merge_phase(int32_t n_parts, int64_t n_rows, int32_t n_heads, const void* O_part, int32_t part_dtype,
                               const float* lse_part, const float2* seg_cs, const int32_t* row_pos, const double* rope_turns,
                               void* O, float* lse, int sm_count, cudaStream_t stream);
cudaError_t launch_combine(const void* z_on_g, const void* z_on_l, const void* z_off, const int32_t* inv_map, int64_t T,
                           int64_t width, void* z, int64_t n_prot, DeviceStatus* status, int sm_count, cudaStream_t stream);
cudaError_t launch_check_selftest(DeviceStatus* status, cudaStream_t stream);  // does something in the bounds-checked build only

// ---- selection rules (Eq. protected, Eq. moe) --------------------------------------------------
constexpr uint8_t kPolicyStructural = 1, kPolicyCandidate = 2, kPolicyDirty = 4;

struct PolicyState {
  unsigned n_cand, n_struct_cand, blocks_done, n_top, k_rem, done;
  unsigned long long prefix;  // digits of the n_top-th largest (score,row) key found so far
  unsigned hist[256];
};

struct PolicyParams {
  const int32_t* seg_off;
  const int32_t* seg_delta;
  const uint8_t* seg_has_artifact;
  const float* scores;
  uint8_t* flags;
  PolicyState* state;
  unsigned* block_counts;
  int32_t* rows_out;
  long long* count_out;
  DeviceStatus* status;
  long long req_end, tail_rows;
  int32_t n_segs, T, edge_rows, budget_bp;
};

struct PolicyHost {
  const int32_t* seg_tab_host;  // [seg_off (S+1) | seg_delta (S)]
  const uint8_t* has_host;      // [S]
  int32_t n_segs;
  int64_t T, req_end, tail_rows;
  int32_t edge_rows, budget_bp;
  const int32_t* dirty;
  int64_t n_dirty;
  const float* scores;
  int32_t* rows_out;
  long long* count_out;
  void* workspace;
  DeviceStatus* status;
};

size_t policy_workspace_bytes(int64_t T, int32_t n_segs);
cudaError_t launch_protected_rows(const PolicyHost& h, cudaStream_t stream);
cudaError_t launch_moe_fanout(const float* p, int64_t n, float tau, int fence, uint8_t* k_out, uint8_t* keep_out,
                              cudaStream_t stream);

// ---- 4-bit paged latent cache, single-token attention over it ------------------------------------
constexpr int kCache4PageRows = 64;
constexpr int kCache4Units = 26;  // 16-byte units of a row: 16 of codes, 2 of scales, 8 of rope dims
constexpr int64_t kCache4PageBytes = kCache4Units * kCache4PageRows * 16;
constexpr int kDecodeKeys = 128;   // keys per tile of the decode attention (two pages)
constexpr int kDecodeMaxRows = 64; // query rows (token x head) per row tile
constexpr int kDecodeMaxCtas = 512; // bound of n_ctas (one per SM)
constexpr int kJoinFewParts = 16;   // up to here a row's partial results are joined by one warp

struct Cache4Table {  // device arrays
  const int32_t* seg_len;
  const int32_t* page_off;
  const int32_t* page_ids;
  int64_t n_listed;
  int32_t n_segs;
};

struct RopeTurns {
  double t[32];  // theta_j / (2 pi)
};

constexpr int32_t kDecodePlanMagic = 0x524b4450;
struct DecodePlanHeader {
  int64_t n_pages;
  int32_t magic, n_seqs, q_len, n_items, max_tiles, n_heads;
  int32_t n_tiles;  // key tiles over all sequences
  int32_t n_joins;  // row tiles whose keys several CTAs share
  int32_t chunk;    // tiles per CTA of the attention: CTA i takes [i * chunk, (i + 1) * chunk) of (sequence, row tile, key tile)
};
struct __align__(32) DecodeTile {  // at most 128 keys of one segment, as one sequence sees it
  int32_t page0, page1;  // pages of keys 0-63 and 64-127
  int32_t base;          // request position of key 0
  int32_t n;             // keys some query token of the sequence may see
  int32_t delta;         // request offset of the segment: the queries' rope part is turned by R(-delta)
  int32_t pad[3];
};

struct DecodePlanArgs {
  Cache4Table tab;
  const int32_t* seq_off;     // [n_seqs + 1] into the items
  const int32_t* item_seg;    // [n_items]
  const int32_t* item_delta;  // [n_items]
  const int32_t* q_pos;       // [n_seqs][q_len]
  DecodePlanHeader* header;
  int32_t* pos_out;    // copy of q_pos, limited to -1 .. 2^30
  int32_t* item_tile;  // [n_items + 1]
  int32_t* seq_tile;   // [n_seqs + 1]
  int4* cta_start;     // [n_ctas] (sequence, row tile, key tile, used)
  int4* joins;         // [n_ctas] (sequence * n_row_tiles + row tile, first CTA, parts, work units up to here)
  DecodeTile* tiles;   // [max_tiles]
  DeviceStatus* status;
  int64_t n_pages;
  int32_t n_seqs, q_len, n_items, max_tiles, n_heads, n_row_tiles, n_ctas, row_tile;
};

struct DecodeAttnParams {
  CUtensorMap tm_q;  // [n_seqs * q_len * n_heads][576] bf16, box 64 columns x row-tile rows
  const DecodePlanHeader* header;
  const int32_t* pos;
  const int32_t* seq_tile;
  const int4* cta_start;
  const int4* joins;
  const DecodeTile* tiles;
  const uint8_t* pages;
  const void* q;
  void* O;       // bf16 [rows][512]
  float* lse;    // [rows]
  float* part_o;    // [n_ctas][2][64][512] normalised partial results of rows whose keys several CTAs share
  float* part_lse;  // [n_ctas][2][64] base-2
  DeviceStatus* status;
  uint32_t wait_ns;  // limit of one device-side wait (the low word of the timer: at most 4 s)
  RopeTurns rope;
  int64_t n_pages;
  float scale_log2;
  int32_t n_seqs, q_len, n_items, max_tiles, n_heads, n_row_tiles, n_ctas;
  int32_t starve;  // rk_test_starve_loads: 0, or which signals the test instantiation withholds
};

int decode_row_tile(int rows_per_seq);  // 16, 32 or 64 query rows per CTA
cudaError_t decode_attn_setup();
cudaError_t launch_decode_attn(const DecodeAttnParams& p, int row_tile, cudaStream_t stream);
cudaError_t launch_decode_plan(const DecodePlanArgs& a, cudaStream_t stream);
cudaError_t launch_cache4_append(void* pages, int64_t n_pages, const Cache4Table& tab, const void* c, int64_t c_stride,
                                 const void* k_rope, int64_t r_stride, const int32_t* new_off, int64_t n_new,
                                 const RopeTurns& rope, DeviceStatus* status, cudaStream_t stream);
cudaError_t launch_cache4_read(const void* pages, int64_t n_pages, const Cache4Table& tab, const int32_t* row_off, int64_t n_rows,
                               void* kv, DeviceStatus* status, cudaStream_t stream);

// ---- 4-bit matrix-vector products ----------------------------------------------------------------
struct Matvec4Params {
  const uint4* codes;      // [n_mat][n_out / 16][k / 64][32 lanes]
  const uint32_t* scales;  // [n_mat][n_out / 16][k / group][8] pairs (row g, row g + 8) of bf16
  const void* x;           // bf16, token t at x + t * x_stride: [n_mat][k]
  void* y;                 // token t at y + t * y_stride: [n_mat][n_out]
  int64_t x_stride, y_stride, n_tok;
  int32_t n_mat, n_out, k, group, out_f32;
  // set by the launcher: thread blocks along k, rounds of them, 64-wide blocks of k per thread block; tiles per run, runs per
  // matrix; pipeline depth and shared memory
  int32_t split, passes, slice, run, runs, stages;
  uint32_t stage_bytes, red_bytes;
  DeviceStatus* status;
  unsigned long long wait_ns;
  int32_t starve;  // rk_test_starve_loads
};
cudaError_t launch_quant4(const void* w, int32_t n_mat, int32_t n_out, int32_t k, int32_t group, void* codes, void* scales,
                          cudaStream_t stream);
// slots[i]: clusters of 1 << i thread blocks that run at the same time on the current device
cudaError_t matvec4_setup(int32_t* slots, int sm_count);
cudaError_t launch_matvec4(Matvec4Params p, const int32_t* slots, cudaStream_t stream);

// ---- routing to experts, products in 8-bit integers, sampling --------------------------------------
constexpr int kMaxExperts = 1024;
constexpr int kMaxSlots = 16;      // experts per token
constexpr int kMaxGroups = 32;
constexpr int kMaxVocab = 1 << 20;
constexpr int kMaxK8 = 131072;     // 127^2 k stays below 2^31

struct RouteParams {
  const void* logits;  // [n][n_groups * group_size], rows `stride` elements apart
  const float* bias;   // [n_groups * group_size] or null
  int32_t* ids;        // [n][k]
  float* weights;      // [n][k]
  int64_t n, stride;
  int32_t bf16, softmax, renorm, k, n_groups, group_size, top_groups, group_top;
  float scale;
  // set by the launcher: lanes of a warp per group; tokens of a warp; experts of a lane; whether all lanes have as many, aligned
  int32_t lanes_log2, turns, per, whole;
};
cudaError_t launch_moe_route(RouteParams p, int sm_count, cudaStream_t stream);

struct GroupParams {
  const int32_t* ids;   // [n][k]
  const uint8_t* keep;  // [n] bit s = slot s stays, or null
  int32_t* row_off;     // [n_experts + 1]
  int32_t* rows;        // [n * k]
  int64_t n;
  int32_t k, n_experts;
};
// group_blocks: thread blocks of the cluster that makes long lists
cudaError_t experts_setup(int32_t* group_blocks);
cudaError_t launch_moe_group(const GroupParams& p, int32_t group_blocks, cudaStream_t stream);

struct Matmul8Params {
  CUtensorMap tm_w;      // [n_mat * n_out][k_pad] bytes, box 128 x 128
  CUtensorMap tm_x;      // dense: [token rows][k_pad] bytes, box 128 x tile_rows / 2
  const uint8_t* x;      // by expert: the same rows
  const float* sw;       // [n_mat * n_out]
  const float* sx;       // [token rows]
  const int32_t* row_off;  // by expert: [n_mat + 1] into rows
  const int32_t* rows;     // by expert: [n_tok] pairs; null: dense
  void* y;
  int64_t y_stride;
  DeviceStatus* status;
  unsigned long long wait_ns;
  int32_t n_tok;  // token rows; by expert: pairs (places of the list, rows of y)
  int32_t n_out, k_pad, n_mat, per, out_f32;
  int32_t starve;  // rk_test_starve_loads
  int32_t paired;  // set by the launcher: rows and channels allow 4-byte stores of bf16 pairs
  int32_t tile_rows, split;  // set by rk_matmul8_plan for the dense product: token rows of a tile at most, pairs that share its k
};
// split_slots[i]: clusters of 4 << i thread blocks that run at the same time on the current device, 0 where there is no room for one
cudaError_t matmul8_setup(int32_t* split_slots);
cudaError_t launch_quant8(const void* x, int64_t x_stride, int64_t n_rows, int32_t k, void* codes, float* scales, cudaStream_t stream);
// chooses the dense product's tiles (host arithmetic alone; by a C name, which the tests call)
extern "C" void rk_matmul8_plan(int64_t n_out, int64_t n_tok, int32_t k_pad, int32_t sm_count, const int32_t* split_slots, int32_t* tile_rows,
                                int32_t* split);
cudaError_t launch_matmul8(Matmul8Params p, int sm_count, cudaStream_t stream);

struct SampleParams {
  const void* logits;  // [n][vocab], rows `stride` elements apart
  const float *u, *temperature, *top_p, *min_p;  // [n]; all but u may be null
  const int32_t* top_k;
  int32_t* tokens;  // [n]
  float* probs;     // [n] or null
  int64_t n, stride;
  int32_t vocab, bf16;
  int32_t blocks;  // set by the launcher: thread blocks per row (a cluster)
};
cudaError_t sample_setup();
cudaError_t launch_sample(SampleParams p, int sm_count, cudaStream_t stream);

#ifdef __CUDACC__
// scale byte -> the bf16 value in both halves: 2^((b >> 3) - 20) (1 + (b & 7) / 8); 255 is NaN
__device__ __forceinline__ uint32_t cache4_scale(uint32_t b) {
  const uint32_t v = b == 255u ? 0x7fc0u : (b << 4) + (107u << 7);
  return v * 0x10001u;
}
// four scale bytes -> the bf16 values, each in both halves; 255 comes out as a number here, see cache4_nan_bytes
__device__ __forceinline__ void cache4_scale_quad(uint32_t b, uint32_t* s2) {
  const uint32_t even = (b & 0x00ff00ffu) * 16u + 0x35803580u, odd = ((b >> 8) & 0x00ff00ffu) * 16u + 0x35803580u;
  s2[0] = __byte_perm(even, 0u, 0x1010);
  s2[1] = __byte_perm(odd, 0u, 0x1010);
  s2[2] = __byte_perm(even, 0u, 0x3232);
  s2[3] = __byte_perm(odd, 0u, 0x3232);
}
// the top bit of every byte that is 255
__device__ __forceinline__ uint32_t cache4_nan_bytes(uint32_t b) { return ((b & 0x7f7f7f7fu) + 0x01010101u) & b & 0x80808080u; }
// -24 times a scale, in both halves (exact: 24 has two significant bits)
__device__ __forceinline__ uint32_t cache4_offset(uint32_t scale2) {
  const uint32_t k = 0xc1c0c1c0u;
  const __nv_bfloat162 r = __hmul2(*reinterpret_cast<const __nv_bfloat162*>(&k), *reinterpret_cast<const __nv_bfloat162*>(&scale2));
  return *reinterpret_cast<const uint32_t*>(&r);
}
// Eight 4-bit codes n + 8 times a scale -> eight bf16 values n * scale, exactly: a code in mantissa bits 3-6 of 0x4180
// is the bf16 number 16 + code = 24 + n; one fused product and sum with -24 * scale leaves n * scale, which has at
// most seven significant bits.
__device__ __forceinline__ uint4 cache4_dequant(uint32_t v, uint32_t scale2, uint32_t offset2) {
  uint32_t o[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const uint32_t t = ((i == 0 ? v << 3 : v >> (4 * i - 3)) & 0x00780078u) | 0x41804180u;
    const __nv_bfloat162 r = __hfma2(*reinterpret_cast<const __nv_bfloat162*>(&t), *reinterpret_cast<const __nv_bfloat162*>(&scale2),
                                     *reinterpret_cast<const __nv_bfloat162*>(&offset2));
    o[i] = *reinterpret_cast<const uint32_t*>(&r);
  }
  return make_uint4(o[0], o[1], o[2], o[3]);
}
// (cos, sin) of d * theta_j: the angle is reduced in double in units of turns, so that positions of any size are exact
// to float rounding
__device__ __forceinline__ void rope_cos_sin(const RopeTurns& r, int d, int j, float& c, float& s) {
  const double t = (double)d * r.t[j];
  const float f = (float)(t - rint(t));
  sincospif(2.f * f, &s, &c);
}
#endif

}  // namespace rk
