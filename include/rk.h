/* rk.h -- C ABI of the B200 (sm_100a) MLA-Online step of RedKnot-MLA.
 *
 * One online layer (Algorithm 2 "Relocate, recompute, and merge one online layer"):
 *   for every document segment i:  q_i = R(-delta_i) q;  SelectiveMLA(q_i, C_i, A)
 *   SegmentedLSEMerge over segments;  z_online = W_{a,G} O_G + W_{a,L} O_{L,A};
 *   z = RestoreAndReplace(z_off, z_online, A);  y = W_b z.
 *
 * Conventions
 *  - Every function returns an rk_status (0 = RK_OK) and never throws.  All argument errors
 *    are found on the host before anything is enqueued.  rk_last_error() gives a message.
 *  - "device" pointers are CUDA device memory owned by the caller; "host" pointers are
 *    ordinary host memory that is copied during the call and not retained.
 *  - bf16 tensors are passed as `const void*` holding 16-bit bfloat16 (the bits of
 *    torch.bfloat16 / __nv_bfloat16); all tensors are dense row-major, innermost dimension
 *    contiguous, base pointers 16-byte aligned.
 *  - Rows are in PACKED order: document 0, 1, ..., then the query suffix -- the order of the
 *    packed latent stream.  Packed row r of segment i sits at request position
 *    pos[r] = seg_delta[i] + (r - seg_off[i]).  Row t sees key k iff pos[k] <= pos[t].
 *  - `stream` is a cudaStream_t (0 = default stream).  Calls enqueue work and return; the
 *    only blocking calls are rk_create / rk_request_create / rk_poll_status / *_destroy and
 *    rk_layer_host.  The decode calls and those behind them can be captured into a CUDA graph.
 *  - The library allocates device memory only inside rk_create and rk_request_create (small
 *    tables) and frees it in the matching destroy.  kv, weights and z_off are never written.
 *  - No kernel traps: a device-side wait that expires records RK_ERR_TIMEOUT in a status
 *    word, the kernel drains and returns; rk_poll_status() reads (and clears) that word.
 *  - There is no fallback: rk_create fails with RK_ERR_UNSUPPORTED on a device that is not
 *    compute capability 10.x.
 */
#ifndef RK_H_
#define RK_H_

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef enum rk_status {
  RK_OK = 0,
  RK_ERR_NULL = 1,        /* a required pointer is NULL */
  RK_ERR_PROFILE = 2,     /* head/group geometry inconsistent */
  RK_ERR_LAYOUT = 3,      /* segment table invalid */
  RK_ERR_ROWS = 4,        /* protected-row list invalid */
  RK_ERR_ALIGN = 5,       /* pointer or stride not 16-byte aligned */
  RK_ERR_WORKSPACE = 6,   /* workspace too small */
  RK_ERR_UNSUPPORTED = 7, /* dims / device not supported */
  RK_ERR_CUDA = 8,        /* a CUDA call failed */
  RK_ERR_TIMEOUT = 9      /* a bounded device-side wait expired */
} rk_status;

/* Head partition and projection geometry (Eq. partition; Section "DeepSeek-V4 Flash and Pro
 * profiles": one Global head per native group of eight).  Supported: group_size 8,
 * d_latent 512, d_rope 64, d_v 128; o_rank and d_model multiples of 128. */
typedef struct rk_profile {
  int32_t n_heads;              /* H */
  int32_t n_groups;             /* G = H / group_size */
  int32_t group_size;           /* 8 */
  int32_t d_latent;             /* 512: width of the shared latent c (also the value width) */
  int32_t d_rope;               /* 64 */
  int32_t d_v;                  /* 128: per-head width after W_uv */
  int32_t o_rank;               /* r_o: rows of each group's block of W_a */
  int32_t d_model;              /* rows of W_b */
  float sm_scale;               /* softmax scale applied to q.k */
  float rope_base;              /* theta_j = rope_base^(-2j/d_rope), interleaved pairs */
  const int32_t* global_heads;  /* host [n_groups]: absolute index of each group's Global head,
                                   global_heads[g] / group_size == g */
} rk_profile;

/* Segment geometry of one request (Section "Online position restoration and segmented
 * merge"): document i was built at positions 0..n_i-1 and appears at request offset
 * seg_delta[i].  Request-position intervals must not overlap; gaps are legal. */
typedef struct rk_layout {
  int32_t n_segs;
  const int64_t* seg_off;          /* host [n_segs+1], packed-row prefix sums, seg_off[0] = 0 */
  const int64_t* seg_delta;        /* host [n_segs], >= 0 */
  const uint8_t* seg_has_artifact; /* host [n_segs]; 0 = no offline artifact (all its rows must be protected) */
} rk_layout;

typedef struct rk_request_info {
  int64_t n_rows;        /* T */
  int64_t n_prot;        /* A */
  int64_t n_off_rows;    /* rows the z_off tensor must have (end of the last segment with artifact) */
  int64_t pairs_global;  /* visible (row,key) pairs summed over rows: T(T+1)/2 for gap-free layouts */
  int64_t pairs_local;   /* visible pairs summed over protected rows */
  int32_t n_tiles_global;
  int32_t n_tiles_local;
} rk_request_info;

typedef struct rk_ctx rk_ctx;
typedef struct rk_request rk_request;

const char* rk_version(void);
const char* rk_status_string(rk_status s);

/* Creates a context on the CURRENT CUDA device.  Copies the profile (including global_heads). */
rk_status rk_create(const rk_profile* profile, rk_ctx** out);
/* Output-phase variant (Eq. offonline: z = W_a R^{-1}(O); Algorithm 2: RestorePhase(O_i, delta_i) per
 * segment before SegmentedLSEMerge and R^{-1} in the z_online statement).  With RK_VALUE_PHASE the
 * value of a key is its whole stored row [c | k_rope] (576 wide), not the latent alone, so an
 * attention output carries 64 rotated dims.  Inside a segment they accumulate in the document's
 * position-zero frame; RestorePhase turns them by R(+seg_delta[i]) into the request frame, where
 * segments may be merged; R^{-1} turns row t's merged rope dims by R(-pos[t]), after which they
 * depend on relative positions only.  The attention kernel does all three inside its running merge.
 * What changes at the interface, and nothing else:
 *   O_g / O_l (and O_part / O of rk_segmented_merge_phase) rows are 576 wide, rope dims last;
 *   W_uv is [H][128][576];  rk_mla_off_build applies R^{-1} at the row's canonical position.
 * The plain context (flags = 0) treats both maps as the identity: its values carry no rotated dims. */
#define RK_VALUE_PHASE 1u
rk_status rk_create_ex(const rk_profile* profile, uint32_t flags, rk_ctx** out);
rk_status rk_destroy(rk_ctx* ctx);
/* Message of the last failing call on this context (valid until the next call). */
const char* rk_last_error(const rk_ctx* ctx);
/* Synchronises `stream`, returns the device status word and clears it: RK_OK, RK_ERR_TIMEOUT, RK_ERR_ROWS (a bad
 * entry in the tables of a decode call or of the experts' products, or a report of the bounds-checked build), RK_ERR_WORKSPACE or RK_ERR_LAYOUT
 * (a decode plan that is too small, or made for another call).  The first report wins. */
rk_status rk_poll_status(rk_ctx* ctx, void* stream);
/* Per-wait time limit of device-side waits, in milliseconds (default 2000). */
rk_status rk_set_wait_limit_ms(rk_ctx* ctx, int32_t ms);
/* Test hook for the timeout path (failure detection without a GPU fault): while `on` is non-zero the
 * attention launches of this context use an instantiation whose load warp leaves every ring stage
 * empty, so the consumers' bounded waits expire, the kernel drains and returns, and
 * rk_poll_status() reports RK_ERR_TIMEOUT.  Results are not produced while it is on.  Use it
 * together with a short rk_set_wait_limit_ms.
 * rk_matvec4, rk_matmul8 and rk_matmul8_experts likewise issue no copies of the weights, and rk_cache4_attn withholds one of
 * the signals below, whichever `on` names (any other number counts as RK_STARVE_LOADS); the other calls make no difference between them. */
#define RK_STARVE_LOADS 1      /* the keys' rope part is not copied */
#define RK_STARVE_QUERIES 2    /* the queries' latent part is not copied */
#define RK_STARVE_QUERY_ROPE 3 /* their turned rope part is not announced */
#define RK_STARVE_KEYS 4       /* nor are unpacked keys */
#define RK_STARVE_KEYS_FREE 5  /* nor that the scores are done with them */
#define RK_STARVE_SCORES 6     /* nor the scores */
#define RK_STARVE_WEIGHTS 7    /* nor the softmax weights */
#define RK_STARVE_VALUES 8     /* nor the end of the value products */
rk_status rk_test_starve_loads(rk_ctx* ctx, int32_t on);
/* The library can be built with -DRK_CHECK (paper_2609_07008_b200/build.py, check=True): its kernels then
 * test every index they derive from a request table (protected-row list, inverse row map, work list,
 * compaction offsets) before using it, skip the access when it is out of range and record RK_ERR_ROWS in
 * the status word that rk_poll_status reads.  It is a debugging aid for small cases, not the production
 * build.  rk_check_selftest pushes one deliberately bad index through that check (nothing is accessed):
 * on the checking build the next rk_poll_status returns RK_ERR_ROWS; the ordinary build returns
 * RK_ERR_UNSUPPORTED here. */
rk_status rk_check_selftest(rk_ctx* ctx, void* stream);

/* Request geometry object: validates the layout and the protected-row list (Eq. protected;
 * the list is data here), builds row positions, per-segment relocation tables
 * cos/sin(delta_i * theta_j) in double precision, the inverse row map and the tile work
 * lists, and uploads them.  prot_rows: host [n_prot], strictly ascending packed rows; must
 * contain every row of every segment without artifact.  Reusable across layers and calls. */
rk_status rk_request_create(rk_ctx* ctx, const rk_layout* layout, const int32_t* prot_rows, int64_t n_prot,
                            rk_request** out);
rk_status rk_request_destroy(rk_request* req);
/* The same validation as rk_request_create, on the host only (no device, no context): returns the
 * status rk_request_create would return for this layout / row list and writes a message into msg
 * (may be NULL). */
rk_status rk_check_request(const rk_layout* layout, const int32_t* prot_rows, int64_t n_prot, char* msg,
                           size_t msg_len);
rk_status rk_request_get_info(const rk_request* req, rk_request_info* out);
/* Bytes of device scratch that rk_group_sliced_proj needs (per-head o = W_uv O_lat in bf16). */
rk_status rk_workspace_bytes(const rk_request* req, size_t* out);

/* (1) Query-side RoPE relocation, standalone form (Algorithm 2: q_i <- R(-delta_i) q; Eq. rope).
 * q_rope: device bf16, rope sub-vectors (64 wide) of n_rows x n_heads queries already rotated at
 * their request positions; element (r, h, e) at q_rope[r*row_stride + h*head_stride + e]
 * (strides in elements, multiples of 8).  out: device bf16 [seg_end-seg_begin][n_rows][n_heads][64],
 * out[i] = R(-seg_delta[seg_begin+i]) q.  The same rotation is fused into rk_mla_online_attn. */
rk_status rk_relocate_q(rk_ctx* ctx, const rk_request* req, const void* q_rope, int64_t n_rows, int32_t n_heads,
                        int64_t row_stride, int64_t head_stride, int32_t seg_begin, int32_t seg_end, void* out,
                        void* stream);

/* (2) Absorbed-MLA attention over the packed latent (Algorithm 2: SelectiveMLA for every
 * segment + running SegmentedLSEMerge inside the kernel; relocation fused into the Q load).
 *   kv   device bf16 [T][576] = [c (512) | k_rope at the document's canonical position (64)]
 *   q_g  device bf16 [T][G][576]  queries of the Global heads (group order), request position
 *   q_l  device bf16 [A][L][576]  queries of the Local heads (ascending head index) on the
 *        protected rows in list order
 *   O_g  device bf16 [T][G][512], lse_g device fp32 [T][G]   (natural-log LSE of scaled scores)
 *   O_l  device bf16 [A][L][512], lse_l device fp32 [A][L]
 * Either pass may be skipped by passing NULL for its q, O and lse. */
rk_status rk_mla_online_attn(rk_ctx* ctx, const rk_request* req, const void* kv, const void* q_g, const void* q_l,
                             void* O_g, float* lse_g, void* O_l, float* lse_l, void* stream);

/* (3) Stable segmented log-sum-exp merge, standalone form (Algorithm 2: SegmentedLSEMerge):
 * lse = log sum_j exp(lse_j), O = sum_j exp(lse_j - lse) O_j over n_parts partial results.
 *   O_part   device [n_parts][n_rows][n_heads][512], bf16 (part_dtype 0) or fp32 (part_dtype 1)
 *   lse_part device fp32 [n_parts][n_rows][n_heads]; -inf marks an empty part (its O is ignored)
 *   O device bf16 [n_rows][n_heads][512], lse device fp32 [n_rows][n_heads]
 * All parts empty gives O = 0, lse = -inf.  n_parts <= 4096. */
rk_status rk_segmented_merge(rk_ctx* ctx, int32_t n_parts, int64_t n_rows, int32_t n_heads, const void* O_part,
                             int32_t part_dtype, const float* lse_part, void* O, float* lse, void* stream);

/* The same merge for per-segment partial results of the output-phase variant (Algorithm 2:
 * RestorePhase, then SegmentedLSEMerge, then R^{-1}).  Part j is the partial result against the
 * canonical rows of segment seg_begin + j: its 64 rope dims (the last of 576) are in that document's
 * frame and are turned by R(+seg_delta[seg_begin + j]) before they are added.
 *   O_part   device [n_parts][n_rows][n_heads][576], bf16 (part_dtype 0) or fp32 (part_dtype 1)
 *   lse_part device fp32 [n_parts][n_rows][n_heads]; -inf marks an empty part (its O is ignored)
 *   row_pos  device int32 [n_rows]: request position of each row, whose merged rope dims are turned by
 *            R(-row_pos[r]); NULL leaves the result in the request frame
 *   O device bf16 [n_rows][n_heads][576], lse device fp32 [n_rows][n_heads]
 * seg_begin + n_parts <= number of segments of `req`; n_parts <= 4096. */
rk_status rk_segmented_merge_phase(rk_ctx* ctx, const rk_request* req, int32_t seg_begin, int32_t n_parts, int64_t n_rows,
                                   int32_t n_heads, const void* O_part, int32_t part_dtype, const float* lse_part,
                                   const int32_t* row_pos, void* O, float* lse, void* stream);

/* (4) Group-aligned sliced first output projection (Eq. offonline; Algorithm 2: z_online):
 * per head o = W_uv[h] O_lat (512 -> 128), then the head's 128-column slice of its group's W_a:
 *   z_on_g[t][g] = W_a[g][:, 128 j_g : 128 j_g + 128] o[t][global head of g]         (all T rows)
 *   z_on_l[a][g] = sum over the 7 Local heads j of group g of W_a[g][:, 128 j : ..] o[a][8g+j]
 *   W_uv device bf16 [H][128][512];  W_a device bf16 [G][r_o][1024]
 *   z_on_g device bf16 [T][G*r_o];   z_on_l device bf16 [A][G*r_o]
 * workspace: device scratch of at least rk_workspace_bytes().  Either half may be skipped by
 * passing NULL for its O and z. */
rk_status rk_group_sliced_proj(rk_ctx* ctx, const rk_request* req, const void* O_g, const void* O_l,
                               const void* W_uv, const void* W_a, void* z_on_g, void* z_on_l, void* workspace,
                               size_t workspace_bytes, void* stream);

/* The same projection for callers that cannot allocate device memory (the paper has no
 * counterpart; it is a property of this library's interface only).  A serving process that has
 * given the whole device to its own memory pool, or a request path that must not pay the
 * device-wide synchronisation an allocation can trigger, has no workspace to pass to
 * rk_group_sliced_proj.  Here the per-head intermediate lives in a fixed 32 MiB
 * (33 554 432 bytes) array inside the loaded library image; every device that loads the library
 * holds that array until the process exits.  The call allocates and frees nothing.
 *  - Requests whose scratch need (rk_workspace_bytes) exceeds 32 MiB are rejected with
 *    RK_ERR_WORKSPACE and a message; use rk_group_sliced_proj with your own workspace then.
 *  - rk_create looks up the array's device address on the context's device (the lookup makes the
 *    runtime place the array on that device, which may allocate and synchronise once); the entry
 *    point itself only reads the cached address, so create the context before any stream capture.
 *    The context's device must be current when the entry point is called.
 *  - All calls, from all contexts and streams of a process, share the one array, and it keeps
 *    whatever the previous call left in it.  Nothing in it needs to start at zero.  Two calls
 *    whose kernels overlap on the GPU (different streams) race on it: serialise them.
 * Arguments and results are exactly those of rk_group_sliced_proj, minus the workspace. */
rk_status rk_group_sliced_proj_static(rk_ctx* ctx, const rk_request* req, const void* O_g, const void* O_l,
                                      const void* W_uv, const void* W_a, void* z_on_g, void* z_on_l, void* stream);

/* (5) Add the offline MLA-Off artifact and run the shared second projection (Algorithm 2:
 * RestoreAndReplace, then W_b z; the paragraph after Eq. protected: a row in A takes the online Local
 * value in place of the artifact's, the two are never added):
 *   z[t] = z_on_g[t] + (t in A ? z_on_l[slot(t)] : z_off[t]);  y = W_b z.
 *   z_off device bf16 [n_off_rows][G*r_o] (packed rows; rows in A are never read)
 *   W_b   device bf16 [d_model][G*r_o], may be NULL to stop at z
 *   z     device bf16 [T][G*r_o] (required);  y device bf16 [T][d_model] (required iff W_b) */
rk_status rk_combine_offline(rk_ctx* ctx, const rk_request* req, const void* z_on_g, const void* z_on_l,
                             const void* z_off, const void* W_b, void* z, void* y, void* stream);

/* Offline side (Algorithm 1 "Build one canonical MLA-Off document artifact"): for packed rows
 * [row_begin, row_end) each row attends only the keys of its own segment, causally in the
 * segment's position-zero frame, with the Local heads; then z_off = W_{a,L} (W_uv O_L) summed over
 * each group's seven Local heads.  Queries are given at their REQUEST positions (like q_l); the
 * kernel rotates them by -seg_delta into the document's frame, which is the query the document had
 * when it was processed alone at position zero.
 *   q_l_rows   device bf16 [row_end-row_begin][L][576]
 *   z_off_rows device bf16 [row_end-row_begin][G*r_o]  (row row_begin of the artifact tensor)
 *   workspace  device scratch of at least rk_mla_off_workspace_bytes(req, row_end-row_begin)
 * Long requests are built in several calls over row ranges (the scratch holds the Local-head
 * attention output of the range). */
rk_status rk_mla_off_workspace_bytes(const rk_request* req, int64_t n_rows, size_t* out);
rk_status rk_mla_off_build(rk_ctx* ctx, const rk_request* req, const void* kv, int64_t row_begin, int64_t row_end,
                           const void* q_l_rows, const void* W_uv, const void* W_a, void* z_off_rows, void* workspace,
                           size_t workspace_bytes, void* stream);

/* Controller of the protected-row set (Eq. protected).  The paper's values: edge_rows 128,
 * tail_rows 32768, budget_bp 0 (no expansion), 1000, 2000 or 2500. */
typedef struct rk_policy {
  int32_t edge_rows;  /* B_edge: first and last rows of every relocated segment; >= 0 */
  int64_t tail_rows;  /* T_tail: the last request positions; >= 0 */
  int32_t budget_bp;  /* active budget in basis points of the candidate rows; 0..10000 */
} rk_policy;

/* Builds the protected token-row set A = Q u N u D u B_edge u I_top u T_tail (Eq. protected;
 * `ProtectedRows` of Algorithm 2) on the device, as the strictly ascending packed-row list that
 * rk_request_create takes.  Packed row t of segment i has canonical index j = t - seg_off[i] and
 * request position seg_delta[i] + j.
 *   Q u N   every row of a segment without artifact
 *   D       dirty_rows: device int32 [n_dirty], any order, duplicates allowed, entries outside
 *           [0,T) ignored; may be NULL iff n_dirty == 0
 *   B_edge  rows with j < edge_rows or j >= n_i - edge_rows of every segment that has an artifact
 *           and seg_delta[i] != 0 (artifacts are built at offset 0; any other offset relocates)
 *   T_tail  rows at request positions >= end - tail_rows, end = largest position + 1
 *   I_top   candidate rows = rows of segments with artifact.  If the sets above hold fewer than
 *           floor(budget_bp * candidates / 10000) candidate rows, the candidate rows outside them
 *           with the largest scores are added until that number is reached (equal scores: lower
 *           packed row first; -0.0 equals +0.0).  The sets above are never cut.
 *           scores: device float32 [T] (the Indexer's row scores, recomputed by the caller for
 *           this request; entries of non-candidate rows are not read), no NaN; NULL = no top-up.
 *   rows_out  device int32 [T] (capacity); the first *count_out entries are the result
 *   count_out device int64 [1]
 *   workspace device scratch of at least rk_protected_rows_workspace_bytes(T, n_segs), 256-byte aligned
 * The layout is host data and is validated like in rk_request_create (RK_ERR_LAYOUT).  The call
 * enqueues on `stream` and does not synchronise; read rows_out / count_out after the stream has
 * passed it.  The selection is exact (integer work; the scores are only compared), so the list is
 * bit-identical to the definition. */
rk_status rk_protected_rows_workspace_bytes(int64_t n_rows, int32_t n_segs, size_t* out);
rk_status rk_protected_rows(rk_ctx* ctx, const rk_layout* layout, const rk_policy* policy, const int32_t* dirty_rows,
                            int64_t n_dirty, const float* scores, int32_t* rows_out, int64_t* count_out,
                            void* workspace, size_t workspace_bytes, void* stream);

/* Retained expert fan-out of the adaptive sparse-MoE path (Eq. moe) for n tokens.
 *   p        device float32 [n][6]: the router weights of the token's Top-6 experts, any slot
 *            order, positive, no NaN; 8-byte aligned
 *   tau      the cumulative-share threshold
 *   fence    non-zero: a full-recompute fence layer, every token keeps all six (K_t = 6)
 *   k_out    device uint8 [n]: K_t in {3,4,5,6}
 *   keep_out device uint8 [n]: bit s set = the expert in slot s stays (the K_t largest weights;
 *            equal weights: lower slot first)
 * The weights are not renormalised and not written.  Decision arithmetic (float32, fixed order):
 * weights sorted descending, c_1 = p_(1), c_k = c_(k-1) + p_(k); K_t = the smallest k in {3,4,5}
 * with c_k >= tau * c_6, else 6 -- the paper's condition with both sides multiplied by the sum. */
rk_status rk_moe_fanout(rk_ctx* ctx, const float* p, int64_t n, float tau, int32_t fence, uint8_t* k_out,
                        uint8_t* keep_out, void* stream);

/* Device buffers that rk_layer_host stages through; all owned by the caller. */
typedef struct rk_layer_buffers {
  void *kv, *q_g, *q_l, *z_off;            /* device copies of the per-request inputs */
  void *O_g, *O_l, *z_on_g, *z_on_l, *z, *y;
  float *lse_g, *lse_l;
  void* workspace;
  size_t workspace_bytes;
} rk_layer_buffers;

/* rk_layer_host and rk_layer_stack_host use one set of internal copy streams and events per
 * context: at most one of them may be running on a context at any time (two host threads must not
 * call them concurrently on the same rk_ctx; use one context per thread).
 *
 * One whole layer from HOST inputs: copies kv, q_g, q_l, z_off host->device (use pinned host
 * memory; pageable memory works but serialises), runs (2), (4), (5), copies y device->host and
 * synchronises `stream`.  Weights stay resident on the device.  Copies that the running kernel
 * does not need yet travel on an internal second stream beside it (the Local pass needs only kv
 * and q_l; q_g and the artifact arrive meanwhile; the Global pass and everything after it run in
 * two row ranges, and the y rows of the first range return while the second computes) and are
 * ordered by device events, not by host polling (Section "Turning omitted
 * work into latency reduction": prefetch stream guarded by device events). */
rk_status rk_layer_host(rk_ctx* ctx, const rk_request* req, const void* kv_host, const void* q_g_host,
                        const void* q_l_host, const void* z_off_host, const void* W_uv, const void* W_a,
                        const void* W_b, const rk_layer_buffers* dev, void* y_host, void* stream);

/* One layer of a stack for rk_layer_stack_host. */
typedef struct rk_layer_io {
  const rk_request* req;                                    /* geometry + protected rows of this layer */
  const void *kv_host, *q_g_host, *q_l_host, *z_off_host;   /* pinned host inputs (shapes as in rk_layer_host) */
  const void *W_uv, *W_a, *W_b;                             /* device weights of this layer */
  void* y_host;                                             /* pinned host output [T][d_model] */
} rk_layer_io;

/* A stack of layers from HOST inputs with cross-layer prefetch (Section "Turning omitted work into
 * latency reduction": while layer l runs, a dedicated stream brings in the inputs of layer l+1;
 * device events, not host polling, guard consumption).  Two complete buffer sets are used in turn:
 * the inputs of layer l+1 are copied into the other set while layer l computes, and y of layer l
 * is copied out on a third stream while layer l+1 computes.  Synchronises `stream` before it
 * returns.  Every request must belong to `ctx`; the sets must be large enough for every layer. */
rk_status rk_layer_stack_host(rk_ctx* ctx, int32_t n_layers, const rk_layer_io* layers, const rk_layer_buffers* dev0,
                              const rk_layer_buffers* dev1, void* stream);

/* ---- Decode: generating tokens after the online step ------------------------------------------------------
 *
 * The latent rows live in a paged cache that holds the latent in 4 bits.  A SEGMENT is a document, or the suffix
 * that a request has generated so far; its row j is stored at canonical position j (like every document here),
 * so a document's pages serve every request that reuses it, at whatever offset it appears there.
 *
 * A page holds 64 rows of one segment in RK_CACHE4_PAGE_BYTES = 26 units of 16 bytes per row, unit-major: byte
 * u * 1024 + row * 16 + i is byte i of unit u of the row.
 *   units 0-15   latent dims 32 u .. 32 u + 31 as 4-bit codes n + 8: dim 32 u + 8 w + 2 i + e is the four bits at
 *                16 e + 4 i of the unit's w-th 32-bit word
 *   units 16-17  scale bytes: group g (dims 16 g .. 16 g + 15) is byte 4 (g >> 3) + (g & 3) of unit 16 + ((g >> 2) & 1);
 *                byte b is the scale 2^((b >> 3) - 20) * (1 + (b & 7) / 8), and 255 is NaN
 *   units 18-25  the 64 rope dims (bf16), turned by R(j)
 * The stored latent value is n * scale, which is a bf16 number exactly.
 *
 * The segment and page tables are device arrays: a captured graph can be replayed after their contents changed.  They
 * are bounds-checked on the device; a bad entry is skipped and rk_poll_status() returns RK_ERR_ROWS.  The
 * context's device must be the current one (RK_ERR_CUDA otherwise), and these calls need a context without
 * RK_VALUE_PHASE (RK_ERR_UNSUPPORTED otherwise). */
#define RK_CACHE4_PAGE_ROWS 64
#define RK_CACHE4_PAGE_BYTES 26624

typedef struct rk_cache4_table {
  int32_t n_segs;
  int64_t n_listed;          /* entries of page_ids */
  const int32_t* seg_len;    /* device [n_segs]: rows of each segment */
  const int32_t* page_off;   /* device [n_segs + 1]: its pages are page_ids[page_off[s]] .. page_ids[page_off[s+1] - 1] */
  const int32_t* page_ids;   /* device [n_listed]: row j of the segment is row j % 64 of its page j / 64 */
} rk_cache4_table;

/* Appends rows to segments.  Rows new_off[s] .. new_off[s+1] - 1 of the inputs become the LAST rows of segment s, whose
 * seg_len already counts them; rows from new_off[n_segs] on are padding and are not read into the cache.
 *   c       device bf16: latent of row i at c + i * c_stride (512 values; stride in elements, a multiple of 8)
 *   k_rope  device bf16: key rope part of row i BEFORE rotation at k_rope + i * r_stride (64 values; likewise)
 *   new_off device int32 [n_segs + 1], ascending from 0
 * Every 16 latent dims share the scale nearest to max|c| / 7 among the scales above (ties to the even byte), at least
 * 2^-20 and at most 3584; the codes are c / scale rounded half to even and limited to -7..7.  A group that holds an
 * infinity or a NaN is stored as NaN.  k_rope is turned by R(row index in its segment) in fp32 and rounded to bf16.
 * Only the units of the appended rows are written.  Pages that the call writes must each belong to one segment of
 * the table: a page listed for two growing segments holds a mixture afterwards.  Calls on different streams must
 * not write the same rows. */
rk_status rk_cache4_append(rk_ctx* ctx, void* pages, int64_t n_pages, const rk_cache4_table* table, const void* c,
                           int64_t c_stride, const void* k_rope, int64_t r_stride, const int32_t* new_off, int64_t n_new,
                           void* stream);

/* Reads rows back as the packed bf16 stream [c | k_rope] that rk_mla_online_attn takes: rows row_off[s] ..
 * row_off[s+1] - 1 of kv are the LAST row_off[s+1] - row_off[s] rows of segment s (the whole segment where that is
 * its length).
 *   kv  device bf16 [n_rows][576]; rows from row_off[n_segs] on, and rows of bad table entries, are left as they were */
rk_status rk_cache4_read(rk_ctx* ctx, const void* pages, int64_t n_pages, const rk_cache4_table* table,
                         const int32_t* row_off, int64_t n_rows, void* kv, void* stream);

/* Shape of a decode step: n_seqs requests with q_len query tokens each, which see n_items segments together, in at
 * most max_tiles key tiles (a tile is up to 128 consecutive rows of one segment; the sum over the items of
 * ceil(rows / 128)).  Limits: n_seqs * q_len * n_heads < 2^31 - 256, q_len <= 64, max_tiles <= 2^20. */
typedef struct rk_decode_shape {
  int32_t n_seqs, q_len, n_items, max_tiles;
} rk_decode_shape;

/* The work list of a decode step, for all layers whose caches share the tables: made once per step, on the device.
 *   seq_off    device int32 [n_seqs + 1]: request b sees items seq_off[b] .. seq_off[b+1] - 1
 *   item_seg   device int32 [n_items]: the segment; one segment may be an item of several requests
 *   item_delta device int32 [n_items]: the request position of its row 0, >= 0; item_delta + seg_len <= 2^30
 *   q_pos      device int32 [n_seqs][q_len]: request positions of the query tokens
 *   plan       device, rk_decode_plan_bytes() bytes, 256-byte aligned
 * Row j of an item sits at position item_delta + j; query token t sees it iff item_delta + j <= q_pos[t] (so a
 * padding request is one without items, or with negative positions, and a padding token has a negative position; any
 * will do).  A bad item is left out, and so is a key tile whose pages are not in the pool (RK_ERR_ROWS); more key tiles than
 * max_tiles make an empty plan (RK_ERR_WORKSPACE). Both are reported by rk_poll_status(). */
rk_status rk_decode_plan_bytes(const rk_ctx* ctx, const rk_decode_shape* shape, size_t* out);
rk_status rk_decode_plan(rk_ctx* ctx, const rk_decode_shape* shape, const rk_cache4_table* table, int64_t n_pages,
                         const int32_t* seq_off, const int32_t* item_seg, const int32_t* item_delta, const int32_t* q_pos,
                         void* plan, size_t plan_bytes, void* stream);

/* Absorbed-MLA attention of the query tokens over the cache (all heads):
 *   q    device bf16 [n_seqs][q_len][n_heads][576], at the request positions; relocated by R(-item_delta) per item
 *   O    device bf16 [n_seqs][q_len][n_heads][512];  lse  device fp32 [n_seqs][q_len][n_heads] (natural log)
 * A row that sees no key gets O = 0, lse = -inf.  `plan` must come from rk_decode_plan with this shape, head count and
 * n_pages (else RK_ERR_LAYOUT from rk_poll_status, O and lse left as they were) and the pages it names must still hold the rows; the plan
 * and the pages are only read, so concurrent calls may share them.  The workspace may not be shared by calls that overlap. A cached
 * row that holds a NaN makes the query rows that see it NaN, O and lse, and only those; an infinity in its rope part may do
 * the same (the turned query is multiplied in two parts).
 * The result does not depend on timing: partial results are joined in a fixed order. */
rk_status rk_cache4_attn_workspace_bytes(const rk_ctx* ctx, const rk_decode_shape* shape, size_t* out);
rk_status rk_cache4_attn(rk_ctx* ctx, const rk_decode_shape* shape, const void* plan, size_t plan_bytes, const void* pages,
                         int64_t n_pages, const void* q, void* O, float* lse, void* workspace, size_t workspace_bytes,
                         void* stream);

/* 4-bit weight matrices for products with a few token rows (the decode-time W_uv, W_a, W_b).  A row's weights share
 * a bf16 scale per `group` columns: scale = bf16(max|w| / 7), codes w / scale rounded half to even and limited to
 * -7..7; a group with a non-finite weight has the scale NaN.  codes and scales are laid out for the kernel.
 * group is 32, 64 or 128; n_out a multiple of 16; k a multiple of 64 and of group. */
typedef struct rk_w4 {
  int32_t n_mat, n_out, k, group;
  void* codes;    /* device, n_mat * n_out * k / 2 bytes, 16-byte aligned */
  void* scales;   /* device, n_mat * n_out * (k / group) * 2 bytes, 16-byte aligned */
} rk_w4;

/* Lays out weights: w device bf16 [n_mat][n_out][k] -> w4->codes, w4->scales. */
rk_status rk_quant4(rk_ctx* ctx, const void* w, const rk_w4* w4, void* stream);

/* y[t][m] = W[m] x[t][m] for n_tok token rows; sums in fp32.
 *   x  device bf16: token t at x + t * x_stride, [n_mat][k] (stride in elements, a multiple of 8, >= n_mat * k)
 *   y  device bf16 (out_dtype 0) or fp32 (out_dtype 1): token t at y + t * y_stride, [n_mat][n_out] (>= n_mat * n_out) */
rk_status rk_matvec4(rk_ctx* ctx, const rk_w4* w4, const void* x, int64_t x_stride, int64_t n_tok, void* y,
                     int64_t y_stride, int32_t out_dtype, void* stream);

/* ---- Behind the attention: experts and tokens ---------------------------------------------------------------
 *
 * The rest of a generating step: which experts a token goes to (the weights are what rk_moe_fanout takes), the experts'
 * products, the large products of prompts in 8-bit integers, and the token out of the logits.  These calls need the
 * context's device to be the current one (RK_ERR_CUDA otherwise), read only the tensors that they are given, keep nothing
 * and can be captured into a CUDA graph; calls on different streams may overlap as long as their outputs differ.
 * n = 0 is allowed everywhere and does nothing. */

#define RK_SCORE_SOFTMAX 0
#define RK_SCORE_SIGMOID 1
typedef struct rk_route {
  int32_t n_experts;   /* E, at most 1024, a multiple of n_groups */
  int32_t k;           /* experts per token, 1..16 and at most top_groups * E / n_groups */
  int32_t n_groups;    /* groups of E / n_groups consecutive experts, 1..32 */
  int32_t top_groups;  /* groups that a token's experts may come from, 1..n_groups */
  int32_t group_top;   /* 1 or 2: a group is ranked by the sum of that many of its best experts */
  int32_t score;       /* RK_SCORE_SOFTMAX (over all experts) or RK_SCORE_SIGMOID */
  int32_t renorm;      /* non-zero: the weights of a token are divided by their sum */
  float scale;         /* factor of the weights, finite */
} rk_route;

/* Routes n tokens.  s = the scores of the token's logits, c = s + bias.  The top_groups groups of the highest rank take
 * part (equal: the lower group), and the k experts of the largest c in them are chosen (equal: the lower index), in
 * descending order.  Their weights are their s (without bias), divided by their sum with `renorm` (0 where that is 0),
 * times scale.  Scores are compared and weighted in 64 bits (the sum of a softmax whose weights are not renormalised is right to
 * 2^-31); the weights are rounded to fp32.
 *   logits  device [n][E], bf16 (logits_dtype 0) or fp32 (1), rows `stride` elements apart (stride >= E)
 *   bias    device fp32 [E], or NULL
 *   ids     device int32 [n][k];  weights  device fp32 [n][k]
 * An expert whose logit or bias is -inf is never chosen; a group is ranked by the experts that it has left, and slots without
 * an expert get id -1 and weight 0.  A token with a NaN among its scores (a NaN logit or bias, +inf with softmax) gets
 * ids -1 and weights NaN. */
rk_status rk_moe_route(rk_ctx* ctx, const rk_route* route, const void* logits, int32_t logits_dtype, int64_t stride,
                       const float* bias, int64_t n, int32_t* ids, float* weights, void* stream);

/* Lists the pairs p = t * k + s of a routing by expert.
 *   ids      device int32 [n][k]; a pair whose id is outside 0 .. n_experts - 1 is not listed
 *   keep     device uint8 [n]: bit s set = slot s of the token stays (rk_moe_fanout's keep_out); NULL = all stay.  k <= 8 with it
 *   row_off  device int32 [n_experts + 1];  rows  device int32 [n * k]
 * rows[row_off[e]] .. rows[row_off[e + 1] - 1] are the pairs of expert e, ascending; the places from row_off[n_experts] on
 * hold -1.  n * k < 2^30; n_experts <= 1024. With n = 0 row_off is all 0. */
rk_status rk_moe_group(rk_ctx* ctx, const int32_t* ids, const uint8_t* keep, int64_t n, int32_t k, int32_t n_experts,
                       int32_t* row_off, int32_t* rows, void* stream);

/* Rows in 8 bits: n_mat * n_rows rows of k values, codes -127..127 times the row's scale. */
typedef struct rk_q8 {
  int32_t n_mat;      /* matrices (experts); 1 for tokens and dense weights; at most 1024 */
  int64_t n_rows;     /* rows of a matrix: output channels, or tokens */
  int32_t k;          /* 1 .. 131072 */
  void* codes;        /* device int8 [n_mat][n_rows][k rounded up to a multiple of 16], zeros behind k; 16-byte aligned */
  float* scales;      /* device fp32 [n_mat][n_rows] */
} rk_q8;

/* Quantises rows: scale = fp32(max|x| / 127), codes = x / scale rounded half to even (exactly) and limited to -127..127.  A
 * row of zeros has scale 0; a row with an infinity or a NaN has the scale NaN and codes 0, and makes NaN what it is
 * multiplied with.
 *   x  device bf16: row i at x + i * x_stride (in elements, >= k, of any alignment to 2 bytes; multiples of 16 bytes are faster) */
rk_status rk_quant8(rk_ctx* ctx, const void* x, int64_t x_stride, const rk_q8* q8, void* stream);

/* y[t][o] = sum_j x.codes[t][j] w.codes[o][j] * x.scales[t] * w.scales[o]; the sums are exact, then they and the two products,
 * from the left, are rounded to fp32 (tokens beyond 1e29 can overflow there) and, for out_dtype 0, to bf16.
 * w.n_mat = x.n_mat = 1, w.k = x.k.
 *   y  device bf16 (out_dtype 0) or fp32 (1): token t at y + t * y_stride, w.n_rows values (y_stride >= w.n_rows) */
rk_status rk_matmul8(rk_ctx* ctx, const rk_q8* w, const rk_q8* x, void* y, int64_t y_stride, int32_t out_dtype, void* stream);

/* The experts' products over the lists of rk_moe_group: y[p] = W_e x[p / per] for every pair p of expert e, W_e = matrix e of w.
 *   row_off  device int32 [w.n_mat + 1];  rows  device int32 [n_pairs]
 *   per      the slots per token where x has a row per token (first products), 1 where it has a row per pair (second
 *            products); x.n_rows * per >= n_pairs
 *   y        device, n_pairs rows; rows that no list names are left as they were
 * The tables are bounds-checked on the device: an expert whose bounds are not 0 <= row_off[e] <= row_off[e + 1] <= n_pairs,
 * and a listed pair outside 0 .. n_pairs - 1, is skipped and rk_poll_status() returns RK_ERR_ROWS.  A pair listed twice gets,
 * element by element, the product of one of its experts. */
rk_status rk_matmul8_experts(rk_ctx* ctx, const rk_q8* w, const rk_q8* x, const int32_t* row_off, const int32_t* rows,
                             int64_t n_pairs, int32_t per, void* y, int64_t y_stride, int32_t out_dtype, void* stream);

/* Samples a token from each row of logits.  p_i = exp((l_i - max l) / temperature).  In the order of falling logits (equal:
 * the lower index first; -0.0 equals +0.0) a token stays if
 *   its rank is below top_k,   the p in front of it sum to less than top_p * (the sum over the top_k),   p_i >= min_p;
 * the first one always stays.  The token is the first that stayed, by index, whose cumulated p (over those that stayed, by
 * index) exceeds u times their sum.
 *   logits  device [n][vocab], bf16 (logits_dtype 0) or fp32 (1), rows `stride` elements apart; -inf is never drawn
 *   u       device fp32 [n]: uniform random numbers in [0, 1); values outside count as the nearest inside, NaN as 0
 *   temperature, top_k, top_p, min_p  device [n] (top_k int32, the others fp32), each NULL where all rows leave it off.
 *     temperature below 2^-100 or NaN: the largest logit; top_k <= 0, top_p >= 1 or NaN, min_p <= 0 or NaN: off
 *   tokens  device int32 [n];  probs  device fp32 [n], the token's p over the sum of those that stayed, or NULL
 * A row with a NaN, and a row of nothing but -inf, gets token -1 and prob NaN.  +inf: only those are drawn, each alike.
 * p is rounded to multiples of 2^-42: a token below 2^-42 of the largest is not drawn.  1 <= vocab <= 2^20, n * 8 < 2^31. */
rk_status rk_sample(rk_ctx* ctx, const void* logits, int32_t logits_dtype, int64_t stride, int64_t n, int32_t vocab, const float* u,
                    const float* temperature, const int32_t* top_k, const float* top_p, const float* min_p, int32_t* tokens,
                    float* probs, void* stream);

#ifdef __cplusplus
}
#endif
#endif /* RK_H_ */
