/*
 * rollout_attn.h — C ABI of the MI355X (gfx950) rollout-attention library.
 *
 * The library implements the GPU work that dominates multi-turn agent rollouts
 * as described in "ProRL Agent: Rollout-as-a-Service for RL Training of
 * Multi-Turn LLM Agents" (arXiv 2603.18815):
 *   - every agent step is one LLM completion over the whole conversation
 *     history (Sec. 3.3.2), i.e. a decode step of one new token per trajectory
 *     against that trajectory's cached keys and values;
 *   - all calls of one task go to one backend so that its cached prefix is
 *     reused (Sec. 3.3.2, load balancing), so each trajectory keeps a
 *     persistent paged KV cache across turns;
 *   - earlier turns keep their token ids and only new observations are
 *     tokenised and appended (Sec. 3.3.3), i.e. a causal chunked prefill of the
 *     observation tokens against the existing cache ("append").
 * The paper states no attention formula; the library computes standard
 * scaled dot-product softmax attention with grouped KV heads (query head h
 * reads KV head h / (Hq / Hkv)), bf16 inputs, fp32 accumulation and fp32
 * outputs.
 *
 * Conventions for every entry point
 *   - All array arguments are DEVICE pointers unless marked "host". The caller
 *     owns every buffer (pools, tables, outputs, workspace); the library
 *     allocates nothing and keeps no pointer after it returns.
 *   - Work is enqueued asynchronously on `stream` (0 = the null stream). Buffers
 *     must stay alive until the stream has executed the enqueued kernels.
 *     Concurrent calls on different streams are safe if their outputs and
 *     workspaces do not overlap.
 *   - Every function returns an ra_status. Arguments the host can check are
 *     checked before any HIP call. Nothing aborts. A softmax or logit `scale`
 *     must be finite (any sign; 0 weighs every key equally), else
 *     RA_ERR_SHAPE.
 *   - Zero work (B == 0, total_q == 0, total_new == 0) returns RA_OK without
 *     launching anything.
 *   - Device-resident metadata (lengths, block tables, cu_* offsets) is a
 *     precondition and is not read by the host: lengths >= 0, every position
 *     used lies below bt_stride * page_size, page ids lie in [0, num_pages),
 *     cu_* arrays are non-decreasing with cu[0] = 0. As a guard against
 *     memory faults the kernels clamp page ids into [0, num_pages) and
 *     lengths to the host-provided maxima; violating inputs give undefined
 *     numbers, never an out-of-bounds access.
 *   - Results are deterministic: the same inputs give bitwise the same
 *     outputs, independent of which physical pages the block table names.
 *   - Every entry point may be captured into a HIP graph: it allocates
 *     nothing, never synchronizes, issues no memset or copy (work counters
 *     are cleared by its own kernels), so each replay computes what an
 *     eager call would. Replays of one graph must not overlap in time if
 *     they share a workspace.
 *
 * Paged KV layout (ABI versions 2 to 6). Page size P = 16 tokens, head dim D = 128.
 * Logical token j of row b lives in physical page bt[b * bt_stride + j / P]
 * at slot j % P. Within a page each KV head owns one contiguous block:
 *   K pool  [num_pages][Hkv][P][D]   element (page, g, slot, d) at
 *           ((page * Hkv + g) * P + slot) * D + d           (token-major)
 *   V pool  [num_pages][Hkv][D][P]   element (page, g, slot, d) at
 *           ((page * Hkv + g) * D + d) * P + slot           (dim-major)
 * V is stored dimension-major so that the matrix-core operand for P·V (keys
 * along the contraction dimension) is a contiguous read.
 * Element types (kv_dtype):
 *   RA_KV_BF16      bf16 (4 KiB per page and head);
 *   RA_KV_FP8_E4M3  OCP FP8 E4M3 codes (2 KiB per page and head) with one
 *                   scale per pool: an element's value is decode(code) *
 *                   k_scale (K) or * v_scale (V). The paper is silent on KV
 *                   precision; this halves the bytes decode streams. A bf16
 *                   value x is stored as encode(fp32(x) * fp32(1 / scale)):
 *                   round to nearest even, magnitudes beyond 448 (and
 *                   infinities) saturate to +-448, NaN becomes 0x7F.
 *   fp8 pools are supported by every entry point: kv_page_write (and the
 *   write of rollout_attn_append_write) quantizes, kv_page_gather copies the
 *   codes out, the attention entry points convert the codes exactly to bf16
 *   operands. A mixed call takes one element type for both sides
 *   (RA_ERR_UNSUPPORTED otherwise).
 */
#ifndef ROLLOUT_ATTN_H
#define ROLLOUT_ATTN_H

#include <stddef.h>
#include <stdint.h>

#include <hip/hip_runtime_api.h>

#ifdef __cplusplus
extern "C" {
#endif

#define RA_ABI_VERSION 6
#define RA_PAGE_SIZE 16
#define RA_HEAD_DIM 128

typedef enum {
  RA_OK = 0,
  RA_ERR_NULL = 1,        /* a required pointer is NULL */
  RA_ERR_SHAPE = 2,       /* inconsistent sizes (negative, Hq % Hkv != 0, ...) */
  RA_ERR_UNSUPPORTED = 3, /* valid but not built: page_size != 16, head_dim != 128,
                             a decode group size Hq / Hkv above 32, an
                             unknown kv_dtype,
                             pools of two element types in one mixed call */
  RA_ERR_WORKSPACE = 4,   /* workspace smaller than the *_workspace_size value */
  RA_ERR_HIP = 5          /* a HIP launch failed (no device, bad stream, ...) */
} ra_status;

typedef enum { RA_KV_BF16 = 0, RA_KV_FP8_E4M3 = 1 } ra_kv_dtype;

/* Caller-owned paged KV cache (device memory), see the layout above. */
typedef struct {
  void *k_pool;               /* [num_pages][num_kv_heads][page_size][head_dim] */
  void *v_pool;               /* [num_pages][num_kv_heads][head_dim][page_size] */
  const int32_t *block_table; /* int32 [B][bt_stride]; row b of the call's batch */
  int32_t num_pages;
  int32_t bt_stride;          /* entries per block-table row (>= 1) */
  int32_t num_kv_heads;       /* Hkv */
  int32_t page_size;          /* must be 16 */
  int32_t head_dim;           /* must be 128 */
  int32_t kv_dtype;           /* ra_kv_dtype of both pools */
  float k_scale, v_scale;     /* fp8 pools: finite, > 0 and with a finite fp32
                                 reciprocal (RA_ERR_SHAPE otherwise); ignored for
                                 bf16 pools */
} ra_paged_kv;

/* ABI version of the loaded library (RA_ABI_VERSION). */
int ra_abi_version(void);

/* Static, human-readable name of a status code. */
const char *ra_status_string(int status);

/*
 * Decode: one query token per trajectory against its cached keys
 * (Sec. 3.3.2: each agent step is a completion over the full history).
 * For row b and query head h with g = h / (Hq / Hkv):
 *   out[b][h] = softmax_j(scale * <q[b][h], K_j>) · V_j over j in [0, kv_lens[b])
 *   lse[b][h] = ln sum_j exp(scale * <q[b][h], K_j>)
 * kv_lens counts the token being decoded (write it with kv_page_write first).
 * Rows with kv_lens[b] <= 0 give out = 0 and lse = -inf.
 *
 *   q           bf16 [B][Hq][128]
 *   kv          pools and block table ([B][bt_stride])
 *   kv_lens     int32 [B]
 *   max_kv_len  host: an upper bound of kv_lens (plans the split over pages);
 *               must satisfy max_kv_len <= bt_stride * 16
 *   out         fp32 [B][Hq][128]
 *   lse         fp32 [B][Hq] or NULL
 *   workspace   device scratch of at least
 *               rollout_attn_decode_workspace_size(B, Hq, Hkv, max_kv_len) bytes
 *               (split partial results; contents on entry are ignored). The
 *               size is that of the fastest splits and can fall as B or
 *               max_kv_len grows. On a smaller workspace the splits are
 *               lengthened until their partials fit, to 512 keys or the longer
 *               splits that much work takes, which can change the rounding of
 *               the results (order of fp32 sums); RA_ERR_WORKSPACE if those do
 *               not fit either. So a workspace sized for the largest call of a
 *               loop need not hold every smaller one (65 rows of 32768 keys over
 *               8 KV heads: too small for 64 rows): take the largest size over
 *               the calls to come.
 * Errors: RA_ERR_NULL, RA_ERR_SHAPE (B < 0, Hq % Hkv, max_kv_len > bt_stride*16),
 *         RA_ERR_UNSUPPORTED, RA_ERR_WORKSPACE, RA_ERR_HIP.
 */
size_t rollout_attn_decode_workspace_size(int32_t B, int32_t Hq, int32_t Hkv,
                                          int32_t max_kv_len);
int rollout_attn_decode(const void *q, const ra_paged_kv *kv, const int32_t *kv_lens, int32_t B,
                        int32_t Hq, int32_t max_kv_len, float scale, float *out, float *lse,
                        void *workspace, size_t workspace_bytes, hipStream_t stream);

/*
 * Decode that allocates nothing, for callers that cannot allocate device
 * memory or pass a workspace: code under HIP graph capture, tight serving
 * loops, harnesses that forbid hipMalloc. Arguments, results and errors are
 * those of rollout_attn_decode with a workspace of its size; the split partial
 * results go to a scratch array of RA_NOALLOC_SCRATCH_BYTES that the library
 * holds in each GPU's memory until the process ends. A call whose
 * rollout_attn_decode_workspace_size(B, Hq, Hkv, max_kv_len) exceeds
 * RA_NOALLOC_SCRATCH_BYTES returns RA_ERR_WORKSPACE before any HIP call (64
 * MiB holds, e.g., 64 rows of 32 query heads at up to 32768 keys). Every call
 * on one GPU uses that GPU's one array and leaves its contents behind: calls
 * that overlap in time on one GPU (different streams, or threads whose calls
 * are in flight together) race and give wrong results; issue them on one
 * stream.
 */
#define RA_NOALLOC_SCRATCH_BYTES (64u << 20)
int rollout_attn_decode_noalloc(const void *q, const ra_paged_kv *kv, const int32_t *kv_lens,
                                int32_t B, int32_t Hq, int32_t max_kv_len, float scale,
                                float *out, float *lse, hipStream_t stream);

/*
 * Shared-prefix decode: decode for groups of rows whose caches begin with the
 * same physical pages, e.g. the rollouts of one task, which share its prompt
 * (Sec. 4 generates several rollouts per task instance; Sec. 3.3.2 keeps all
 * calls of a task on one backend so that its cached prefix is reused). The
 * result is that of rollout_attn_decode on the same rows (up to rounding: the
 * keys are split differently); the shared keys are read once for up to
 * 16 / (Hq / Hkv) rows of a group (one row per read for groups of more than
 * 16 query heads) instead of once per row, and the reads of one group's
 * chunks of rows are scheduled together so that the later ones mostly hit
 * the cache.
 * For group i, rows group_start[i] .. group_start[i+1]-1 attend their first P_i
 * keys together, P_i = min(prefix_len[i], shortest kv_lens of the group)
 * rounded down to a multiple of 32, read through the block table of the
 * group's first row; each row attends its keys P_i .. kv_lens[b]-1 alone.
 *
 *   q, kv, kv_lens, out, lse, scale: as rollout_attn_decode
 *   group_start     int32 [num_groups + 1], group_start[0] = 0, non-decreasing,
 *                   group_start[num_groups] = B (every row in one group)
 *   prefix_len      int32 [num_groups]: positions [0, prefix_len[i]) of every
 *                   row of group i map to the same pages as the group's first
 *                   row (a precondition: not checked; violating it gives wrong
 *                   numbers, never an out-of-bounds access)
 *   max_group_rows  host: an upper bound of the rows of a group, <= B
 *   max_prefix_len  host: an upper bound of prefix_len, <= max_kv_len
 *   workspace       device scratch of at least
 *                   rollout_attn_decode_shared_prefix_workspace_size(B, Hq, Hkv,
 *                   max_kv_len, max_prefix_len) bytes (contents on entry ignored)
 * Errors: as rollout_attn_decode; RA_ERR_SHAPE also for num_groups == 0 or
 *         max_group_rows == 0 with B > 0, max_group_rows > B, num_groups > B,
 *         max_prefix_len > max_kv_len; RA_ERR_UNSUPPORTED when the launch grid
 *         needs more than 65535 planes: num_groups * max_group_rows row planes
 *         plus ceil(num_groups * chunks * prefix splits / splits) prefix planes,
 *         chunks = ceil(max_group_rows / rows per chunk).
 */
size_t rollout_attn_decode_shared_prefix_workspace_size(int32_t B, int32_t Hq, int32_t Hkv,
                                                        int32_t max_kv_len,
                                                        int32_t max_prefix_len);
int rollout_attn_decode_shared_prefix(const void *q, const ra_paged_kv *kv,
                                      const int32_t *kv_lens, const int32_t *group_start,
                                      const int32_t *prefix_len, int32_t B, int32_t Hq,
                                      int32_t num_groups, int32_t max_group_rows,
                                      int32_t max_prefix_len, int32_t max_kv_len, float scale,
                                      float *out, float *lse, void *workspace,
                                      size_t workspace_bytes, hipStream_t stream);

/*
 * Append: causal chunked prefill of newly appended observation tokens against
 * each trajectory's cache (Sec. 3.3.3: earlier turns keep their tokens, new
 * observations are tokenised and appended). Row b owns packed queries
 * cu_q[b] .. cu_q[b+1]-1; its i-th query sits at absolute position
 * ctx_lens[b] + i and attends keys 0 .. ctx_lens[b] + i (inclusive):
 *   out[t][h] = softmax_j(scale * <q[t][h], K_j>) · V_j,  lse likewise.
 * The chunk's own keys and values must already be in the pool at positions
 * ctx_lens[b] .. ctx_lens[b] + T_b - 1 (kv_page_write with start_pos = ctx_lens
 * on the same stream first).
 *
 *   q           bf16 [total_q][Hq][128]
 *   cu_q        int32 [B+1], cu_q[0] = 0, cu_q[B] = total_q
 *   ctx_lens    int32 [B]
 *   max_q_len   host: an upper bound of T_b = cu_q[b+1] - cu_q[b]
 *   max_kv_len  host: an upper bound of ctx_lens[b] + T_b; <= bt_stride * 16
 *   out         fp32 [total_q][Hq][128]
 *   lse         fp32 [total_q][Hq] or NULL
 *   workspace   device scratch of at least
 *               rollout_attn_append_workspace_size(B, Hq, Hkv, max_q_len) bytes
 *               (the call's work lists, counters and partial results, up to
 *               some 68 MB of them, less for chunks of fewer tokens than a
 *               tile's 256 / (Hq / Hkv); rewritten by every call; contents on
 *               entry are ignored).
 *               Calls that share a workspace must not overlap.
 * The work is planned on the device (a one-workgroup kernel orders the rows
 * longest first and queues each KV head's tiles for one XCD, or, with too few
 * tiles to fill the GPU, cuts their key ranges into equal shares whose partial
 * results are merged) and run by one persistent workgroup per CU. The cuts
 * depend on the lengths of all the call's rows and their order in the call, and
 * on nothing else: the same call gives the same bits, while a row's result in
 * another call (beside other rows) can differ by the order of fp32 sums.
 * Errors as for decode; RA_ERR_UNSUPPORTED also for more than 256 KV heads.
 */
size_t rollout_attn_append_workspace_size(int32_t B, int32_t Hq, int32_t Hkv,
                                          int32_t max_q_len);
int rollout_attn_append(const void *q, const int32_t *cu_q, const int32_t *ctx_lens,
                        const ra_paged_kv *kv, int32_t B, int32_t Hq, int32_t total_q,
                        int32_t max_q_len, int32_t max_kv_len, float scale, float *out,
                        float *lse, void *workspace, size_t workspace_bytes,
                        hipStream_t stream);

/*
 * Append with the page write fused in: writes the chunk's keys and values into
 * the pages and computes the append attention in one launch (plus the
 * planning kernel). Equivalent, bitwise, to kv_page_write(k_new, v_new, cu_q,
 * start_pos = ctx_lens) followed by rollout_attn_append on the same stream
 * (Sec. 3.3.3: each new observation is appended to the retained tokens and
 * attended in the same step). The write runs inside the planning kernel's
 * launch (its other workgroups write while one plans), so the call is two
 * launches instead of the three of the separate calls; the attention kernel
 * then reads the chunk from the pages.
 *
 *   q, cu_q, ctx_lens, kv, B, Hq, total_q, max_q_len, max_kv_len, scale, out,
 *   lse, workspace: as rollout_attn_append (same workspace size)
 *   k_new, v_new  bf16 [total_q][Hkv][128]: the chunk tokens' keys and values,
 *                 packed like q; token i of row b goes to position
 *                 ctx_lens[b] + i
 * fp8 pools: the chunk is quantized as by kv_page_write (encode(fp32(x) *
 * fp32(1 / scale)), see the layout above) and attended as stored.
 * Precondition (not checked): no row of the call reads, below its ctx, a page
 * slot that another row of the call writes.
 * Errors: as rollout_attn_append.
 */
int rollout_attn_append_write(const void *q, const void *k_new, const void *v_new,
                              const int32_t *cu_q, const int32_t *ctx_lens, const ra_paged_kv *kv,
                              int32_t B, int32_t Hq, int32_t total_q, int32_t max_q_len,
                              int32_t max_kv_len, float scale, float *out, float *lse,
                              void *workspace, size_t workspace_bytes, hipStream_t stream);

/*
 * Rotary position embedding on write. Models of the paper's kind (e.g. Qwen3)
 * rotate each query and key by its position before attention; the paper does
 * not describe model internals, so the rotation is an option of the write
 * path: the key is rotated as it is written into its page, and in the fused
 * call the chunk's queries are rotated as they are loaded.
 *
 * Rotation of a 128-dim head row x at position p with the table cos_sin
 * (fp32 [rope_rows][128]; row p holds c_i = cos(p w_i) in columns 0..63 and
 * s_i = sin(p w_i) in columns 64..127, computed by the caller for its model's
 * frequencies w_i), for i in [0, 64):
 *   y_i      = fp32(x_i c_i) - fp32(x_{i+64} s_i)
 *   y_{i+64} = fp32(x_{i+64} c_i) + fp32(x_i s_i)
 * each product and each sum rounded to fp32 (no fused multiply-add), then y
 * rounded to bf16 (nearest even). The rotated bf16 row is what is written
 * (bit copy, or E4M3 quantization for fp8 pools, exactly as kv_page_write
 * writes a bf16 row) and what the attention uses.
 *
 * kv_page_write_rope: kv_page_write with the keys rotated at their positions
 *   start_pos[b] + t (values unrotated). Needs max_pos <= rope_rows.
 * rollout_attn_append_write_rope: rollout_attn_append_write with the chunk's
 *   keys rotated at ctx_lens[b] + i as they are written and its queries
 *   rotated at the same positions; equal, bitwise, to kv_page_write_rope
 *   followed by rollout_attn_append on the rotated queries. Needs
 *   max_kv_len <= rope_rows.
 * Errors: as the unrotated calls; RA_ERR_NULL (cos_sin NULL); RA_ERR_SHAPE
 * (rope_rows <= 0 or too few rows).
 */
int kv_page_write_rope(const void *k_new, const void *v_new, const int32_t *cu_new,
                       const int32_t *start_pos, const ra_paged_kv *kv, int32_t B,
                       int32_t total_new, int32_t max_new, int32_t max_pos, const float *cos_sin,
                       int32_t rope_rows, hipStream_t stream);
int rollout_attn_append_write_rope(const void *q, const void *k_new, const void *v_new,
                                   const int32_t *cu_q, const int32_t *ctx_lens,
                                   const ra_paged_kv *kv, int32_t B, int32_t Hq, int32_t total_q,
                                   int32_t max_q_len, int32_t max_kv_len, float scale,
                                   const float *cos_sin, int32_t rope_rows, float *out, float *lse,
                                   void *workspace, size_t workspace_bytes, hipStream_t stream);

/*
 * Mixed step: the attention of one rollout step in which some trajectories
 * decode a token while others have just had tool observations appended
 * (Sec. 3.3.1: many rollout workers drive their agent loops concurrently, each
 * firing LLM calls; Sec. 3.3.3: observations are appended to the retained
 * tokens). Computes, in one persistent launch over the GPU (plus the one-
 * workgroup planning kernel before it and the decode combine after it):
 *   - for the decode rows, exactly what rollout_attn_decode computes
 *     (up to rounding: each split is summed by twice as many waves);
 *   - for the append rows, bitwise what rollout_attn_append computes.
 * Append tiles are taken longest first and the decode splits are spread
 * among them, so that decode's HBM traffic can overlap append's matrix work.
 * The two sides may use different block tables (and pools); either side may
 * be empty (B_decode == 0, or B_append == 0 / total_q == 0 / max_q_len == 0),
 * in which case its pointers are not used and may be NULL.
 *
 *   decode side:  q_decode, kv_decode, kv_lens, B_decode, max_kv_len_decode,
 *                 out_decode, lse_decode: as q, kv, kv_lens, B, max_kv_len,
 *                 out, lse of rollout_attn_decode
 *   append side:  q_append, cu_q, ctx_lens, kv_append, B_append, total_q,
 *                 max_q_len, max_kv_len_append, out_append, lse_append: as q,
 *                 cu_q, ctx_lens, kv, B, total_q, max_q_len, max_kv_len, out,
 *                 lse of rollout_attn_append (the chunks' K/V already written)
 *   Hq, scale     shared by both sides
 *   workspace     device scratch of at least rollout_attn_mixed_workspace_size(
 *                 B_decode, B_append, Hq, Hkv_decode, Hkv_append,
 *                 max_kv_len_decode, max_q_len) bytes: work lists, work
 *                 counters and partial results, all rewritten by every call
 *                 (contents on entry are ignored). Calls that share a
 *                 workspace must not overlap.
 * Errors: as rollout_attn_decode / rollout_attn_append for each non-empty
 *         side; RA_ERR_UNSUPPORTED also for more than 256 KV heads or more
 *         than 2^31 - 2^16 work entries.
 */
size_t rollout_attn_mixed_workspace_size(int32_t B_decode, int32_t B_append, int32_t Hq,
                                         int32_t Hkv_decode, int32_t Hkv_append,
                                         int32_t max_kv_len_decode, int32_t max_q_len);
int rollout_attn_mixed(const void *q_decode, const ra_paged_kv *kv_decode,
                       const int32_t *kv_lens, int32_t B_decode, int32_t max_kv_len_decode,
                       float *out_decode, float *lse_decode, const void *q_append,
                       const int32_t *cu_q, const int32_t *ctx_lens, const ra_paged_kv *kv_append,
                       int32_t B_append, int32_t total_q, int32_t max_q_len,
                       int32_t max_kv_len_append, float *out_append, float *lse_append,
                       int32_t Hq, float scale, void *workspace, size_t workspace_bytes,
                       hipStream_t stream);

/*
 * Token log-probabilities under an LM head: for each position n, the
 * log-probability of the emitted token targets[n] (Sec. 3.3.3: token-in /
 * token-out returns every generated token with its log-probability), fused
 * into one pass over the LM-head matrix without writing the logits:
 *   z_v = scale * <h[n], W[v]>,  lse[n] = ln sum_v exp z_v,
 *   logprob[n] = z_{targets[n]} - lse[n]   (NaN if targets[n] is not in [0, V))
 * bf16 inputs, fp32 products and outputs.
 *
 *   h          bf16 [N][D] hidden states (row n: the position's last-layer output)
 *   W          bf16 [V][D] LM-head matrix, one row per vocabulary entry
 *   targets    int32 [N]
 *   scale      multiplies the logits (1 / temperature; 1 for the raw model)
 *   logprob    fp32 [N]
 *   lse        fp32 [N] or NULL
 *   workspace  device scratch of at least token_logprob_workspace_size(N, V, D)
 *              bytes (per-chunk partials and, from N = 512 on, a copy of h in
 *              the order the large-batch kernel loads it: N rounded up to 256
 *              rows x D bf16; contents on entry ignored)
 * Errors: RA_ERR_NULL; RA_ERR_SHAPE (N < 0, V <= 0, D <= 0);
 *         RA_ERR_UNSUPPORTED (D not a multiple of 64); RA_ERR_WORKSPACE;
 *         RA_ERR_HIP. N == 0 returns RA_OK without launching anything.
 */
size_t token_logprob_workspace_size(int32_t N, int32_t V, int32_t D);
int token_logprob(const void *h, const void *W, const int32_t *targets, int32_t N, int32_t V,
                  int32_t D, float scale, float *logprob, float *lse, void *workspace,
                  size_t workspace_bytes, hipStream_t stream);

/*
 * The same log-probabilities from a packed copy of the LM-head matrix. The
 * matrix is constant for a policy version, so it can be repacked once into
 * the order the kernel's matrix products consume it; each wave then reads
 * 4 KB contiguous per 64-dim step instead of 32 rows 128 bytes at a time,
 * and the waves on one step read one narrow window of memory.
 * Results are bitwise those of token_logprob on the unpacked matrix.
 *
 * Packed layout: bf16, 16-byte units; with T = ceil(V / 384) * 12 tiles of
 * 32 rows (V rounded up to a multiple of 384), unit
 *   i = ((s * T + tile) * 4 + u) * 64 + lane
 * holds W[32 * tile + lane % 32][64 * s + 32 * (lane / 32) + 8 * u + 0..7],
 * zeros for rows at or past V. ABI versions 4 and 5 stored the units tile by
 * tile, i = ((tile * (D / 64) + s) * 4 + u) * 64 + lane, and version 4 rounded
 * V up to 256 rows: a copy made by an older library must be packed again.
 *
 * token_logprob_packed_weight_size: bytes of the packed copy (0 if V <= 0,
 *   D <= 0 or D is not a multiple of 64).
 * token_logprob_pack_weight: writes the packed copy of W (bf16 [V][D]) into
 *   W_packed (device, packed_bytes >= the size above). Errors: RA_ERR_SHAPE
 *   (V <= 0, D <= 0), RA_ERR_NULL, RA_ERR_UNSUPPORTED (D % 64 != 0),
 *   RA_ERR_WORKSPACE (packed_bytes too small), RA_ERR_HIP.
 * token_logprob_packed: token_logprob with W_packed in place of W; the same
 *   arguments, errors and workspace size.
 */
size_t token_logprob_packed_weight_size(int32_t V, int32_t D);
int token_logprob_pack_weight(const void *W, int32_t V, int32_t D, void *W_packed,
                              size_t packed_bytes, hipStream_t stream);
int token_logprob_packed(const void *h, const void *W_packed, const int32_t *targets, int32_t N,
                         int32_t V, int32_t D, float scale, float *logprob, float *lse,
                         void *workspace, size_t workspace_bytes, hipStream_t stream);

/*
 * Drawing tokens: one token a row from a row of logits (Sec. 3.3.2: every agent step is a
 * completion; Sec. 3.3.3: each generated token is returned with its log-probability), by
 * the row's own sampling parameters and a given uniform random number. Stands behind the
 * LM head as token_logprob does: that scores given tokens, this draws them.
 * For row n, with z the logits (NaN counts as -inf) and M the largest:
 *   1. weight of v: e_v = exp((z_v - M) / T), T = temperature[n] (NULL: 1);
 *   2. order the elements by logit, largest first, equal ones by index, lowest first;
 *   3. top-k keeps the first k = top_k[n] (NULL, k <= 0 or k >= V: all);
 *   4. top-p keeps, of those, each whose predecessors weigh less than p = top_p[n] times
 *      what top-k kept (NULL, p >= 1 or NaN: all), always the first one;
 *   5. min-p keeps, of those, each with e_v >= min(min_p[n], 1) (NULL, <= 0 or NaN: all);
 *   6. the token is the first v, in the order of the indices, at which the running sum of
 *      the kept weights exceeds uniform[n] times their whole sum S;
 *      logprob = (z_v - M) / T - ln S: under the distribution that was drawn from.
 * T <= 0 or NaN is greedy: the lowest index of M, logprob 0. Logits of -inf are never
 * drawn; a row of nothing else gives token -1 and logprob NaN. If M is +inf the elements
 * at +inf share the weight. uniform[n] is taken into [0, 1) (NaN as 0). Weights are summed
 * as whole numbers of 2^-44 of the largest one (exact in any order; weights below half of
 * that are never drawn), so that the draw is that of sums in 64-bit floating point.
 *
 *   logits       fp32 or bf16 (logits_dtype) [N] rows of V, row_stride elements apart
 *                (any alignment of an element)
 *   temperature  fp32 [N] or NULL; top_k int32 [N] or NULL; top_p, min_p fp32 [N] or NULL
 *   uniform      fp32 [N] in [0, 1)
 *   tokens       int32 [N]
 *   logprob      fp32 [N] or NULL
 *   workspace    device scratch of at least token_sample_workspace_size(N, V) bytes (9 KB a
 *                row and 1 to 5 bytes a logit), 16-byte aligned (contents on entry ignored).
 *                Calls that share one must not overlap.
 * Errors: RA_ERR_NULL; RA_ERR_SHAPE (N < 0, V <= 0, row_stride < V with N > 1);
 *         RA_ERR_UNSUPPORTED (an unknown logits_dtype, V > 2^19, N > 2^20);
 *         RA_ERR_WORKSPACE; RA_ERR_HIP. N == 0 returns RA_OK without launching anything.
 */
typedef enum { RA_LOGITS_FP32 = 0, RA_LOGITS_BF16 = 1 } ra_logits_dtype;
size_t token_sample_workspace_size(int32_t N, int32_t V);
int token_sample(const void *logits, int32_t logits_dtype, int32_t N, int32_t V,
                 int64_t row_stride, const float *temperature, const int32_t *top_k,
                 const float *top_p, const float *min_p, const float *uniform, int32_t *tokens,
                 float *logprob, void *workspace, size_t workspace_bytes, hipStream_t stream);

/*
 * Linear attention with a decay for each KV head: decode and append for layers that keep a
 * state of fixed size instead of cached keys (the paper does not describe model internals;
 * such layers take the place of the paged attention in some of a model's layers, and serve
 * the same steps: Sec. 3.3.2 one token against the whole history, Sec. 3.3.3 the
 * observation tokens after it). For query head h and KV head g = h / (Hq / Hkv), with
 * l_g = exp(log_decay[g]):
 *   S_t = l_g S_{t-1} + k_t v_t^T         (S [128 key dims][128 value dims], fp32)
 *   o_t = scale * S_t^T q_t
 * A row's state lives in a pool, states[slots[b]], and is updated in place; the state
 * before a row's first token is zero whatever the pool holds. Slots of one call must
 * differ. The state is kept to fp32 accuracy: append multiplies the decayed values in three
 * bf16 parts each. Its scores, and the state as it meets the queries, are taken in two bf16
 * parts each (off by 2^-17 of every term of their sums), and out is rounded to bf16 (nearest
 * even) in both calls. An infinite or NaN input never reaches an earlier token's results;
 * the results and the state it reaches may hold NaN where the formula has an infinity.
 *
 * rollout_linear_attn_decode: one token a row.
 *   q          bf16 [B][Hq][128];  k_new, v_new  bf16 [B][Hkv][128]
 *   states     fp32 [num_slots][Hkv][128][128], read and written
 *   slots      int32 [B]; a row whose slot is outside [0, num_slots) gives out = 0
 *   kv_lens    int32 [B]: tokens of the row with this one (1: its first). Rows with
 *              kv_lens[b] <= 0 give out = 0 and leave their state as it is.
 *   log_decay  fp32 [Hkv], <= 0 (larger values and NaN count as 0; -inf: no memory)
 *   out        bf16 [B][Hq][128]
 * rollout_linear_attn_append: row b's new tokens are packed rows cu_q[b] .. cu_q[b+1]-1.
 *   q          bf16 [total_q][Hq][128];  k_new, v_new  bf16 [total_q][Hkv][128]
 *   cu_q       int32 [B+1]; tokens behind cu_q[B] are not touched
 *   ctx_lens   int32 [B]: tokens of the row before these (<= 0: none, the state is zero)
 *   max_q_len  host: an upper bound of cu_q[b+1] - cu_q[b]
 *   out        bf16 [total_q][Hq][128]
 *   workspace  device scratch of at least rollout_linear_attn_append_workspace_size(B, Hq,
 *              Hkv, total_q, max_q_len) bytes (contents on entry ignored), 16-byte
 *              aligned; NULL where the size is 0. Calls that share one must not overlap.
 *   The rest as for decode; rows without tokens leave their state as it is. Whether
 *   long rows are cut into stretches, and with it the order of fp32 sums, depends on B, Hq,
 *   Hkv, total_q and max_q_len alone.
 * Errors: RA_ERR_NULL; RA_ERR_SHAPE (B < 0, Hq or Hkv or num_slots <= 0, Hq % Hkv,
 *         total_q < 0, max_q_len < 0, scale not finite); RA_ERR_UNSUPPORTED (Hq / Hkv > 32,
 *         B > 65535, Hq > 65535, B * Hkv > 2^22, or q, k_new, v_new, states or out not
 *         16-byte aligned); RA_ERR_WORKSPACE; RA_ERR_HIP. B == 0, total_q == 0 or
 *         max_q_len == 0 launch nothing.
 */
int rollout_linear_attn_decode(const void *q, const void *k_new, const void *v_new, float *states,
                               const int32_t *slots, int32_t num_slots, const int32_t *kv_lens,
                               const float *log_decay, int32_t B, int32_t Hq, int32_t Hkv,
                               float scale, void *out, hipStream_t stream);
size_t rollout_linear_attn_append_workspace_size(int32_t B, int32_t Hq, int32_t Hkv,
                                                 int32_t total_q, int32_t max_q_len);
int rollout_linear_attn_append(const void *q, const void *k_new, const void *v_new,
                               const int32_t *cu_q, const int32_t *ctx_lens, float *states,
                               const int32_t *slots, int32_t num_slots, const float *log_decay,
                               int32_t B, int32_t Hq, int32_t Hkv, int32_t total_q,
                               int32_t max_q_len, float scale, void *out, void *workspace,
                               size_t workspace_bytes, hipStream_t stream);

/*
 * Block tables from lengths: the bookkeeping of a step on the GPU, so that a step whose
 * lengths are only known there (sampled stops, captured graphs) needs no host between its
 * calls. Pages that no row owns are on a free list (free_pages[0 .. *free_count), taken
 * and given back at its end).
 *
 * kv_block_table_extend gives row b the pages that its tokens start_pos[b] ..
 * start_pos[b] + num_new[b] - 1 need beyond the ceil(start_pos[b] / 16) it has:
 *   block_table[b][j] = the next page off the list, rows in order, for
 *       j in [ceil(start_pos / 16), ceil((start_pos + num_new) / 16)); other entries stay
 *   cu_new[b]   = sum of num_new before b (B+1 entries)        } the arguments of
 *   kv_lens[b]  = start_pos[b] + num_new[b]                    } kv_page_write and decode
 *   slot_map[cu_new[b] + t] = page * 16 + (start_pos[b] + t) % 16 of each new token (its
 *       place in a pool laid out by tokens), -1 from cu_new[B] on
 *   *taken      = pages taken off the list
 * All or nothing: if the list is too short, a row would pass its table (bt_stride * 16
 * tokens), the new tokens are more than total_new, or a length or the list's count is out
 * of range, *taken = -1, the list and the table stay, and the outputs are those of no new
 * token (cu_new 0, kv_lens = start_pos, slot_map -1): a kv_page_write that follows writes
 * nothing.
 * kv_block_table_release puts the pages ceil(keep_lens[b] / 16) .. ceil(lens[b] / 16) - 1
 * of every row back on the list (a row that ends: keep 0; a draft that is cut: its new
 * length); table entries stay. Releasing what an extend took, with lens its kv_lens and
 * keep_lens its start_pos, restores the list exactly. *released = pages given back, or -1
 * with nothing changed if keep_lens[b] is not in [0, lens[b]], a length passes the table,
 * or the list would pass its capacity.
 *
 *   start_pos, num_new, lens, keep_lens  int32 [B]
 *   free_pages   int32 [free_capacity], free_count int32 [1] (read and written)
 *   block_table  int32 [B][bt_stride], written by extend
 *   total_new    host: an upper bound of the sum of num_new; slot_map's length
 *   max_pages    host: how many pages a release may give back (more are correct, but
 *                slower: it sizes the launch); B * bt_stride always holds
 *   cu_new       int32 [B+1];  kv_lens int32 [B];  taken, released int32 [1]
 *   slot_map     int64 [total_new] or NULL
 * What a call writes (the outputs, extend's block_table, the free list) must not share memory
 * with another of its arrays: extend cannot set the lengths in place. Calls on one free list
 * must not overlap in time.
 * Errors: RA_ERR_NULL; RA_ERR_SHAPE (B < 0, bt_stride <= 0, total_new < 0, max_pages < 0,
 *         free_capacity < 0); RA_ERR_UNSUPPORTED (B > 65535, bt_stride * 16 > 2^31 - 1,
 *         arrays that share memory as above); RA_ERR_HIP. With B == 0 (row arrays may be NULL) extend writes cu_new[0] = 0,
 *         *taken = 0 and the slots' -1, release *released = 0.
 */
int kv_block_table_extend(const int32_t *start_pos, const int32_t *num_new,
                          const int32_t *free_pages, int32_t *free_count, int32_t free_capacity,
                          int32_t *block_table, int32_t B, int32_t bt_stride, int32_t total_new,
                          int32_t *cu_new, int32_t *kv_lens, int64_t *slot_map, int32_t *taken,
                          hipStream_t stream);
int kv_block_table_release(const int32_t *lens, const int32_t *keep_lens,
                           const int32_t *block_table, int32_t B, int32_t bt_stride,
                           int32_t *free_pages, int32_t *free_count, int32_t free_capacity,
                           int32_t max_pages, int32_t *released, hipStream_t stream);

/*
 * Trees of drafted tokens: a step that checks several guessed continuations of a trajectory
 * at once, for rollouts that are bound by decode (Sec. 3.3.1, 3.3.2: an agent's steps wait for
 * its completions one after the other). A row's tree has T nodes, packed at cu_q[b] ..
 * cu_q[b+1]-1; node 0, the root, is the token that is known (the last one drawn), and every
 * other node is a guess that follows its parent, a node before it. A step is
 *   kv_block_table_extend, draft_tree_mask, kv_page_write (node i at position ctx + i),
 *   rollout_attn_decode_tree in each layer, the LM head,
 *   token_logits_adjust, token_sample (one token a node: chosen), draft_tree_accept,
 *   kv_page_compact in each layer, kv_block_table_release (keep_lens = the new kv_lens).
 * In a model with rotary embedding a node's key and query are rotated at positions[i], by the
 * caller and before these calls: kv_page_write_rope and rollout_attn_append_write_rope rotate at
 * ctx + i, the node's place in the pages, which is not its position where it has siblings.
 * The tokens it emits are those that were drawn, node after node, so their distribution is
 * that of steps of one token whatever the guesses are.
 *
 * draft_tree_mask: from the parents, the mask of each node (itself and its ancestors) and
 * its position.
 *   parents     int32 [total_q]: the parent's index in its row, below the node's own; anything
 *               else: the node has none
 *   cu_q        int32 [B+1];  ctx_lens  int32 [B] or NULL (0)
 *   max_q_len   host: an upper bound of T, at most RA_MAX_DRAFT_NODES
 *   mask_words  host: 64-bit words of a mask, at least ceil(max_q_len / 64)
 *   tree_mask   uint64 [total_q][mask_words]: bit j of a node's mask (word j / 64, bit j % 64)
 *   positions   int32 [total_q] or NULL: ctx_lens[b] + ancestors of the node
 * draft_tree_accept: the walk of the chosen tokens down the tree. From the root on, the next
 * node is the first child (lowest index) of the last one whose drafted token is the one chosen
 * there; the walk ends where there is none.
 *   draft_tokens  int32 [total_q];  chosen  int32 [total_q], the token drawn behind each node
 *                 (negative: none, the walk ends)
 *   path        int32 [total_q]: row b's nodes on the walk, ascending, from cu_q[b] on, then -1
 *   tokens      int32 [total_q]: chosen[] of those nodes: the tokens that the step emits
 *   accepted    int32 [B]: nodes on the walk (0 for a row without nodes)
 *   kv_lens     int32 [B]: ctx_lens[b] + accepted[b]
 *   next_tokens int32 [B]: the last of the row's tokens, the next step's root (-1: no nodes)
 * Entries behind cu_q[B] are not touched; what a call writes must not share memory with another
 * of its arrays.
 * Errors: RA_ERR_NULL; RA_ERR_SHAPE (negative sizes, too few mask_words);
 *         RA_ERR_UNSUPPORTED (B > 65535, max_q_len > RA_MAX_DRAFT_NODES, shared memory);
 *         RA_ERR_HIP. B == 0 launches nothing, nor does draft_tree_mask with total_q == 0 or
 *         max_q_len == 0; draft_tree_accept sets the rows' outputs then too (with total_q == 0
 *         the nodes' arrays may be NULL).
 */
#define RA_MAX_DRAFT_NODES 1024
int draft_tree_mask(const int32_t *parents, const int32_t *cu_q, const int32_t *ctx_lens,
                    int32_t B, int32_t total_q, int32_t max_q_len, int32_t mask_words,
                    uint64_t *tree_mask, int32_t *positions, hipStream_t stream);
int draft_tree_accept(const int32_t *parents, const int32_t *draft_tokens, const int32_t *chosen,
                      const int32_t *cu_q, const int32_t *ctx_lens, int32_t B, int32_t total_q,
                      int32_t max_q_len, int32_t *path, int32_t *tokens, int32_t *accepted,
                      int32_t *kv_lens, int32_t *next_tokens, hipStream_t stream);

/*
 * Decode of drafted trees: attention of every node over the row's cache and over the nodes
 * that its mask names. Node i of row b (packed t = cu_q[b] + i, its key and value in the pool at
 * position ctx_lens[b] + i) attends keys 0 .. ctx_lens[b] - 1 and ctx_lens[b] + j for every
 * j < T whose bit in tree_mask[t] is set:
 *   out[t][h] = softmax_j(scale * <q[t][h], K_j>) . V_j,  lse likewise.
 * One node that sees itself is rollout_attn_decode with kv_lens = ctx_lens + 1; a chain is
 * rollout_attn_append, with decode's precision. A node that sees no key gives out = 0 and lse
 * = -inf. A masked key and value reach no result, infinite or NaN as they may be. A result that an
 * infinite value reaches, of the context or of a node, may hold NaN where the formula has an
 * infinity: the second part of a weight (below) can be 0 or negative.
 *
 *   q           bf16 [total_q][Hq][128]
 *   cu_q        int32 [B+1];  ctx_lens  int32 [B]
 *   tree_mask   uint64 [total_q][mask_words]; bits at and past T are ignored
 *   max_q_len   host: an upper bound of T, at most RA_MAX_DRAFT_NODES
 *   max_kv_len  host: an upper bound of ctx_lens[b] + T; <= bt_stride * 16
 *   out         fp32 [total_q][Hq][128];  lse  fp32 [total_q][Hq] or NULL; rows behind cu_q[B]
 *               are not touched
 *   workspace   device scratch of at least rollout_attn_decode_tree_workspace_size(B, Hq, Hkv,
 *               total_q, max_q_len, max_kv_len) bytes (contents on entry ignored); NULL where
 *               the size is 0. Calls that share one must not overlap. The size can fall, to 0
 *               too, as B, max_q_len or max_kv_len grows (32 heads on 8, 8 nodes, 4,096 keys: 17 MB
 *               for 16 rows, none for 64), so that of a loop's largest call need not hold the
 *               smaller ones: rollout_attn_decode_tree_max_workspace_size is enough for all
 *               calls of up to that many rows, nodes and keys (at most 68 MB and 8 bytes a row).
 * Longer calls (max_kv_len above 512, and more where there are many rows and KV heads) are cut
 * into equal shares of their work. Where rows are cut, and with it the order of fp32 sums, depends on
 * the lengths and trees' sizes of all the call's rows, their order and number, Hq, Hkv, max_q_len and
 * max_kv_len, and on nothing else: the same call gives
 * the same bits, while a row's result beside other rows can differ by the order of sums.
 * Weights meet the values in two bf16 parts, off by 2^-16 of a weight, as in decode (in three, off
 * by 2^-24, where max_q_len * Hq / Hkv is at most 32 and the pools are bf16).
 * Errors: as rollout_attn_append; RA_ERR_SHAPE also for too few mask_words; RA_ERR_UNSUPPORTED
 *         (Hq / Hkv > 256, B > 65535, max_q_len > RA_MAX_DRAFT_NODES, max_kv_len > 2^30, total_q *
 *         Hq >= 2^31, a launch of 2^32 threads or more: B * Hkv tiles of up to 128 query rows >= 2^24
 *         or of 256 >= 2^23 where rows are not cut, total_q * Hkv >= 2^26 where they are; q, pools,
 *         out or workspace not 16-byte aligned).
 *         B == 0, total_q == 0 or max_q_len == 0 launch nothing.
 */
size_t rollout_attn_decode_tree_workspace_size(int32_t B, int32_t Hq, int32_t Hkv,
                                               int32_t total_q, int32_t max_q_len,
                                               int32_t max_kv_len);
size_t rollout_attn_decode_tree_max_workspace_size(int32_t B, int32_t Hq, int32_t Hkv,
                                                   int32_t max_q_len, int32_t max_kv_len);
int rollout_attn_decode_tree(const void *q, const int32_t *cu_q, const int32_t *ctx_lens,
                             const uint64_t *tree_mask, int32_t mask_words, const ra_paged_kv *kv,
                             int32_t B, int32_t Hq, int32_t total_q, int32_t max_q_len,
                             int32_t max_kv_len, float scale, float *out, float *lse,
                             void *workspace, size_t workspace_bytes, hipStream_t stream);

/*
 * Logits before a token is drawn: penalties for tokens that a trajectory holds already, biases,
 * and masks of what a grammar (a tool call's schema) allows. Stands between the LM head and
 * token_sample. For row n of logits, with b its history row, s_v whether token v is in the
 * history, c_v how often it is in the part behind the prompt:
 *   1. z_v <- (z_v > 0 ? z_v / repetition[b] : z_v * repetition[b])   where s_v
 *   2. z_v <- z_v - frequency[b] * c_v - presence[b]                  where c_v > 0
 *   3. z_v <- z_v + bias_values[e]   for the last e in cu_bias[b] .. cu_bias[b+1]-1 with
 *                                    bias_tokens[e] = v
 *   4. z_v <- -inf                   where the row's mask has bit v clear
 * in fp32, rounded once (to nearest even) to the type of the logits; elements that none of them
 * concerns keep their bits. Tokens outside [0, V) are passed over. A repetition that is not
 * finite and > 0 counts as 1, a frequency or presence that is not finite as 0.
 *
 *   logits        fp32 or bf16 (logits_dtype) [N] rows of V, row_stride elements apart (any
 *                 alignment of an element); out likewise, out_stride apart; out = logits with
 *                 the same stride works in place (and reads and writes only what changes).
 *                 Rows of trees share the counting of their history where rows are a multiple
 *                 of 16 bytes apart; otherwise each row's is counted by itself (slower)
 * ra_logits_adjust (all arrays may be NULL where not said otherwise):
 *   history       int32 [B] rows of history_width, history_stride apart, of which history_lens[b]
 *                 (int32 [B], needed with history; more than history_width count as that many)
 *                 are the row's tokens, the first prompt_lens[b] (int32 [B]; NULL: 0) of them
 *                 its prompt
 *   repetition, frequency, presence  fp32 [B] (NULL: off)
 *   bias_tokens   int32 [num_bias], bias_values fp32 [num_bias], cu_bias int32 [B+1] (needed with
 *                 bias_tokens)
 *   allowed       uint32 [num_allowed] rows of bits, allowed_stride words apart: bit v % 32 of
 *                 word v / 32; allowed_rows int32 [N]: the row's mask (outside
 *                 [0, num_allowed): none; NULL: mask n)
 *   cu_rows       int32 [B+1]: history row b has the rows cu_rows[b] .. cu_rows[b+1]-1 of
 *                 logits (rows behind cu_rows[B] are not touched); NULL: B = N, a row each
 *   draft_tokens  int32 [N], tree_mask uint64 [N][mask_words] (both or neither, with cu_rows):
 *                 the rows are nodes of drafted trees; the drafted tokens of the nodes in row
 *                 n's mask are in its history, behind the prompt. The root's is among them, so
 *                 history ends before the root (history_lens = the step's ctx_lens): a token
 *                 in both counts twice
 * What is written must not share memory with another array (but in place as above).
 * Errors: RA_ERR_NULL; RA_ERR_SHAPE (N < 0, B < 0, V <= 0, a stride < V with N > 1,
 *         history_width < 0, history_stride < history_width with B > 1, num_bias < 0,
 *         allowed_stride < ceil(V / 32), num_allowed < 0, mask_words <= 0 with tree_mask, B != N
 *         without cu_rows); RA_ERR_UNSUPPORTED (an unknown
 *         logits_dtype, V > 2^24, a launch of 2^32 threads or more: N * ceil(V / 8184) >= 2^23, with
 *         cu_rows a 32nd of it, shared memory); RA_ERR_HIP.
 *         N == 0 or B == 0 launch nothing.
 */
typedef struct {
  const int32_t *history, *history_lens, *prompt_lens;
  int64_t history_stride;
  const float *repetition, *frequency, *presence;
  const int32_t *bias_tokens;
  const float *bias_values;
  const int32_t *cu_bias;
  int32_t history_width, num_bias;
  const uint32_t *allowed;
  const int32_t *allowed_rows;
  int64_t allowed_stride;
  int32_t num_allowed;
  int32_t mask_words;
  const int32_t *cu_rows;
  const int32_t *draft_tokens;
  const uint64_t *tree_mask;
} ra_logits_adjust;
int token_logits_adjust(const void *logits, int32_t logits_dtype, int32_t N, int32_t V,
                        int64_t row_stride, const ra_logits_adjust *adjust, int32_t B, void *out,
                        int64_t out_stride, hipStream_t stream);

/*
 * Rows that share pages (Sec. 4: several rollouts of one task; rollout_attn_decode_shared_prefix
 * reads such pages once for a group). shares[p] (int32 [num_pages], zeros to begin with) counts
 * the rows that hold page p beyond the first; kv_block_table_extend's pages have none.
 *
 * kv_block_table_fork gives row dst_rows[i] the first lens[i] tokens of row src_rows[i]: its
 * whole pages are shared (the same entries, one more share each), and where lens[i] is not a
 * multiple of 16 the last page is one off the free list (in the order of the forks), to be
 * filled by kv_page_copy in each layer:
 *   copy_src[i], copy_dst[i] = the pages to copy between; -1, -1 where there is none
 *   *taken = pages taken off the list
 * dst_rows' earlier entries are overwritten, not released. All or nothing: if the list is too
 * short, a row is outside [0, B), a length outside [0, bt_stride * 16], two forks go into one
 * row, one goes into a row that another (or itself) comes from, or the list's count is out of
 * range, *taken = -1, copy_src and copy_dst are -1 and nothing else changes.
 * A shared page must not be written: append behind lens[i], and do not cut a row back into a
 * page that it shares (whole pages may be released).
 *
 * kv_block_table_release_shared is kv_block_table_release for such rows: each entry it covers
 * takes one holder off its page, and a page goes back on the free list when none is left (its
 * last entry in the order of rows counts for its place). *released = pages put on the list, or
 * -1 with nothing changed where kv_block_table_release would refuse for a length or the list's
 * count. Entries that name no page are passed over.
 *   workspace   at least kv_block_table_release_shared_workspace_size(B) bytes, 16-byte aligned
 *
 * kv_page_copy copies the pages src_pages[i] to dst_pages[i] (int32 [n]) of both pools, all KV
 * heads, bit for bit; pairs with a page outside [0, num_pages) are passed over. No page may be
 * the destination of two pairs, or of one and the source of another. The block table and
 * its bt_stride are not used, whatever they hold.
 *
 * What is written must not share memory with another array. Calls on one free list must not
 * overlap in time.
 * Errors: RA_ERR_NULL; RA_ERR_SHAPE (negative sizes, bt_stride <= 0, num_pages <= 0,
 *         free_capacity < num_pages for the release); RA_ERR_UNSUPPORTED (B > 65535, n > 65535
 *         for a fork, n * Hkv >= 2^24, B * bt_stride >= 2^30 for the release, bt_stride * 16 >
 *         2^31 - 1, shared memory, pools not 16-byte aligned); RA_ERR_WORKSPACE; RA_ERR_HIP.
 *         n == 0 forks set *taken = 0, B == 0 releases *released = 0; n == 0 copies launch
 *         nothing.
 */
int kv_block_table_fork(const int32_t *src_rows, const int32_t *dst_rows, const int32_t *lens,
                        int32_t n, int32_t *block_table, int32_t B, int32_t bt_stride,
                        int32_t *shares, int32_t num_pages, const int32_t *free_pages,
                        int32_t *free_count, int32_t free_capacity, int32_t *copy_src,
                        int32_t *copy_dst, int32_t *taken, hipStream_t stream);
size_t kv_block_table_release_shared_workspace_size(int32_t B);
int kv_block_table_release_shared(const int32_t *lens, const int32_t *keep_lens,
                                  const int32_t *block_table, int32_t B, int32_t bt_stride,
                                  int32_t *shares, int32_t num_pages, int32_t *free_pages,
                                  int32_t *free_count, int32_t free_capacity, int32_t *released,
                                  void *workspace, size_t workspace_bytes, hipStream_t stream);
int kv_page_copy(const ra_paged_kv *kv, const int32_t *src_pages, const int32_t *dst_pages,
                 int32_t n, hipStream_t stream);

/*
 * Compaction: the kept tokens at a row's end move together, e.g. the accepted path of a drafted
 * tree behind the context (src_index = path, counts = accepted, start_pos = ctx_lens).
 * Token start_pos[b] + src_index[cu_src[b] + i] of row b moves to position start_pos[b] + i,
 * for i in [0, counts[b]), keys and values of all KV heads, bit for bit (codes of fp8 pools).
 * A row's indices must ascend strictly from 0 or more (so no token moves back); entries that
 * are below their own i, or past the row's table, are passed over. Slots that no token moves
 * to keep their contents. Rows of one call must not share the pages that they move in.
 *
 *   kv         pools written in place, block table read
 *   start_pos  int32 [B];  cu_src  int32 [B+1];  src_index  int32 [total]
 *   counts     int32 [B] or NULL (all of cu_src[b] .. cu_src[b+1]-1)
 *   max_count  host: an upper bound of the tokens of a row
 * Errors: RA_ERR_NULL; RA_ERR_SHAPE (negative sizes); RA_ERR_UNSUPPORTED (the page layout,
 *         B > 65535, B * Hkv >= 2^24, pools not 16-byte aligned); RA_ERR_HIP. B == 0, total == 0
 *         or max_count == 0 launch nothing.
 */
int kv_page_compact(const ra_paged_kv *kv, const int32_t *start_pos, const int32_t *cu_src,
                    const int32_t *src_index, const int32_t *counts, int32_t B, int32_t total,
                    int32_t max_count, hipStream_t stream);

/*
 * Page write: append new tokens' keys and values to each trajectory's cache
 * (Sec. 3.3.3: the tokens of earlier turns are kept as they are and only the
 * new observation tokens are tokenised and added after them; Sec. 3.3.2: each
 * agent step's completion extends the same history, so every decoded token is
 * added too). The cache that later steps reuse (Sec. 3.3.2, load balancing
 * keeps a task on one backend for this) is therefore only ever extended at
 * its end, one chunk or one token per row and call.
 * The write is a bit copy into bf16 pools and a quantization into fp8 pools
 * (each element stored as encode(fp32(x) * fp32(1 / scale)), see the layout
 * above). Row b's new tokens are packed rows cu_new[b] .. cu_new[b+1]-1 of
 * k_new / v_new; token t of the row goes to logical position start_pos[b] + t,
 * i.e. page bt[b][(start_pos[b] + t) / 16], slot (start_pos[b] + t) % 16. No
 * other pool byte changes. Rows of one call must not write the same slot.
 *
 *   k_new, v_new  bf16 [total_new][Hkv][128] (token-major), read only
 *   cu_new        int32 [B+1], non-decreasing, cu_new[0] = 0
 *   start_pos     int32 [B]
 *   kv            pools written in place (caller-owned), block table read
 *   B, total_new  host: rows and packed tokens of the call
 *   max_new       host: an upper bound of cu_new[b+1] - cu_new[b]
 *   max_pos       host: an upper bound of start_pos[b] + new tokens of row b;
 *                 <= bt_stride * 16
 * Errors: RA_ERR_NULL (a NULL pointer), RA_ERR_SHAPE (negative sizes,
 *         max_pos > bt_stride * 16, max_new > max_pos, bad fp8 scales),
 *         RA_ERR_UNSUPPORTED (page_size != 16, head_dim != 128, B > 65535),
 *         RA_ERR_HIP. B == 0, total_new == 0 or max_new == 0 launch nothing.
 */
int kv_page_write(const void *k_new, const void *v_new, const int32_t *cu_new,
                  const int32_t *start_pos, const ra_paged_kv *kv, int32_t B, int32_t total_new,
                  int32_t max_new, int32_t max_pos, hipStream_t stream);

/*
 * Page gather (test and export helper): read back, in logical order, the
 * cached history of each trajectory that the attention entry points attend to
 * (Sec. 3.3.2: a task's later calls reuse its cached prefix; Sec. 3.3.3: that
 * prefix is the retained token sequence with the observations appended). It
 * copies logical tokens 0 .. lens[b]-1 of every row out of the pages (token j
 * from page bt[b][j / 16], slot j % 16) into packed token-major arrays; row b
 * starts at packed row cu_out[b]. A bit copy of the stored elements (E4M3
 * codes for fp8 pools); it checks a write and exports a trajectory's cache.
 *
 *   kv       pools and block table, read only
 *   lens     int32 [B]; max_len host upper bound of lens (<= bt_stride * 16)
 *   cu_out   int32 [B+1], non-decreasing, cu_out[0] = 0, cu_out[B] <= total
 *   k_out, v_out  [total][Hkv][128] of the pools' element type (caller-owned,
 *            written)
 * Errors: RA_ERR_NULL, RA_ERR_SHAPE (negative sizes, max_len > bt_stride *
 *         16), RA_ERR_UNSUPPORTED (B > 65535, unsupported page layout),
 *         RA_ERR_HIP. B == 0, total == 0 or max_len == 0 launch nothing.
 */
int kv_page_gather(const ra_paged_kv *kv, const int32_t *lens, const int32_t *cu_out, int32_t B,
                   int32_t total, int32_t max_len, void *k_out, void *v_out,
                   hipStream_t stream);

#ifdef __cplusplus
}
#endif

#endif /* ROLLOUT_ATTN_H */
