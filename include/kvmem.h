/* kvmem.h - C ABI of the KVMem recall step on one NVIDIA B200 (sm_100a).
 *
 * One recall step (paper Sec. 4.1, Sec. 5.2): score every historical paged-KV block of a
 * session against the current query through the Mean-K attention-space index, select the
 * top blocks under the active-context budget, assemble the query-dependent execution
 * view from the block table, and run GQA decode attention over that view.
 *
 * Conventions
 *   - Every pointer is marked HOST or DEVICE.  Device buffers, including the pool's backing
 *     storage, views, outputs and workspaces, are owned by the caller; the library owns only
 *     the opaque handle and its host-side metadata and never allocates device memory.
 *   - All device work is enqueued on the given stream (a cudaStream_t passed as void*) and is
 *     asynchronous unless a call says otherwise.  A pool is not thread-safe.  The pool's device must be the calling
 *     thread's current device in every call that enqueues work (KVMEM_E_STATE otherwise).
 *   - Every call returns a kvmem_status_t.  Argument, state and capacity errors are detected
 *     on the host before anything is enqueued and leave the pool unchanged; kvmem_last_error()
 *     then describes the failure.  Anomalies seen on the device (a block id out of range, a
 *     bounded wait that expired) set a sticky status word read by kvmem_device_status().
 *   - Element type of K, V, q and the index is bf16 (2 bytes).  Scores, attention outputs
 *     and log-sum-exp values are fp32.
 *   - Logical block ids are the append order within a session, i.e. chronological order
 *     (Sec. 5.2, block records).  Only whole blocks of block_tokens tokens exist: the Mean-K
 *     index covers completed blocks only (Sec. 5.2).
 *   - Keys and queries are taken to be position-independent already (Sec. 4.3, "Mean-K
 *     Retrieval-Index Construction"); K is copied into the view unchanged.
 *   - Query head h reads KV head h / (n_q_heads / n_kv_heads).
 */
#ifndef KVMEM_H_
#define KVMEM_H_

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef struct kvmem_pool kvmem_pool_t; /* opaque; created and destroyed by the library */

typedef enum {
    KVMEM_OK = 0,
    KVMEM_E_INVALID = -1,     /* bad argument (null, out of range, misaligned, partial block)   */
    KVMEM_E_CAPACITY = -2,    /* pool, session or caller buffer too small                       */
    KVMEM_E_STATE = -3,       /* page already in use, session empty, stale handle               */
    KVMEM_E_CUDA = -4,        /* a CUDA runtime or driver call failed                           */
    KVMEM_E_TIMEOUT = -5,     /* device status: a bounded wait inside a kernel gave up          */
    KVMEM_E_UNSUPPORTED = -6, /* shape outside what the kernels were built for                  */
    KVMEM_E_DEVICE_RANGE = -7 /* device status: a block or page id was out of range and skipped */
} kvmem_status_t;

/* Geometry of the paged KV repository (Sec. 3.1: logical blocks of B_blk tokens; Sec. 5.2:
 * blocks aligned with physical pages). */
typedef struct {
    int32_t n_layers;               /* scored attention layers L (1 in the benchmark configurations)   */
    int32_t n_q_heads;              /* H                                                               */
    int32_t n_kv_heads;             /* G; H % G == 0                                                   */
    int32_t head_dim;               /* d; 128 is what the kernels are built for                        */
    int32_t block_tokens;           /* B_blk; a multiple of 16, at most 256                            */
    int32_t max_sessions;           /* independent workspaces sharing the page pool                    */
    int32_t max_blocks;             /* physical pages in the pool                                      */
    int32_t max_blocks_per_session; /* rows of one session's block table and index                     */
    int32_t device;                 /* CUDA device ordinal                                             */
    int32_t rope_max_positions;     /* 0: no rotary support.  Else the pool holds a cos/sin table for
                                       positions [0, rope_max_positions): the native window, since every
                                       token is encoded and re-encoded inside an execution view (8 bytes x
                                       head_dim / 2 per position)                                      */
    float rope_theta;               /* rotary base (e.g. 1e6); used when rope_max_positions > 0        */
    int32_t rope_in_block_keys;     /* 0: the pages hold raw (position-free) keys.  1 (needs rotary support with
                                       rope_max_positions >= block_tokens; the fused materialise+attend pass on this
                                       layout needs 64-token blocks): a page holds k' = RoPE(k, t), t the token's offset inside its
                                       block, so that a block placed at compact position p0 needs the rotation
                                       of p0 alone: the position-consistent view rotates by one angle set per
                                       block, and the copy-free attention rotates the QUERY back by p0 once per
                                       block instead of every key forward (q . R(p0 + t) k = (R(-p0) q) . R(t) k).
                                       The Mean-K index is built from the raw keys either way              */
    int32_t fp8_pages;              /* 0: pages hold bf16.  1 (head_dim 128, 64-token blocks; rotary support only together
                                       with rope_in_block_keys, in which case the codes are those of RoPE(k, t) and
                                       kvmem_paged_attend_fp8_rope is the position-consistent reader): the
                                       repository itself is FP8 (Sec. 6.1: the KV cache is kept in FP8): a page holds the
                                       E4M3 codes of k / fp8_k_scale ([64 tokens][128] bytes per layer and KV head) and
                                       of v / fp8_v_scale transposed ([128 dims][64 tokens] bytes), i.e. the tiles of the
                                       FP8 execution view; half the memory and half the traffic of every pass over
                                       pages.  kvmem_append_blocks still takes bf16 K and V and builds the bf16 Mean-K
                                       index from them; kvmem_materialize_fp8 and kvmem_paged_attend_fp8 are the calls
                                       that read such pages, the bf16 page readers return KVMEM_E_STATE            */
    float fp8_k_scale;              /* static per-tensor scales of an FP8 repository (positive, finite)              */
    float fp8_v_scale;
} kvmem_pool_config_t;

/* Selection budget (Eq. "active_budget", Eq. "active_capacity" in Sec. 3.1; selector in
 * Sec. 4.3).  The number of blocks kept is
 *     k = min(budget_blocks, floor((max_view_tokens - mandatory_tokens) / block_tokens), NB), k >= 0.
 * The oldest n_sink_blocks and newest n_recent_blocks are kept first (sinks before recents,
 * truncated to k, overlap counted once); remaining slots go to the largest scores, equal
 * scores to the lower block id.  Reserved blocks still take part in the softmax. */
typedef struct {
    int32_t budget_blocks;    /* requested k                                    */
    int32_t max_view_tokens;  /* B_a = min(B_model, B_gpu), in tokens           */
    int32_t mandatory_tokens; /* N(Q_tau): context the view must leave room for */
    int32_t n_sink_blocks;
    int32_t n_recent_blocks;
} kvmem_select_params_t;

/* ---- pure host helpers (no CUDA call) -------------------------------------------------- */

/* Bytes of DEVICE storage kvmem_pool_create needs for this geometry (0 if cfg is invalid).
 * Holds the K/V pages, the Mean-K index, the block tables, a status word and, if enabled, the rotary table. */
size_t kvmem_pool_bytes(const kvmem_pool_config_t* cfg /*HOST*/);

/* The budget clamp above for a session of n_blocks blocks; never negative. */
int32_t kvmem_budget_blocks(const kvmem_select_params_t* params /*HOST*/, int32_t block_tokens, int32_t n_blocks);

/* Bytes of DEVICE workspace kvmem_select needs for n_sessions sessions and n_q_tokens query
 * tokens per session (0 if the arguments are invalid). */
size_t kvmem_select_workspace_bytes(const kvmem_pool_config_t* cfg /*HOST*/, int32_t n_sessions, int32_t n_q_tokens);

/* Bytes of DEVICE workspace kvmem_view_attend needs (split-K partial results). */
size_t kvmem_attend_workspace_bytes(const kvmem_pool_config_t* cfg /*HOST*/, int32_t n_sessions, int32_t n_q_tokens);

/* Description of the calling thread's last failure (static storage, never NULL). */
const char* kvmem_last_error(void);

/* ---- pool lifetime ---------------------------------------------------------------------- */

/* Create a pool inside caller-owned DEVICE storage of at least kvmem_pool_bytes(cfg) bytes,
 * 256-byte aligned.  The storage must outlive the pool.  Clears the tables and the status word
 * (synchronous).  KVMEM_E_UNSUPPORTED if the device is not compute capability 10.x. */
int kvmem_pool_create(const kvmem_pool_config_t* cfg /*HOST*/, void* storage /*DEVICE*/, size_t bytes,
                      kvmem_pool_t** out /*HOST*/);
int kvmem_pool_destroy(kvmem_pool_t* pool);

/* Forget a session's blocks and return its pages to the free list.  The host-side bookkeeping changes at once; the
 * session's block count on the device is cleared on `stream`, so calls enqueued after it on that stream (select, top-k,
 * attention over its pages) see an empty session: n_sel = 0, nothing read.  Work enqueued earlier that still reads
 * the session's pages must have been ordered before any append that reuses them (same stream, or an event). */
int kvmem_session_reset(kvmem_pool_t* pool, int32_t session, void* stream);

/* Blocks appended to a session so far, or a negative status. */
int32_t kvmem_session_blocks(const kvmem_pool_t* pool, int32_t session);

/* ---- repository and index (Sec. 4.3, Eq. "mean_k_index"; Sec. 5.3 "Incremental Indexing") - */

/* Append n_blocks completed blocks to a session: copy their K and V into physical pages,
 * extend the block table and compute the Mean-K entry of each new block,
 *     kbar[l][b][g] = (1/B) * sum_{i in b} k[l][i][g]
 * (fp32 sum in ascending token order, one round-to-nearest-even to bf16).
 *   k, v       DEVICE bf16 [n_blocks * block_tokens][n_layers][n_kv_heads][head_dim], 16-byte aligned;
 *              may be released once the stream has run the call
 *   phys_ids   HOST int32 [n_blocks] page ids to use, or NULL to take free pages in ascending order
 * On a pool created with rope_in_block_keys, k holds raw keys, the index is built from them, and the
 * page receives RoPE(k, t), t = the token's offset inside its block.
 * Errors: KVMEM_E_CAPACITY (session or pool full), KVMEM_E_STATE (page in use), KVMEM_E_INVALID.  The session's block
 * count on the device is raised only after the kernel that writes the new pages and index rows has been enqueued, so
 * a KVMEM_E_CUDA from this call leaves the session as it was, on the host and on the device. */
int kvmem_append_blocks(kvmem_pool_t* pool, int32_t session, const void* k /*DEVICE*/, const void* v /*DEVICE*/,
                        int32_t n_blocks, const int32_t* phys_ids /*HOST*/, void* stream);

/* ---- position-consistent keys (Sec. 4.3: positional encoding removed before indexing and from the
 * query; Sec. 4.4: RoPE applied to raw K at the assigned compact position, V copied unchanged, with
 * precomputed sine/cosine tables).  Needs rope_max_positions > 0.  Rotary variant: pairs (i, i + d/2),
 * frequency theta^(-2i/d), table = fp32 cos/sin of the fp64 angle; a rotated element is four fp32
 * products and two fp32 sums (no fused multiply-add), rounded once to bf16. ------------------------ */

/* kvmem_append_blocks for keys that still carry RoPE: token t of new block i was encoded at position
 * block_pos0[i] + t (its position in the execution window it was computed in).  The encoding is removed,
 * the raw keys are stored in the pages and indexed; block_pos0 is kept in the block record.  (With
 * rope_in_block_keys the raw keys are indexed and the pages receive RoPE(raw, t), t the offset in the block.)
 *   block_pos0  HOST int32 [n_blocks]; every position must lie in [0, rope_max_positions) */
int kvmem_append_blocks_rope(kvmem_pool_t* pool, int32_t session, const void* k_roped /*DEVICE*/, const void* v /*DEVICE*/,
                             int32_t n_blocks, const int32_t* phys_ids /*HOST*/, const int32_t* block_pos0 /*HOST*/,
                             void* stream);

/* Rotate n_rows x n_vec vectors of head_dim elements: y[r][v] = RoPE(x[r][v], positions[r]), or the
 * inverse rotation (inverse != 0), e.g. to bring the current query into the position-independent space
 * the index lives in.  x, y DEVICE bf16 [n_rows][n_vec][head_dim] (may alias); positions DEVICE int32
 * [n_rows].  Rows with a position outside the table are left unwritten and flagged in the status word. */
int kvmem_rope_rotate(kvmem_pool_t* pool, const void* x /*DEVICE*/, void* y /*DEVICE*/, int64_t n_rows, int32_t n_vec,
                      const int32_t* positions /*DEVICE*/, int32_t inverse, void* stream);

/* kvmem_materialize with position-consistent keys: the key of view token j*B + t is the raw key rotated
 * to compact position first_position + j*B + t; values are copied unchanged.  With rope_in_block_keys the
 * stored key already carries the rotation of t and is rotated by first_position + j*B: one set of angles per
 * block (the result differs from the raw-key path by one extra bf16 rounding of the stored key).
 * first_position + budget * B must not exceed rope_max_positions (KVMEM_E_INVALID otherwise). */
int kvmem_materialize_rope(kvmem_pool_t* pool, int32_t session_first, int32_t n_sessions, const int32_t* sel_ids /*DEVICE*/,
                           int32_t sel_stride, const int32_t* n_sel /*DEVICE*/, void* view_k /*DEVICE*/,
                           void* view_v /*DEVICE*/, int32_t view_cap_tokens, int32_t first_position, void* stream);

/* ---- the recall step ----------------------------------------------------------------------- */

/* Scores only (Eq. "kvmem-block-score", Sec. 4.3): the first half of kvmem_select, same arguments and
 * definitions; scores (required) receives score_scale * R for every session.  score_scale (0 selects 1) lets a rank
 * that holds 1/N of the heads of a session write its share of the head mean directly (score_scale = 1/N): the sum of
 * the ranks' outputs is then R, with no arithmetic outside the library. */
int kvmem_score(kvmem_pool_t* pool, int32_t session_first, int32_t n_sessions, const void* q /*DEVICE*/, int32_t n_q_tokens,
                float* scores /*DEVICE*/, float score_scale, void* workspace /*DEVICE*/, size_t workspace_bytes, void* stream);

/* Selection alone (Sec. 4.3: reserve sink and recent blocks, fill the budget with the largest R_b, ties to the
 * lower id, chronological output): the second half of kvmem_select, for scores the caller already has (for
 * example from kvmem_score_host_index).  scores DEVICE fp32 [n_sessions][scores_stride], non-negative; the
 * session lengths are the pool's.  sel_ids, sel_stride, n_sel and errors as in kvmem_select. */
int kvmem_topk(kvmem_pool_t* pool, int32_t session_first, int32_t n_sessions, const float* scores /*DEVICE*/,
               int32_t scores_stride, const kvmem_select_params_t* params /*HOST*/, int32_t* sel_ids /*DEVICE*/,
               int32_t sel_stride, int32_t* n_sel /*DEVICE*/, void* stream);

/* Block relevance against an index that lives in HOST memory (Sec. 5.2: the index is streamed to the GPU in
 * tiles and softmax statistics are carried across tiles; Sec. 5.3 "Incremental Indexing" keeps the index small
 * enough for that).  R is the same quantity kvmem_score computes (Eq. "kvmem-block-score"), for one session.
 *   index_host  HOST bf16 [n_layers][n_kv_heads][index_stride_blocks][head_dim], 16-byte aligned; page-locked
 *               memory makes the copies asynchronous and fast, pageable memory works but serialises
 *   n_blocks    blocks to score (<= index_stride_blocks)
 *   q           DEVICE bf16 [n_q_tokens][n_layers][n_q_heads][head_dim], 1..16 query tokens
 *   tile_blocks blocks per head and tile, a multiple of 128
 *   scores      DEVICE fp32 [n_blocks]
 *   staging     DEVICE, kvmem_score_host_staging_bytes(): two tiles, 256-byte aligned
 *   workspace   DEVICE, kvmem_score_host_workspace_bytes(): fp32 logits of all blocks and the per-tile statistics
 * Tile i + 1 is copied (on a stream the pool owns) while tile i is scored on `stream`; the two are ordered by
 * events only.  When the call returns, work is queued on both streams; `stream` alone has to be waited for.
 * index_host must stay valid until then.  Calls on one pool must not overlap.  Errors: KVMEM_E_INVALID,
 * KVMEM_E_CAPACITY, KVMEM_E_CUDA as elsewhere. */
size_t kvmem_score_host_workspace_bytes(const kvmem_pool_t* pool, int32_t n_blocks, int32_t n_q_tokens, int32_t tile_blocks);
size_t kvmem_score_host_staging_bytes(const kvmem_pool_t* pool, int32_t tile_blocks);
int kvmem_score_host_index(kvmem_pool_t* pool, const void* index_host /*HOST*/, int32_t n_blocks, int32_t index_stride_blocks,
                           const void* q /*DEVICE*/, int32_t n_q_tokens, int32_t tile_blocks, float* scores /*DEVICE*/,
                           void* staging /*DEVICE*/, size_t staging_bytes, void* workspace /*DEVICE*/,
                           size_t workspace_bytes, void* stream);

/* Score and select (Sec. 4.3, Eq. "kvmem-block-score"; selector; Sec. 5.2 tiled scoring with the
 * softmax kept global across tiles).  For each session s in [session_first, session_first + n_sessions):
 *     R_b = sum_m (1/(L*H)) sum_{l,h} softmax_{b' in all blocks of s}( q[m][l][h] . kbar[l][b'][g(h)] / sqrt(d) )_b
 * then the selector described at kvmem_select_params_t.
 *   q          DEVICE bf16 [n_sessions][n_q_tokens][n_layers][n_q_heads][head_dim], 16-byte aligned
 *   sel_ids    DEVICE int32 [n_sessions][sel_stride]: ascending logical ids; entries past n_sel untouched
 *   sel_stride >= the clamped budget of every session
 *   n_sel      DEVICE int32 [n_sessions]
 *   scores     DEVICE fp32 [n_sessions][max_blocks_per_session] receives R (first NB entries), or NULL
 *   workspace  DEVICE, kvmem_select_workspace_bytes(), 256-byte aligned; contents undefined afterwards
 * One query chunk gives one score vector and one selection (sum over its tokens). */
int kvmem_select(kvmem_pool_t* pool, int32_t session_first, int32_t n_sessions, const void* q /*DEVICE*/,
                 int32_t n_q_tokens, const kvmem_select_params_t* params /*HOST*/, int32_t* sel_ids /*DEVICE*/,
                 int32_t sel_stride, int32_t* n_sel /*DEVICE*/, float* scores /*DEVICE*/, void* workspace /*DEVICE*/,
                 size_t workspace_bytes, void* stream);

/* Assemble the execution view (Sec. 4.4 "execution view"; Sec. 5.2): view tokens
 * [j*B, (j+1)*B) of session s are block sel_ids[s][j]'s K and V, fetched through the block table.
 *   view_k, view_v  DEVICE bf16 [n_sessions][n_layers][n_kv_heads][view_cap_tokens][head_dim], 16-byte aligned
 *   n_sel is read on the device; blocks that would not fit view_cap_tokens are skipped and flagged.
 * An id outside the session (or a table entry outside the pool) is skipped as well: its view tokens are left
 * untouched and kvmem_device_status reports KVMEM_E_DEVICE_RANGE.  Tokens past n_sel * B are left untouched. */
int kvmem_materialize(kvmem_pool_t* pool, int32_t session_first, int32_t n_sessions, const int32_t* sel_ids /*DEVICE*/,
                      int32_t sel_stride, const int32_t* n_sel /*DEVICE*/, void* view_k /*DEVICE*/,
                      void* view_v /*DEVICE*/, int32_t view_cap_tokens, void* stream);

/* Incremental execution view (Eq. "kvmem-working-set-delta", Sec. 4.4: only what changed between two consecutive
 * working sets moves).  view_k / view_v hold the view kvmem_materialize (or this call) built from prev_ids; afterwards
 * they hold the view of sel_ids, bit-identical to kvmem_materialize's.  A slot j whose block stays (prev_ids[s][j] ==
 * sel_ids[s][j], j < n_prev[s]) is neither read nor written; every other slot receives its block from the pages
 * through the block table.  (A retained block that changes its slot is fetched from the repository rather than
 * shifted inside the view: with the whole history in HBM both cost one read and one write, and fetching has no
 * ordering hazard.)  HBM traffic: 2 bytes per byte of the slots that change.
 *   prev_ids  DEVICE int32 [n_sessions][sel_stride], n_prev DEVICE int32 [n_sessions]: the selection the view holds
 *   stats     DEVICE int32 [n_sessions][3] or NULL: slots unchanged, retained blocks that moved, incoming blocks
 * Other arguments and errors as kvmem_materialize.  prev_ids and sel_ids must be different buffers. */
int kvmem_materialize_delta(kvmem_pool_t* pool, int32_t session_first, int32_t n_sessions, const int32_t* prev_ids /*DEVICE*/,
                            const int32_t* n_prev /*DEVICE*/, const int32_t* sel_ids /*DEVICE*/, int32_t sel_stride,
                            const int32_t* n_sel /*DEVICE*/, void* view_k /*DEVICE*/, void* view_v /*DEVICE*/,
                            int32_t view_cap_tokens, int32_t* stats /*DEVICE, may be NULL*/, void* stream);

/* GQA decode attention over the view (QW3 attention kernels, Sec. 5.1; decode over the fixed
 * working set, Sec. 5.2).  For every query token m, layer l and head h, over the first
 * T = n_sel[s] * B view tokens of KV head g(h), without mask:
 *     out = softmax(q . K^T * scale) V        lse = ln sum_t exp(q . k_t * scale)
 * lse lets the caller merge attention over the tokens it appends after the view.
 *   q        DEVICE bf16 [n_sessions][n_q_tokens][n_layers][n_q_heads][head_dim]
 *   out      DEVICE fp32 [n_sessions][n_q_tokens][n_layers][n_q_heads][head_dim]
 *   lse      DEVICE fp32 [n_sessions][n_q_tokens][n_layers][n_q_heads]
 *   scale    0 selects 1/sqrt(head_dim)
 *   workspace DEVICE, kvmem_attend_workspace_bytes(), 256-byte aligned
 * T = 0 gives out = 0 and lse = -inf.  n_q_tokens * (H/G) <= 64 query rows per KV head and call (e.g. 1 + 7 draft tokens
 * with 8 query heads per KV head): up to 16 rows the K/V stream bounds the pass, with 32 or 64 rows the same stream
 * is read once and the tensor-core work per byte doubles or quadruples (the position-consistent and FP8 variants
 * take 16 rows).  Any block size the pool accepts (the view is walked in 64-token tiles; a shorter last tile is
 * masked); head_dim 128.  The calls that read pages through the block table (kvmem_materialize_attend,
 * kvmem_paged_attend, kvmem_paged_attend_rope on raw keys, kvmem_view_cache_attend) take block sizes that divide
 * 64 tokens (a tile is then 64 / B selected blocks, the last one possibly partly filled) or are a multiple of it,
 * among them the paper's default of 32 tokens (Sec. 4.3), also on the in-block key layout (kvmem_paged_attend_rope
 * then rotates the query back once per block of a tile); kvmem_materialize_attend_rope on the in-block layout and the
 * FP8 repository are built for 64-token blocks.  Other shapes return KVMEM_E_UNSUPPORTED. */
int kvmem_view_attend(kvmem_pool_t* pool, int32_t n_sessions, const void* q /*DEVICE*/, int32_t n_q_tokens,
                      const void* view_k /*DEVICE*/, const void* view_v /*DEVICE*/, int32_t view_cap_tokens,
                      const int32_t* n_sel /*DEVICE*/, float scale, float* out /*DEVICE*/, float* lse /*DEVICE*/,
                      void* workspace /*DEVICE*/, size_t workspace_bytes, void* stream);

/* kvmem_materialize followed by kvmem_view_attend as ONE pass over the selected blocks (Sec. 4.4 execution
 * view + Sec. 5.2 decode over it): each selected K/V tile is read once from the page pool through the
 * block table, written to its place in the view, and attended over while it sits in shared memory.
 * Same arguments, results, limits and error behaviour as the two separate calls; the view it leaves
 * behind is bit-identical to kvmem_materialize's, and out/lse are those of kvmem_view_attend on it.
 * HBM traffic per view byte drops from 2 reads + 1 write to 1 read + 1 write.  (The one difference: an id outside
 * the session cannot be skipped by a pass that also attends, so page 0 stands in for it, in the view and in out/lse,
 * and KVMEM_E_DEVICE_RANGE is reported; the results of such a call are to be discarded.) */
int kvmem_materialize_attend(kvmem_pool_t* pool, int32_t session_first, int32_t n_sessions, const void* q /*DEVICE*/,
                             int32_t n_q_tokens, const int32_t* sel_ids /*DEVICE*/, int32_t sel_stride,
                             const int32_t* n_sel /*DEVICE*/, void* view_k /*DEVICE*/, void* view_v /*DEVICE*/,
                             int32_t view_cap_tokens, float scale, float* out /*DEVICE*/, float* lse /*DEVICE*/,
                             void* workspace /*DEVICE*/, size_t workspace_bytes, void* stream);

/* Copy-free execution view (Sec. 4.4: the view as a page table over non-contiguous physical pages;
 * Sec. 5.3 "Copy-free execution-view assembly"): GQA decode attention straight over the selected
 * blocks' pages, in the order of sel_ids, through the block table.  No contiguous view is written.
 * out and lse equal kvmem_view_attend's on the view kvmem_materialize would build from the same ids
 * (same tiles, same order, same arithmetic).  HBM traffic: one read per view byte.
 * Arguments as in kvmem_materialize_attend, without the view buffers. */
int kvmem_paged_attend(kvmem_pool_t* pool, int32_t session_first, int32_t n_sessions, const void* q /*DEVICE*/,
                       int32_t n_q_tokens, const int32_t* sel_ids /*DEVICE*/, int32_t sel_stride,
                       const int32_t* n_sel /*DEVICE*/, float scale, float* out /*DEVICE*/, float* lse /*DEVICE*/,
                       void* workspace /*DEVICE*/, size_t workspace_bytes, void* stream);

/* Copy-free execution view with position-consistent keys (Sec. 4.4: the view is a page table over the
 * physical pages, and RoPE is applied to raw K at the block's assigned compact position): as
 * kvmem_paged_attend, but the warps that attend over a tile rotate their key fragments, between the tile's
 * arrival from the pages and their use, to compact position first_position + j*block_tokens + t (j = index in
 * sel_ids).  The angle of a position p1 + b (p1 the first of a warp's 16 positions, b < 16) is composed from the
 * table rows of p1 and of b: cos and sin within a few fp32 units in the last place of the table's own row, so a
 * rotated key is within one bf16 rounding step of kvmem_rope_rotate's, and out and lse are those of
 * kvmem_view_attend on the view kvmem_materialize_rope would build from the same ids within the attention
 * tolerance (not bit for bit); they equal kvmem_materialize_attend_rope's on a raw-key pool bit for bit.  Nothing is
 * written besides out and lse.  The pool's pages must hold raw keys and q must carry RoPE at its own position.
 * HBM traffic: one read per view byte (the rotary rows are 2 KiB per 64-token tile).
 * On a pool created with rope_in_block_keys (pages hold k' = RoPE(k, t)) no key is rotated: the logit
 * q . R(p0 + t) k equals (R(-p0) q) . k', p0 = first_position + j*block_tokens, so the 16 query rows are rotated
 * back by p0 once per block (arithmetic of kvmem_rope_rotate, inverse; the rotated query is a bf16 vector)
 * and the stored keys feed the tensor cores as they are.  The result is the same mathematics as attention
 * over kvmem_materialize_rope's view, one rounding of the query instead of one of each key apart.
 * Extra errors: KVMEM_E_STATE without a rotary table; KVMEM_E_INVALID if
 * [first_position, first_position + sel_stride*block_tokens) leaves the table. */
int kvmem_paged_attend_rope(kvmem_pool_t* pool, int32_t session_first, int32_t n_sessions, const void* q /*DEVICE*/,
                            int32_t n_q_tokens, const int32_t* sel_ids /*DEVICE*/, int32_t sel_stride,
                            const int32_t* n_sel /*DEVICE*/, int32_t first_position, float scale, float* out /*DEVICE*/,
                            float* lse /*DEVICE*/, void* workspace /*DEVICE*/, size_t workspace_bytes, void* stream);

/* kvmem_materialize_rope followed by kvmem_view_attend in one call (Sec. 4.4: the execution view with keys
 * encoded at their compact positions, then decode over it).  Same arguments as kvmem_materialize_attend plus
 * first_position and a q that carries RoPE at its own position.  ONE pass, 1 read + 1 write per view byte.
 * On a pool with rope_in_block_keys each K tile is rotated by its block's compact position while it sits in shared
 * memory, then stored and attended over: the view left behind is kvmem_materialize_rope's and out/lse are
 * kvmem_view_attend's on it, bit for bit.
 * On a raw-key pool the warps that attend over a tile rotate its key fragments to their compact positions on the way
 * to the tensor cores and hand them back to the tile, which is then stored.  Their angles are composed from two
 * table rows as in kvmem_paged_attend_rope, so the view's VALUES are kvmem_materialize_rope's bit for bit and its KEYS
 * are within one bf16 rounding step of them (a small fraction of the elements differs at all); out/lse are the
 * attention over the view this call writes.  Callers that need the key bytes of kvmem_materialize_rope exactly use
 * that call and kvmem_view_attend.  (The view's last 64-token tile must lie inside the rotary table: first_position +
 * the view length rounded up to 64.)
 * Extra errors: KVMEM_E_STATE without a rotary table; KVMEM_E_INVALID if the compact positions leave it. */
int kvmem_materialize_attend_rope(kvmem_pool_t* pool, int32_t session_first, int32_t n_sessions, const void* q /*DEVICE*/,
                                  int32_t n_q_tokens, const int32_t* sel_ids /*DEVICE*/, int32_t sel_stride,
                                  const int32_t* n_sel /*DEVICE*/, void* view_k /*DEVICE*/, void* view_v /*DEVICE*/,
                                  int32_t view_cap_tokens, int32_t first_position, float scale, float* out /*DEVICE*/,
                                  float* lse /*DEVICE*/, void* workspace /*DEVICE*/, size_t workspace_bytes, void* stream);

/* Working-set delta between two consecutive steps (Eq. "kvmem-working-set-delta", Sec. 4.4):
 *     retained R = W_next n W_prev,   incoming L = W_next \ W_prev,   outgoing E = W_prev \ W_next.
 * prev_ids / next_ids are the ascending id lists kvmem_select wrote at the two steps, a block's slot is
 * its index in its list (compact position / block_tokens).  All DEVICE int32:
 *   prev_ids, next_ids [n_sessions][stride];  n_prev, n_next [n_sessions]
 *   retained [n_sessions][stride][3] = (id, slot in prev, slot in next)   ascending ids
 *   incoming [n_sessions][stride][2] = (id, slot in next);  outgoing [n_sessions][stride] = id
 *   counts   [n_sessions][3] = (|R|, |L|, |E|)
 * A retained block whose slot moved needs its resident keys re-rotated by (new - old) * block_tokens
 * positions (kvmem_rope_rotate); only incoming blocks have to be fetched. */
int kvmem_working_set_delta(kvmem_pool_t* pool, int32_t n_sessions, const int32_t* prev_ids /*DEVICE*/,
                            const int32_t* n_prev /*DEVICE*/, const int32_t* next_ids /*DEVICE*/,
                            const int32_t* n_next /*DEVICE*/, int32_t stride, int32_t* retained /*DEVICE*/,
                            int32_t* incoming /*DEVICE*/, int32_t* outgoing /*DEVICE*/, int32_t* counts /*DEVICE*/,
                            void* stream);

/* FP8 execution view (the paper's evaluation keeps the KV cache in FP8, Sec. 6.1): kvmem_materialize and
 * kvmem_view_attend for a view that stores one byte per element.
 * Element = E4M3 code (1 sign, 4 exponent, 3 mantissa bits, bias 7, no infinities, largest value 448) of
 * x * (1 / scale): one fp32 product, round to nearest with ties to even, saturated to +-448; one static scale
 * per tensor (k_scale for keys, v_scale for values), > 0.  (The paper states no scaling rule; static
 * per-tensor scales are how FP8 KV caches are commonly run.)
 *   view_k8   DEVICE uint8 [n_sessions][n_layers][n_kv_heads][view_cap_tokens][head_dim]
 *   view_v8t  DEVICE uint8 [n_sessions][n_layers][n_kv_heads][view_cap_tokens / 64][head_dim][64]: values are
 *             transposed inside every 64-token tile, so that attention reads both operands along the index it
 *             contracts over
 *   both 128-byte aligned; view_cap_tokens a multiple of 64; other arguments as in kvmem_materialize /
 *   kvmem_view_attend.  Built for head_dim 128 and 64-token blocks (KVMEM_E_UNSUPPORTED otherwise).
 * kvmem_materialize_fp8 reads the bf16 pages through the block table and writes the codes (2 bytes read + 1
 * byte written per element).  kvmem_view_attend_fp8 computes out = softmax(q . (k8 * k_scale)^T * scale)
 * (v8 * v_scale) and lse over the first n_sel[s] * 64 view tokens: half the bytes of the bf16 view; the codes
 * are widened to f16 (exactly) in registers and contracted on the tensor cores with fp32 accumulation. */
int kvmem_materialize_fp8(kvmem_pool_t* pool, int32_t session_first, int32_t n_sessions, const int32_t* sel_ids /*DEVICE*/,
                          int32_t sel_stride, const int32_t* n_sel /*DEVICE*/, void* view_k8 /*DEVICE*/,
                          void* view_v8t /*DEVICE*/, int32_t view_cap_tokens, float k_scale, float v_scale, void* stream);
int kvmem_view_attend_fp8(kvmem_pool_t* pool, int32_t n_sessions, const void* q /*DEVICE*/, int32_t n_q_tokens,
                          const void* view_k8 /*DEVICE*/, const void* view_v8t /*DEVICE*/, int32_t view_cap_tokens,
                          const int32_t* n_sel /*DEVICE*/, float scale, float k_scale, float v_scale, float* out /*DEVICE*/,
                          float* lse /*DEVICE*/, void* workspace /*DEVICE*/, size_t workspace_bytes, void* stream);

/* Position-consistent FP8 execution view (Sec. 4.4 + Sec. 6.1) from a pool of bf16 pages with a rotary table: as
 * kvmem_materialize_fp8, but the key of view token j*64 + t is first rotated to compact position first_position + j*64 + t
 * (arithmetic of kvmem_rope_rotate, one rounding to bf16; with rope_in_block_keys the stored key is rotated by
 * first_position + j*64) and then quantised: element = E4M3 code of RoPE(k, position)_bf16 / k_scale.  Values as in
 * kvmem_materialize_fp8.  kvmem_view_attend_fp8 then attends over it with a q that carries RoPE at its own position.
 * Extra errors: KVMEM_E_STATE without a rotary table or on an FP8 repository; KVMEM_E_INVALID if the compact positions
 * leave the table. */
int kvmem_materialize_fp8_rope(kvmem_pool_t* pool, int32_t session_first, int32_t n_sessions, const int32_t* sel_ids /*DEVICE*/,
                               int32_t sel_stride, const int32_t* n_sel /*DEVICE*/, void* view_k8 /*DEVICE*/,
                               void* view_v8t /*DEVICE*/, int32_t view_cap_tokens, int32_t first_position, float k_scale,
                               float v_scale, void* stream);

/* On a pool created with fp8_pages: kvmem_materialize_fp8 copies the selected blocks' 8 KiB tiles as they are (1 byte
 * read + 1 byte written per element; k_scale and v_scale must be the pool's, KVMEM_E_INVALID otherwise), and
 * kvmem_paged_attend_fp8 is the copy-free execution view over such a repository (Sec. 5.3): attention straight
 * over the selected pages through the block table, nothing written besides out and lse; results are those of
 * kvmem_view_attend_fp8 on the view kvmem_materialize_fp8 would build, with the pool's scales (same tiles, same
 * order, same arithmetic).  HBM traffic: one byte per element of the selected blocks.
 * Arguments as kvmem_paged_attend.  KVMEM_E_STATE on a pool with bf16 pages. */
int kvmem_paged_attend_fp8(kvmem_pool_t* pool, int32_t session_first, int32_t n_sessions, const void* q /*DEVICE*/,
                           int32_t n_q_tokens, const int32_t* sel_ids /*DEVICE*/, int32_t sel_stride,
                           const int32_t* n_sel /*DEVICE*/, float scale, float* out /*DEVICE*/, float* lse /*DEVICE*/,
                           void* workspace /*DEVICE*/, size_t workspace_bytes, void* stream);

/* kvmem_paged_attend_fp8 with position-consistent keys, for a pool with fp8_pages AND rope_in_block_keys (the
 * paper's three mechanisms together: FP8 KV cache, Sec. 6.1; keys encoded at their compact positions, Sec. 4.4;
 * copy-free view, Sec. 5.3).  The pages hold the codes of RoPE(k, t) / fp8_k_scale, t the offset inside the block;
 * codes cannot be re-encoded without a second quantisation, so no key is touched: the logit q . R(p0 + t) k equals
 * (R(-p0) q) . RoPE(k, t), and the 16 query rows are rotated back by the block's compact position p0 =
 * first_position + j*64 once per block (arithmetic of kvmem_rope_rotate, inverse; the rotated query is rounded to
 * bf16, then widened to f16 for the tensor cores).  q carries RoPE at its own position.
 * Extra errors: KVMEM_E_STATE unless the pool has both options; KVMEM_E_INVALID if the compact positions leave the
 * rotary table. */
int kvmem_paged_attend_fp8_rope(kvmem_pool_t* pool, int32_t session_first, int32_t n_sessions, const void* q /*DEVICE*/,
                                int32_t n_q_tokens, const int32_t* sel_ids /*DEVICE*/, int32_t sel_stride,
                                const int32_t* n_sel /*DEVICE*/, int32_t first_position, float scale, float* out /*DEVICE*/,
                                float* lse /*DEVICE*/, void* workspace /*DEVICE*/, size_t workspace_bytes, void* stream);

/* kvmem_materialize_fp8 followed by kvmem_view_attend_fp8 as ONE pass: every selected tile is read once from the pages,
 * stored to its place in the FP8 view and attended over while it sits in shared memory.  Over an FP8 repository that is
 * 1 byte read + 1 byte written per element; over a bf16 repository (64-token blocks) the tile is quantised on the way
 * (2 bytes read + 1 byte written per element; arithmetic of kvmem_materialize_fp8) with the pool's fp8_k_scale and
 * fp8_v_scale, 1 where the configuration leaves them at 0.  The view and out/lse are those of the two separate calls
 * with the same scales, bit for bit.  Arguments as kvmem_materialize_attend with the FP8 view buffers. */
int kvmem_materialize_attend_fp8(kvmem_pool_t* pool, int32_t session_first, int32_t n_sessions, const void* q /*DEVICE*/,
                                 int32_t n_q_tokens, const int32_t* sel_ids /*DEVICE*/, int32_t sel_stride,
                                 const int32_t* n_sel /*DEVICE*/, void* view_k8 /*DEVICE*/, void* view_v8t /*DEVICE*/,
                                 int32_t view_cap_tokens, float scale, float* out /*DEVICE*/, float* lse /*DEVICE*/,
                                 void* workspace /*DEVICE*/, size_t workspace_bytes, void* stream);

/* Execution cache: the execution view kept across steps, with working-set reuse and bounded delta
 * re-RoPE (Sec. 4.4: the two views; "Retrieval-Aware Hierarchical Reuse"; Eq. "kvmem-working-set-delta").
 *
 * The cache is cap_blocks slots ("active GPU pages") in caller-owned DEVICE memory of
 * kvmem_view_cache_bytes() bytes, 256-byte aligned, for ONE session.  A slot holds one block in the
 * pool's page format ([K|V][L][G][block_tokens][d] bf16): K encoded for the block's current compact
 * position, V unchanged.  The pool's pages must hold raw (position-independent) keys and the pool must
 * have a rotary table.  kvmem_view_cache_update moves the cache from the previous working set to
 * sel_ids (ascending, as kvmem_select writes them; *n_sel <= cap_blocks):
 *   - a block that is resident and selected again keeps its slot (no data moves); every other slot is
 *     reclaimed; incoming blocks, in ascending id order, take the free slots in ascending slot order,
 *     their K built from raw K with RoPE at compact position first_position + j*block_tokens + t (j =
 *     index in sel_ids), their V copied;
 *   - a retained block whose index j changed has its keys re-encoded: rotated in place by
 *     (j_new - j_old) * block_tokens positions while fewer than max_delta_ropes such rotations have been
 *     applied since its keys were last built from raw K, otherwise rebuilt from raw K (counter reset).
 *     max_delta_ropes = 0 rebuilds every moved block, i.e. the cache always equals
 *     kvmem_materialize_rope's view.
 * Rotation arithmetic as in kvmem_rope_rotate (fp32 products and sums, no fused multiply-add, one
 * rounding to bf16), so cache contents are reproducible bit for bit.
 * stats (DEVICE int32[4], may be NULL) = (retained and unmoved, delta re-RoPEd, rebuilt, incoming).
 * Records inside the cache, at the byte offsets kvmem_view_cache_layout writes to offsets[6] (HOST):
 *   [0] pages  [1] slot_block int32[cap] (-1 = empty)  [2] slot_pos int32[cap]  [3] slot_cnt int32[cap]
 *   [4] view_slots int32[cap]: slot of the j-th selected block (the view's page table)  [5] n_view int32.
 * kvmem_view_cache_attend: GQA decode attention over the cached view through view_slots (no compaction);
 * q [M][L][H][d] bf16, out/lse/workspace/scale as in kvmem_view_attend with n_sessions = 1.
 * Errors: KVMEM_E_STATE without a rotary table; KVMEM_E_INVALID for bad pointers, cap_blocks outside
 * [1, 32768] or positions outside the table; KVMEM_E_CAPACITY if cache_bytes is too small.  A selection
 * longer than cap_blocks or an id outside the session is clamped / skipped on the device and reported as
 * KVMEM_E_DEVICE_RANGE by kvmem_device_status.  Calls on one cache must be ordered (same stream). */
size_t kvmem_view_cache_bytes(const kvmem_pool_t* pool, int32_t cap_blocks);
int kvmem_view_cache_layout(const kvmem_pool_t* pool, int32_t cap_blocks, size_t* offsets /*HOST [6]*/);
int kvmem_view_cache_reset(kvmem_pool_t* pool, void* cache /*DEVICE*/, size_t cache_bytes, int32_t cap_blocks, void* stream);
int kvmem_view_cache_update(kvmem_pool_t* pool, int32_t session, const int32_t* sel_ids /*DEVICE*/,
                            const int32_t* n_sel /*DEVICE*/, void* cache /*DEVICE*/, size_t cache_bytes,
                            int32_t cap_blocks, int32_t max_delta_ropes, int32_t first_position,
                            int32_t* stats /*DEVICE, may be NULL*/, void* stream);
int kvmem_view_cache_attend(kvmem_pool_t* pool, const void* q /*DEVICE*/, int32_t n_q_tokens, void* cache /*DEVICE*/,
                            size_t cache_bytes, int32_t cap_blocks, float scale, float* out /*DEVICE*/,
                            float* lse /*DEVICE*/, void* workspace /*DEVICE*/, size_t workspace_bytes, void* stream);

/* kvmem_view_attend for callers that cannot allocate device memory.  (The paper has no counterpart.)
 * Who needs it: a serving process that gave all of HBM to its KV pool at start-up and runs with
 * its allocator frozen, a plug-in that only ever sees the buffers of one request, or a latency path
 * where a device-synchronising cudaMalloc is not acceptable.  Same arguments, definitions and
 * results as kvmem_view_attend, except that the split-K workspace is a fixed array inside the
 * library (about 4 MiB, held on every GPU that loads the library until the process exits).
 *   - Limit: n_sessions * n_layers * n_kv_heads <= 8 per call; more returns KVMEM_E_CAPACITY with
 *     a message, and nothing is enqueued.
 *   - The call allocates nothing: no cudaMalloc, cudaFree or allocating library routine.
 *   - The first call on a device looks up the array's device address (the pool's device must be
 *     the current device); make that first call before starting any stream capture.  The address
 *     is remembered for the life of the process: the device's primary context must not be reset
 *     (cudaDeviceReset) while the library is in use.
 *   - All calls in the process share the array and it keeps the previous call's contents.  Nothing
 *     in it needs clearing (every slot that is read is overwritten first), but two calls whose
 *     kernels overlap on the GPU (different streams, or different pools on one device) race on it:
 *     keep them on one stream or order them with events. */
int kvmem_view_attend_static(kvmem_pool_t* pool, int32_t n_sessions, const void* q /*DEVICE*/, int32_t n_q_tokens,
                             const void* view_k /*DEVICE*/, const void* view_v /*DEVICE*/, int32_t view_cap_tokens,
                             const int32_t* n_sel /*DEVICE*/, float scale, float* out /*DEVICE*/, float* lse /*DEVICE*/,
                             void* stream);

/* The whole recall step for callers whose query and results live in HOST memory: copies q to the
 * device, runs kvmem_select and kvmem_materialize_attend, copies out and lse back and waits for the
 * stream (synchronous).  Same definitions and limits as the individual calls.
 *   q_host     HOST bf16 [n_sessions][n_q_tokens][L][H][d]   (pinned memory makes the copies asynchronous)
 *   out_host   HOST fp32 [n_sessions][n_q_tokens][L][H][d];  lse_host HOST fp32 [n_sessions][n_q_tokens][L][H]
 *              (when both are pinned, device-mapped memory the last kernel of the step writes them directly
 *              and no copy is issued; otherwise they are copied from the staging buffer)
 *   staging    DEVICE, kvmem_step_staging_bytes(), 256-byte aligned: device copies of q, out, lse
 * sel_ids, n_sel, views and workspaces are DEVICE buffers as in the individual calls and hold the
 * step's selection and view afterwards. */
size_t kvmem_step_staging_bytes(const kvmem_pool_config_t* cfg /*HOST*/, int32_t n_sessions, int32_t n_q_tokens);
int kvmem_recall_step_host(kvmem_pool_t* pool, int32_t session_first, int32_t n_sessions, const void* q_host /*HOST*/,
                           int32_t n_q_tokens, const kvmem_select_params_t* params /*HOST*/, int32_t* sel_ids /*DEVICE*/,
                           int32_t sel_stride, int32_t* n_sel /*DEVICE*/, void* view_k /*DEVICE*/, void* view_v /*DEVICE*/,
                           int32_t view_cap_tokens, float scale, float* out_host /*HOST*/, float* lse_host /*HOST*/,
                           void* staging /*DEVICE*/, size_t staging_bytes, void* select_workspace /*DEVICE*/,
                           size_t select_workspace_bytes, void* attend_workspace /*DEVICE*/,
                           size_t attend_workspace_bytes, void* stream);

/* ---- decode over a view: drafted tokens, accumulated weights, eviction ---------------------------
 * What a serving loop does with an execution view between two recall steps (Sec. 4.1, Sec. 5.2: decode
 * extends the view at its tail; the multi-token prediction of Sec. 5.1 verifies several drafted tokens
 * at once): attention of drafted tokens over view and tail, the attention weight every view token has
 * gathered, and eviction of the tokens that gathered least.
 *
 * Tail: tokens newer than the view that do not fill a block yet, token-major like the input of
 * kvmem_append_blocks (whole blocks of it can be handed to that call as they are).  Session s holds
 * n_tokens[s] committed tokens in rows [0, n_tokens[s]), its drafted tokens in the n_q[s] rows behind them.
 * Rows behind those are not used, whatever they hold. */
typedef struct {
    const void* k;           /* DEVICE bf16 [n_sessions][cap_tokens][n_layers][n_kv_heads][head_dim], 16-byte aligned */
    const void* v;           /* the same for the values                                                                */
    int32_t cap_tokens;      /* at least n_q_tokens                                                                    */
    const int32_t* n_tokens; /* DEVICE int32 [n_sessions]; n_tokens[s] + n_q[s] must not exceed cap_tokens             */
} kvmem_tail_t;

/* Attention of a tree of drafted tokens over view and tail.  For every drafted token i < n_q[s] of session s, layer l
 * and head h, with T = min(n_sel[s] * block_tokens, view_cap_tokens):
 *     visible(i) = the T view tokens, the committed tail tokens, and each drafted token j < n_q[s] whose bit j is set in
 *                  mask[s][i]
 *     out = softmax over visible(i) of (q_i . k * scale), times v          lse = ln sum over visible(i) of exp(q_i . k * scale)
 * A token that sees nothing, or nothing but logits of -inf, gets out = 0 and lse = -inf.  A token that is not visible to i
 * does not reach i's result, whatever its key and value hold (infinities and NaN included).
 *   q        DEVICE bf16 [n_sessions][n_q_tokens][L][H][d], n_q_tokens in [1, 64]
 *   n_q      DEVICE int32 [n_sessions] drafted tokens of each session (clamped to [0, n_q_tokens]); NULL: n_q_tokens each.
 *            out and lse of the tokens behind n_q[s] are left as they were
 *   mask     DEVICE uint64 [n_sessions][n_q_tokens]: bit j of word i says whether drafted token i sees drafted token j (an
 *            ancestor in the tree, and itself); bits at n_q[s] and above count as clear.  NULL: a chain (token i sees
 *            0 .. i), which is also the form for a single token
 *   tail     HOST struct; NULL: no tail, the drafted tokens see the view alone (mask must be NULL)
 *   out      DEVICE bf16 [n_sessions][n_q_tokens][L][H][d]: the result is complete, nothing is left to merge, so it
 *            is rounded once to the type the next layer reads
 *   lse      DEVICE fp32 [n_sessions][n_q_tokens][L][H]
 *   scale    0 selects 1/sqrt(head_dim)
 *   workspace  DEVICE, kvmem_tree_workspace_bytes(), 256-byte aligned; contents undefined afterwards.  Calls that may overlap
 *            on the GPU (two streams, two captured graphs) need one each
 * kvmem_view_tree_attend reads a materialised view (any block size the pool accepts); kvmem_paged_tree_attend reads the
 * selected blocks' pages through the block table in the order of sel_ids (block sizes that divide 64 tokens or are a
 * multiple of it), as kvmem_paged_attend does, with its rule for ids out of range.  Its keys are the stored ones, as they lie, in one
 * softmax with the tail's: on a pool with rotary support these are raw keys without a position, so position-consistent decode
 * (queries and tail at the positions behind the view) materialises first (kvmem_materialize_rope, then kvmem_view_tree_attend); with
 * rope_in_block_keys, whose keys carry angles of their own, the paged form is refused.  Built for head_dim 128.  HBM traffic:
 * one read of the view up to 256 query rows (n_q_tokens * H/G) per KV head, one per 256 rows above.  The result does not
 * depend on timing: the same bits from run to run.
 * An n_tokens[s] outside [0, cap_tokens - n_q[s]] is clamped to it and reported as KVMEM_E_DEVICE_RANGE.
 * A call is limited to 65,536 query rows per KV head, and to fewer than 2^30 units over all sessions, layers and KV heads, counted
 * from the capacities: per KV head one unit for each 128 tokens of the view (or of sel_stride blocks) and of the tail, either rounded
 * up, and 3 more; with more than 128 query rows per KV head two for each 128 tokens and 8 more, for every 256 rows.
 * Errors: KVMEM_E_INVALID (pointers, sizes, n_q_tokens, tail too short), KVMEM_E_UNSUPPORTED (limits, head_dim, block size),
 * KVMEM_E_CAPACITY (workspace), KVMEM_E_STATE (paged form: an FP8 repository, in-block-rotated keys).  The workspace sizes here and below are 0, with
 * kvmem_last_error set, for what their calls refuse whatever else they are given. */
size_t kvmem_tree_workspace_bytes(const kvmem_pool_config_t* cfg /*HOST*/, int32_t n_sessions, int32_t n_q_tokens);
int kvmem_view_tree_attend(kvmem_pool_t* pool, int32_t n_sessions, const void* q /*DEVICE*/, int32_t n_q_tokens,
                           const int32_t* n_q /*DEVICE, may be NULL*/, const uint64_t* mask /*DEVICE, may be NULL*/,
                           const void* view_k /*DEVICE*/, const void* view_v /*DEVICE*/, int32_t view_cap_tokens,
                           const int32_t* n_sel /*DEVICE*/, const kvmem_tail_t* tail /*HOST, may be NULL*/, float scale,
                           void* out /*DEVICE*/, float* lse /*DEVICE*/, void* workspace /*DEVICE*/, size_t workspace_bytes,
                           void* stream);
int kvmem_paged_tree_attend(kvmem_pool_t* pool, int32_t session_first, int32_t n_sessions, const void* q /*DEVICE*/,
                            int32_t n_q_tokens, const int32_t* n_q /*DEVICE, may be NULL*/,
                            const uint64_t* mask /*DEVICE, may be NULL*/, const int32_t* sel_ids /*DEVICE*/, int32_t sel_stride,
                            const int32_t* n_sel /*DEVICE*/, const kvmem_tail_t* tail /*HOST, may be NULL*/, float scale,
                            void* out /*DEVICE*/, float* lse /*DEVICE*/, void* workspace /*DEVICE*/, size_t workspace_bytes,
                            void* stream);

/* kvmem_view_tree_attend for a chain (mask NULL) that also accumulates the attention weight of every view token:
 *     mass[s][l][g][t] = decay * mass[s][l][g][t] + sum over tokens i < n_q[s] and the heads h of KV head g of
 *                        exp(q_i . k_t * scale - lse[s][i][l][h])                     for t < T
 * (fp32 throughout, a fixed order of addition: the same bits from run to run).  Entries at T and above are left as they
 * were.  The weights are those of the whole softmax, tail included.  A query row whose lse is -inf adds nothing; one with a
 * logit of NaN makes the weights of its head's view tokens NaN.
 *   mass   DEVICE fp32 [n_sessions][L][G][view_cap_tokens]; decay finite and non-negative (1: plain sum)
 *   workspace  DEVICE, kvmem_mass_workspace_bytes(), 256-byte aligned
 * n_q_tokens * (H/G) <= 64 and view_cap_tokens <= 2^23 (KVMEM_E_UNSUPPORTED otherwise).  The workspace holds the logits of all
 * query rows: 4 bytes per row, KV head and token of the view's capacity.  Other arguments and errors as above. */
size_t kvmem_mass_workspace_bytes(const kvmem_pool_config_t* cfg /*HOST*/, int32_t n_sessions, int32_t n_q_tokens,
                                  int32_t view_cap_tokens);
int kvmem_view_attend_mass(kvmem_pool_t* pool, int32_t n_sessions, const void* q /*DEVICE*/, int32_t n_q_tokens,
                           const int32_t* n_q /*DEVICE, may be NULL*/, const void* view_k /*DEVICE*/,
                           const void* view_v /*DEVICE*/, int32_t view_cap_tokens, const int32_t* n_sel /*DEVICE*/,
                           const kvmem_tail_t* tail /*HOST, may be NULL*/, float scale, float* mass /*DEVICE*/, float decay,
                           void* out /*DEVICE*/, float* lse /*DEVICE*/, void* workspace /*DEVICE*/, size_t workspace_bytes,
                           void* stream);

/* Evict the tokens of a view that gathered the least attention weight: per session, layer and KV head, with
 * T = min(n_sel[s] * block_tokens, view_cap_tokens), C = keep_blocks * block_tokens and K = min(C, T), the tokens kept are
 * the first min(n_sink_tokens, K), the last min(n_recent_tokens, what is left of K), and of the others those with the
 * largest mass, equal weights to the lower token, until K are kept (every head keeps its own tokens).  They are moved in
 * ascending order to rows [0, K) of another view, their weights with them; n_sel_out[s] = min(keep_blocks, T /
 * block_tokens) is that view's length in blocks, so that kvmem_view_attend and the calls above read it as any other.
 * Rows behind K are left as they were.  Any fp32 weight is ordered by its value (a NaN counts as larger than every number).
 *   dst_k, dst_v  DEVICE bf16 [n_sessions][L][G][dst_cap_tokens][d], 128-byte aligned, dst_cap_tokens >= C; must not overlap the view
 *   dst_mass      DEVICE fp32 [n_sessions][L][G][dst_cap_tokens]; must not overlap mass
 *   kept          DEVICE int32 [n_sessions][L][G][C] receives the kept tokens' places in the old view, or NULL
 *   n_sel_out     DEVICE int32 [n_sessions]; may be n_sel itself
 *   workspace     DEVICE, kvmem_evict_workspace_bytes(), 256-byte aligned
 * A call is limited to 2^28 - 1 KV heads over all sessions and layers, and to 2^31 - 1 pieces of 64 kept tokens over them, counted
 * from min(C, view_cap_tokens).
 * Errors: KVMEM_E_INVALID, KVMEM_E_CAPACITY, KVMEM_E_UNSUPPORTED (these limits, head_dim other than 128). */
size_t kvmem_evict_workspace_bytes(const kvmem_pool_config_t* cfg /*HOST*/, int32_t n_sessions, int32_t keep_blocks);
int kvmem_view_evict(kvmem_pool_t* pool, int32_t n_sessions, const void* view_k /*DEVICE*/, const void* view_v /*DEVICE*/,
                     int32_t view_cap_tokens, const int32_t* n_sel /*DEVICE*/, const float* mass /*DEVICE*/,
                     int32_t keep_blocks, int32_t n_sink_tokens, int32_t n_recent_tokens, void* dst_k /*DEVICE*/,
                     void* dst_v /*DEVICE*/, int32_t dst_cap_tokens, float* dst_mass /*DEVICE*/,
                     int32_t* kept /*DEVICE, may be NULL*/, int32_t* n_sel_out /*DEVICE*/, void* workspace /*DEVICE*/,
                     size_t workspace_bytes, void* stream);

/* ---- new tokens: rotary forms, tail and pages, prompt chunks -------------------------------------
 * The way of new tokens into the loop (Sec. 4.1: the step begins with the prefill of the new tokens; Sec. 4.3: raw keys for
 * the index; Sec. 4.4: keys at their positions for the view; Sec. 5.2: the current query is prefilled over the new view;
 * Sec. 5.3 "Incremental Indexing").
 *
 * Rotary form of a model: which dims of a head are pairs, and how far a position turns each.  The pool itself rotates pairs
 * (i, i + d/2) by the rows of its table.  Any form is that one in another order of the dims: pair p of the model's goes to dims
 * p and d/2 + p, the n = head_dim - rotary_dim dims that pass go, in order, to rotary_dim/2 .. d/2 - 1 and d/2 + rotary_dim/2 .. d - 1,
 * and turn by 0.  That is the "pool's order" of a query or key; no product of a query with a key, and no Mean-K score,
 * depends on an order that both share.  Values have no order of their own.  kvmem_rope_apply and kvmem_append_tokens take
 * queries and keys in the model's order and give the pool's; every other call of this library takes and gives the pool's. */
#define KVMEM_ROPE_HALF 0        /* layout: pairs (i, i + rotary_dim/2) */
#define KVMEM_ROPE_INTERLEAVED 1 /*         pairs (2i, 2i + 1) */
#define KVMEM_ROPE_NONE 0        /* scaling: f_i = rope_theta^(-2i/rotary_dim) */
#define KVMEM_ROPE_LINEAR 1      /*          f_i / factor */
#define KVMEM_ROPE_BASE 2        /*          the same with base rope_theta * factor^(rotary_dim / (rotary_dim - 2)) */
#define KVMEM_ROPE_RAMP 3        /*          f_i/factor * x + f_i * (1 - x), x = (i - lo) / max(hi - lo, 0.001) kept in [0, 1],
                                             lo = max(floor(p(turns_fast)), 0), hi = min(ceil(p(turns_slow)), rotary_dim - 1),
                                             p(t) = rotary_dim ln(original_positions / (2 pi t)) / (2 ln rope_theta): the pair
                                             that makes t turns over the original window */
#define KVMEM_ROPE_BANDS 4       /*          the same with x = (turns_fast - t_i) / (turns_fast - turns_slow) kept in [0, 1],
                                             t_i = original_positions f_i / (2 pi): pair i's turns over the original window */
#define KVMEM_ORDER_MODEL 0
#define KVMEM_ORDER_POOL 1
typedef struct {
    int32_t layout;
    int32_t rotary_dim;       /* the first rotary_dim dims rotate, a multiple of 16; 0: the whole head */
    int32_t scaling;
    float factor;             /* >= 1; not used with KVMEM_ROPE_NONE */
    float original_positions; /* KVMEM_ROPE_RAMP, KVMEM_ROPE_BANDS: the window the unscaled frequencies were made for */
    float turns_fast;         /* 0 selects 32 (ramp) or 4 (bands) */
    float turns_slow;         /* 0 selects 1 */
} kvmem_rope_t;

/* The frequencies of a form (NULL: the pool's own) on a pool of this geometry, in radians per position and in the pool's
 * order: HOST double [head_dim / 2], 0 for the dims that pass.  Pure host.  KVMEM_E_STATE without rotary support,
 * KVMEM_E_INVALID, KVMEM_E_UNSUPPORTED (rotary_dim). */
int kvmem_rope_frequencies(const kvmem_pool_config_t* cfg /*HOST*/, const kvmem_rope_t* rope /*HOST, may be NULL*/,
                           double* frequencies /*HOST*/);

/* Make the pool one of a model with this rotary form (NULL: the pool's own again): its table is rebuilt on `stream` with these
 * frequencies (angles in 64 bits, cos and sin rounded once to fp32; with the pool's own frequencies the bits of its creation, computed on the host
 * as there and copied before the call returns, unless the table holds them already), so that every call that rotates uses them, and
 * kvmem_rope_apply and kvmem_append_tokens go from the model's order to the pool's.  Before any block is appended or reserved
 * (KVMEM_E_STATE otherwise): stored keys stay in the frame they were encoded in.  Work that reads the table must be ordered
 * behind this call (same stream, or an event). */
int kvmem_set_rope(kvmem_pool_t* pool, const kvmem_rope_t* rope /*HOST, may be NULL*/, void* stream);

/* Rotate n_rows x n_vec vectors of head_dim elements, any head_dim that takes rotary support: vector (r, u) of y is vector (r, u) of x
 * turned to positions[r], or back by it (inverse != 0; that is also the gradient of the forward rotation), its rotated dims
 * times amplitude.  Row r, vector u starts r * row_stride + u * vec_stride elements behind x or y (not negative, multiples of 8;
 * that of an axis of length 1 is not looked at; bases 16-byte aligned), so queries and keys can be read where a packed projection left them.  x_order, y_order say which order the
 * dims come and go in.  fp32 products, sums and the amplitude's product, each rounded to fp32, one rounding to bf16; dims that
 * pass are copied.
 *   positions  DEVICE int32 [n_rows]; rows with a position outside the table are left unwritten and flagged in the status word
 *   amplitude  0 selects 1.  (Where a form comes with a factor m on its cos and sin: m^2 on the queries and none on the keys
 *              gives the same logits, and is what fits keys that this library rotates.)
 * x and y may be the same vectors if the two orders are the same; any other overlap is refused (KVMEM_E_INVALID).  Extents are compared, first
 * element to last: y between the rows of x counts as overlap too. */
int kvmem_rope_apply(kvmem_pool_t* pool, const void* x /*DEVICE*/, int64_t x_row_stride, int64_t x_vec_stride, int32_t x_order,
                     void* y /*DEVICE*/, int64_t y_row_stride, int64_t y_vec_stride, int32_t y_order, int64_t n_rows, int32_t n_vec,
                     const int32_t* positions /*DEVICE*/, int32_t inverse, float amplitude, void* stream);

/* The same call with its arguments in one struct, for callers that pay for each argument (a foreign-function interface): the launch of
 * a few tokens takes 2.5 us of host time, sixteen converted arguments half of that again. */
typedef struct {
    kvmem_pool_t* pool;
    const void* x;            /* DEVICE */
    void* y;                  /* DEVICE */
    const int32_t* positions; /* DEVICE */
    void* stream;
    int64_t n_rows, x_row_stride, x_vec_stride, y_row_stride, y_vec_stride;
    int32_t n_vec, x_order, y_order, inverse;
    float amplitude;
} kvmem_rope_call_t;
int kvmem_rope_apply_call(const kvmem_rope_call_t* call /*HOST*/);

/* Pages for n_blocks blocks behind a session's last: taken from the pool now (phys_ids as in kvmem_append_blocks), filled by
 * kvmem_append_tokens, part of the session only once kvmem_commit_blocks makes them so (this call, that one and kvmem_set_rope are
 * refused as KVMEM_E_STATE on a stream that is being captured: they change what the host knows of the pool).  While a session has reserved blocks
 * kvmem_append_blocks refuses it; kvmem_session_reset gives them back.  Errors as kvmem_append_blocks; KVMEM_E_STATE on an FP8
 * repository or with rope_in_block_keys (their pages do not hold the raw keys that the index is made from). */
int kvmem_reserve_blocks(kvmem_pool_t* pool, int32_t session, int32_t n_blocks, const int32_t* phys_ids /*HOST, may be NULL*/,
                         void* stream);

/* Blocks a session has reserved and not committed, or a negative status. */
int32_t kvmem_session_reserved(const kvmem_pool_t* pool, int32_t session);

/* Rows of a batch as a projection leaves them: head h of layer l of token i of session s starts
 * s * session_stride + i * token_stride + l * layer_stride + h * head_stride elements behind data (strides: not negative, multiples of
 * 8; that of an axis of length 1 is not looked at). */
typedef struct {
    const void* data; /* DEVICE bf16, 16-byte aligned */
    int64_t session_stride, token_stride, layer_stride, head_stride;
} kvmem_rows_t;

/* Append new tokens: token i < n_new[s] of session s takes row c = tail->n_tokens[s] + i of the tail, the one behind its committed
 * and earlier new tokens, at position positions[s][i], or first_position + n_sel[s] * block_tokens + c without positions
 * (n_sel NULL: 0), i.e. behind a view that starts at first_position.
 *     q_out     [s][i] = the query turned to that position, times q_amplitude (its rotated dims; 0 selects 1)
 *     tail->k, v [s][c] = the key turned to it, the value
 *     page of block nblocks[s] + c / block_tokens, its token c mod block_tokens = the raw key, the value  (to_pages = 1; the block has to be
 *                 reserved: a row without a reserved page is flagged as KVMEM_E_DEVICE_RANGE, and its tail row written)
 * Queries and keys come in the model's order and leave in the pool's.  On a pool without rotary support nothing turns.
 * tail->n_tokens is read, not changed: the tokens are drafted ones for kvmem_view_tree_attend and kvmem_view_prefill_attend;
 * adding to it commits them, calling again replaces them.  Counts and lengths are read on the device, so a captured call appends
 * wherever the tail then ends.  to_pages goes with a tail whose row 0 is the token behind the session's last block.
 * A tail's keys stay at the positions that they were turned to.  The positions counted here from rows go on behind them only as long as
 * row 0 of the tail and the view in front of it are those of the calls before: see kvmem_commit_blocks for what to do when they are not.
 *   n_new     DEVICE int32 [n_sessions] (clamped to [0, n_new_tokens]); NULL: n_new_tokens each.  Rows behind are left as they were
 *   q         HOST struct, n_q_heads heads per layer; NULL (with q_out NULL): keys and values alone.  k, v: n_kv_heads heads
 *   positions DEVICE int32 [n_sessions][n_new_tokens], or NULL
 *   q_out     DEVICE bf16 [n_sessions][n_new_tokens][L][H][d]
 * A token whose position lies outside the table is left out as a whole and flagged.  An n_tokens[s] outside
 * [0, cap_tokens - n_new[s]] is clamped to it and flagged.  Results must not overlap the inputs or each other (KVMEM_E_INVALID; extents are
 * compared, first element to last).
 * KVMEM_E_UNSUPPORTED: head_dim not a multiple of 16, or 2^31 groups of 16 elements in one session's new tokens.  KVMEM_E_STATE: to_pages
 * on an FP8 repository or with rope_in_block_keys. */
int kvmem_append_tokens(kvmem_pool_t* pool, int32_t session_first, int32_t n_sessions, int32_t n_new_tokens,
                        const int32_t* n_new /*DEVICE, may be NULL*/, const kvmem_rows_t* q /*HOST, may be NULL*/,
                        const kvmem_rows_t* k /*HOST*/, const kvmem_rows_t* v /*HOST*/, const int32_t* positions /*DEVICE, may be NULL*/,
                        const int32_t* n_sel /*DEVICE, may be NULL*/, int32_t first_position, float q_amplitude,
                        const kvmem_tail_t* tail /*HOST*/, void* q_out /*DEVICE, may be NULL*/, int32_t to_pages, void* stream);

/* The same call with its arguments in one struct (see kvmem_rope_apply_call); q.data NULL: no queries. */
typedef struct {
    kvmem_pool_t* pool;
    const int32_t* n_new;     /* DEVICE, may be NULL */
    kvmem_rows_t q, k, v;
    const int32_t* positions; /* DEVICE, may be NULL */
    const int32_t* n_sel;     /* DEVICE, may be NULL */
    kvmem_tail_t tail;
    void* q_out;              /* DEVICE, may be NULL */
    void* stream;
    int32_t session_first, n_sessions, n_new_tokens, first_position, to_pages;
    float q_amplitude;
} kvmem_append_call_t;
int kvmem_append_tokens_call(const kvmem_append_call_t* call /*HOST*/);

/* Make the first n_blocks[s] reserved blocks of each session part of it: their Mean-K rows are computed from the raw keys in
 * their pages (the bits that kvmem_append_blocks gives for the same keys), the session's length is raised and, with a tail, the
 * rows behind them move to its front and n_tokens[s] drops by n_blocks[s] * block_tokens.  (n_tokens below that is flagged as
 * KVMEM_E_DEVICE_RANGE: a block was committed before its tokens were there.)
 * The rows that move keep their bits: row r then holds a key at the position of row r + n_blocks[s] * block_tokens.  Whatever changes
 * where the rows or the view in front of them begin (a commit; another view, i.e. every recall that changes n_sel or first_position) asks
 * for one of these before the next call that appends to the tail or attends over it; nothing on the device can tell that it is missing:
 *   - the view grows at its end by the committed blocks (n_sel[s] by n_blocks[s], first_position as it was): positions fit as they are;
 *   - the view stays as it was, the committed tokens out of sight until a recall: kvmem_append_tokens with first_position larger by
 *     n_blocks[s] * block_tokens (or with positions, where sessions differ), so that new tokens go on behind the tail's;
 *   - any other view: the tail's keys come to their new positions.  Either n_tokens[s] = 0 and the raw keys and values of the rows are
 *     appended again (one rounding, as at first), or the tail's keys are turned in place by the difference, kvmem_rope_apply from
 *     KVMEM_ORDER_POOL to KVMEM_ORDER_POOL, inverse where they go down (no raw keys needed, but one rounding to bf16 more each time).
 *   n_blocks  HOST int32 [n_sessions]; KVMEM_E_STATE if a session has fewer reserved
 *   tail      HOST struct, may be NULL; entry s is session session_first + s */
int kvmem_commit_blocks(kvmem_pool_t* pool, int32_t session_first, int32_t n_sessions, const int32_t* n_blocks /*HOST*/,
                        const kvmem_tail_t* tail /*HOST, may be NULL*/, void* stream);

/* Attention of a prompt chunk over view and tail: kvmem_view_tree_attend for a chain (token i sees the view, the committed tail
 * tokens and the chunk's tokens 0 .. i) of any length.  Same arguments (tail NULL: the view alone), definitions, guarantees and
 * error values, and the same bits from run to run.  Chunks of up to 64 tokens with few query rows (H/G n_q_tokens below 448, or
 * n_sessions L H n_q_tokens below 2,560, or H/G above 128) are that call, with its kernel, workspace and limits.
 * Others: 4 head_dim flops per query row and visible token on the tensor cores; at most 128 query heads may share a KV head;
 *   workspace  DEVICE, kvmem_prefill_workspace_bytes(), 256-byte aligned (about 160 MB whatever the call); calls that may overlap on
 *              the GPU need one each
 * A call is limited to 2^30 tiles, counted from the capacities: one for each 128 tokens of view and tail, either rounded up, and 4 more,
 * for every two row tiles of floor(128 / (H/G)) tokens of every KV head, layer and session (KVMEM_E_UNSUPPORTED). */
size_t kvmem_prefill_workspace_bytes(const kvmem_pool_config_t* cfg /*HOST*/, int32_t n_sessions, int32_t n_q_tokens);
int kvmem_view_prefill_attend(kvmem_pool_t* pool, int32_t n_sessions, const void* q /*DEVICE*/, int32_t n_q_tokens,
                              const int32_t* n_q /*DEVICE, may be NULL*/, const void* view_k /*DEVICE*/, const void* view_v /*DEVICE*/,
                              int32_t view_cap_tokens, const int32_t* n_sel /*DEVICE*/, const kvmem_tail_t* tail /*HOST, may be NULL*/,
                              float scale, void* out /*DEVICE*/, float* lse /*DEVICE*/, void* workspace /*DEVICE*/,
                              size_t workspace_bytes, void* stream);

/* ---- inspection ------------------------------------------------------------------------------ */

/* The pages of a bf16 repository: DEVICE bf16 [max_blocks][K | V][n_layers][n_kv_heads][block_tokens][head_dim] (of an FP8 one, the
 * codes as described at kvmem_pool_config_t).  The pointer aliases pool storage. */
int kvmem_get_pages(kvmem_pool_t* pool, const void** pages /*HOST, receives DEVICE ptr*/);

/* Mean-K index of a session: DEVICE bf16 [n_layers][n_kv_heads][max_blocks_per_session][head_dim]
 * (rows >= *n_blocks undefined).  The pointer aliases pool storage. */
int kvmem_get_index(kvmem_pool_t* pool, int32_t session, const void** index /*HOST, receives DEVICE ptr*/,
                    int32_t* n_blocks /*HOST*/);

/* Block table of a session: DEVICE int32 [max_blocks_per_session], logical id -> physical page. */
int kvmem_get_block_table(kvmem_pool_t* pool, int32_t session, const int32_t** table /*HOST, receives DEVICE ptr*/,
                          int32_t* n_blocks /*HOST*/);

/* Synchronise the stream and fetch (and clear) the sticky device status word: KVMEM_OK,
 * KVMEM_E_TIMEOUT or KVMEM_E_DEVICE_RANGE.  Returns KVMEM_OK if the read itself worked. */
int kvmem_device_status(kvmem_pool_t* pool, int32_t* status /*HOST*/, void* stream);

/* Self-test of the failure path every kernel of this library shares.  (The paper has no counterpart.)  All waits
 * inside the kernels (for a TMA copy, for another warp) are bounded: after a time limit the kernel records
 * KVMEM_E_TIMEOUT in the status word and returns, so that a lost copy cannot hang the GPU.  A healthy run never takes
 * that path; this call does: one warp waits limit_us microseconds (1 .. 100,000) for a barrier nobody arrives at, with
 * the same wait routine, then sets KVMEM_E_TIMEOUT and returns.  The kernel ends by itself and the context and the pool
 * stay usable; kvmem_device_status then reports (and clears) KVMEM_E_TIMEOUT.
 *   waited_ns  DEVICE uint64, may be NULL: receives the time the wait lasted, in nanoseconds */
int kvmem_selftest_wait_timeout(kvmem_pool_t* pool, uint32_t limit_us, uint64_t* waited_ns /*DEVICE*/, void* stream);

/* The same for the wait of the tree attention's MMA thread, which asks up to three barriers together: barrier unmet (0 .. 2) of
 * the three is never arrived at, the other two are complete.  Arguments, status and effects as above.  (No counterpart.) */
int kvmem_selftest_joint_wait_timeout(kvmem_pool_t* pool, int32_t unmet, uint32_t limit_us, uint64_t* waited_ns /*DEVICE*/,
                                      void* stream);

/* Process-wide implementation switches used to compare kernel variants; "gather_mode" and "score_mode"
 * never change results, "chunk_poly" moves scores by a few 1e-6 relative.  (No counterpart in the paper.)  "gather_mode": 1 = bulk asynchronous copies through shared memory
 * (default), 0 = 128-bit load/store copy.  "score_mode" (decode-sized queries): 1 = dot products on the
 * tensor cores (default), 0 = fp32 ALU kernel that reduces the query rows with warp shuffles.
 * "chunk_poly" (multi-token chunks): n in 2..5 = every n-th exponential of the two softmax passes is a
 * degree-4 polynomial on the FMA pipe instead of a special-function-unit instruction (default 4), 0 = none.
 * "topk_cluster" (sessions above 16,384 blocks): 1 = selection by a thread-block cluster of 8 CTAs that merge
 * their histograms through distributed shared memory (default), 0 = by one CTA that re-reads the scores per pass.
 * "topk_items" (sessions of at most 16,384 blocks): 0 = the selection kernel holds the fewest scores per thread
 * (1, 2, 4, 8 or 16) that cover the session (default), n = at least n; never changes a result.
 * "attend_splits" (0 = chosen by the library, else forced split-K count), "attend_lookahead" (0 = chosen by the
 * library, else tiles the attention producers may run ahead), "gather_ctas" (0 = chosen by the library, else the
 * number of copy CTAs), "attend_landed" (-1 = chosen by the library, 1 / 0 = the lookahead counts tiles that have not
 * landed in shared memory yet / that have not been consumed yet): the knobs of the bytes-in-flight sweeps; only
 * "attend_splits" can move a result, by the rounding of a different split-K merge order.
 * "pdl": 1 = the kernels of a step are launched with programmatic stream serialization, so that the
 * launch latency of each overlaps the tail of the one before (default), 0 = plain launches.
 * The switches are process-wide (every pool, every thread) and atomic: a call that runs while another thread changes a
 * switch sees either value. */
int kvmem_set_option(const char* name /*HOST*/, int32_t value);

#ifdef __cplusplus
}
#endif
#endif /* KVMEM_H_ */
