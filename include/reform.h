/*
 * reform.h -- C ABI of the MI355X (gfx950) REFORM compress-and-gather hot path.
 *
 * Three calls, named after the steps of the method (arXiv 2506.01215):
 *
 *   reform_chunk_attend_score   Alg. 1 `layer.Forward(hs, cache)`, attention part: one chunk of
 *                               queries attends causally over [compressed KV cache || chunk KV]
 *                               (Sec. 3.1, Fig. 1 step 1) and, in the same call, produces the
 *                               eviction score of every key (Sec. 3.1 compresses the cache by
 *                               evicting on attention weights, as H2O does; Sec. 5 names fusing
 *                               this score into the attention kernel as the open efficiency item).
 *   reform_evict_topk_compact   Alg. 1 `Compress(cache)`: keep the heavy hitters up to the budget
 *                               and re-pack the cache so retained tokens are consecutive
 *                               (Sec. 3.1, Sec. 1, Sec. 4 common setup).
 *   reform_gather_topk          Alg. 1 `GatherRelevant(input, emb)`: cosine similarity between
 *                               query embeddings and every context embedding, highest scores
 *                               selected, neighbourhood kept contiguous (Sec. 3.3, App. C.6).
 *
 * Around them stand the calls that a model's serving needs next to these: rotary positions
 * (reform_rotary_embed), whole prompts packed into one batch (reform_prompt_attend, with a sliding window
 * reform_window_attend), and generation from a batch of caches, by single tokens or by trees of drafted ones
 * (reform_tree_attend, reform_tree_accept), or from caches in pages (reform_paged_attend, reform_paged_evict).
 *
 * Conventions common to all calls
 *   - Every data pointer is a DEVICE pointer (HIP global memory) owned by the caller.  The
 *     library never allocates, frees or keeps a pointer; scratch comes in through `workspace`,
 *     whose size the matching *_workspace() query returns (bytes; 256-byte aligned base needed).
 *   - Descriptors are HOST structs; `struct_size` must be sizeof() of the struct.
 *   - Work is enqueued on `hip_stream` (a hipStream_t cast to void*; NULL = the default stream)
 *     and the call returns without synchronising.
 *   - Arguments are validated on the host before anything is launched.  On any status other
 *     than REFORM_OK nothing was launched and the outputs are unchanged, except
 *     REFORM_ERR_RUNTIME (a HIP launch failed part-way): outputs are then undefined.
 *   - No C++ type, exception or torch object crosses this boundary.
 *   - Calls on different streams may overlap if their buffers (workspace included) are disjoint.
 *   - bf16 storage is the upper 16 bits of an IEEE fp32; conversions round to nearest even.
 */
#ifndef REFORM_H
#define REFORM_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef enum {
    REFORM_OK = 0,
    REFORM_ERR_INVALID_ARG = 1,   /* null pointer, bad shape, wrong struct_size, ...          */
    REFORM_ERR_UNSUPPORTED = 2,   /* well-formed but outside what the kernels implement       */
    REFORM_ERR_WORKSPACE = 3,     /* workspace missing, misaligned or too small               */
    REFORM_ERR_RUNTIME = 4        /* a HIP call failed                                         */
} reform_status;

typedef enum { REFORM_F32 = 0, REFORM_BF16 = 1 } reform_dtype;

/* ------------------------------------------------------------------------------------------- */
/* reform_chunk_attend_score
 *
 * For query head h (KV head g = h / G, G = n_q_heads / n_kv_heads) and chunk row i:
 *     s_ij   = scale * <q_hi, k_gj>,  j in [0, cache_len + i]     (cache rows all visible, chunk
 *                                                                 rows causal, diagonal included)
 *     p_ij   = softmax_j(s_ij)
 *     out_hi = sum_j p_ij v_gj
 *     lse_hi = log sum_j exp(s_ij)
 *     score_gj (+)= sum_{h in group g} sum_{i >= chunk_len - W} p_ij      (attention mass key j
 *                 received from the last W = obs_window rows; Sec. 4 setup mentions W = 128 for
 *                 the H2O baseline, the chunk's whole length is the default)
 *
 * Layouts (element = dtype):
 *     q      [n_q_heads][chunk_len][head_dim]   head stride / row stride given in elements,
 *                                               head_dim contiguous, 16-byte aligned rows
 *     k, v   [n_kv_heads][capacity][head_dim]   contiguous; rows [0,cache_len) = retained cache,
 *                                               rows [cache_len, cache_len+chunk_len) = this
 *                                               chunk (the caller writes them there); rows
 *                                               beyond are never read
 *     out    like q, with its own strides, dtype as the inputs
 *     lse    [n_q_heads][chunk_len] fp32, may be NULL
 *     score  [n_kv_heads][capacity] fp32, entries [0, cache_len+chunk_len) written (added to when
 *            accumulate != 0), the rest untouched; may be NULL (attention only)
 * Arithmetic: products and sums in fp32; for bf16 the probabilities fed to the P.V product are
 * rounded to bf16, the score sums the unrounded fp32 probabilities.  Results are bitwise
 * reproducible run to run (no floating-point atomics); two cache rows holding bit-identical
 * keys receive bit-identical scores.
 * Supported: REFORM_BF16 with head_dim 64 or 128; REFORM_F32 with head_dim % 4 == 0, <= 256.
 */
typedef struct {
    uint32_t struct_size;
    int32_t  dtype;                          /* reform_dtype                                   */
    int32_t  n_q_heads, n_kv_heads, head_dim;
    int32_t  cache_len, chunk_len, capacity; /* M >= 0, C_t >= 1, capacity >= M + C_t          */
    int64_t  q_head_stride, q_row_stride;    /* elements                                       */
    int64_t  o_head_stride, o_row_stride;    /* elements                                       */
    float    scale;                          /* > 0, finite; 1/sqrt(head_dim) in the paper's models */
    int32_t  obs_window;                     /* W in [1, chunk_len]; 0 means chunk_len         */
    int32_t  accumulate;                     /* 0: score = ..., 1: score += ...                */
    int32_t  phases;                         /* 0 or 3: attention then score (the normal call);
                                                1: attention only (out, lse);
                                                2: score only, reading lse written by an earlier
                                                   phase-1 call with the same inputs (lets a
                                                   profiler bracket each kernel separately)       */
} reform_attn_desc;

/* The query returns room for the lse rows (used if the caller passes lse = NULL) and, for problems
 * whose keys or rows are shared out over more workgroups than there are row or key blocks, for
 * their partial results: up to 68 MB for the attention (bf16; fp32 a few MB), and for the score four
 * bytes per key of every KV head and slice, of which there are up to 32, more where a short pass is
 * cut into single heads as well (the two share it).  Only the lse rows are needed: with a workspace
 * that holds just these (n_q_heads * chunk_len floats, rounded up to 256 bytes), or with none if lse
 * is given, the call runs such problems in their unshared form, slower (one token over 16640 keys,
 * 32/8 heads: 17 times) and with sums in another order; with room for some of the partial results
 * (bf16) it makes as many parts as fit.  A caller that sized its workspace some other way than by
 * this query gets that without further notice.  Whether the score is asked for in the same call
 * (phases 0 or 3, score not NULL) or not can change the order of the sums too: out, lse and score
 * then agree to rounding (fp32 sums of the same terms), not bit for bit.                         */
size_t reform_chunk_attend_score_workspace(const reform_attn_desc *desc);

reform_status reform_chunk_attend_score(const reform_attn_desc *desc,
                                        const void *q, const void *k, const void *v,
                                        void *out, float *lse, float *score,
                                        void *workspace, size_t workspace_bytes,
                                        void *hip_stream);

/* ------------------------------------------------------------------------------------------- */
/* reform_evict_topk_compact
 *
 * Per KV head, among the n_valid = M + C_t candidate slots keep the `budget` slots with the
 * largest score (ties: the lowest slot index wins); the first n_sink and the last n_recent slots
 * are always kept and count inside the budget (Sec. 4 setup keeps the initial and recent 256
 * tokens).  Then row r of the cache becomes old row kept_idx[r] for r < new_len, in ascending
 * slot order, for k, v, score and pos alike -- in place.  new_len = min(n_valid, budget); it is
 * a function of the descriptor, nothing is read back.  If n_valid <= budget nothing moves.
 *
 *     k, v     [n_kv_heads][capacity][head_dim], in/out; rows >= new_len keep stale content
 *     score    [n_kv_heads][capacity] fp32, in/out; must be finite (no NaN/Inf)
 *     pos      [n_kv_heads][capacity] int32 token ids travelling with the rows, in/out, may be NULL
 *     kept_idx [n_kv_heads][budget] int32 out (first new_len entries per head), may be NULL
 * Supported: head_dim * sizeof(element) must be a multiple of 16; capacity <= 2^31 - 65536.
 * Device-side status: when rows move in place (row sizes that divide 16 KB), workgroups order
 * their reads and writes through flags with a bounded wait.  The wait cannot expire unless other
 * work keeps part of this call's workgroups off the device for seconds; if it does, the call
 * still ends, the cache content is then undefined, and the first int32 of the workspace, which
 * such a call clears when it starts, is set to 1.  A caller that wants to know reads that word
 * once the stream has finished (other row sizes clear it too and never set it).
 * Rows of more than 8192 candidates are selected by several workgroups per row that wait for each
 * other inside one launch, at most 128 in all, one on a compute unit.  The waiting workgroups of
 * all evictions, gathers (64 at most) and pooled gathers (128) that overlap on one GPU from
 * different streams share its 256 compute units.  If they do not fit, such a wait expires after
 * some seconds and the workgroup selects by itself: the results are the same, only late.
 */
typedef struct {
    uint32_t struct_size;
    int32_t  dtype;
    int32_t  n_kv_heads, head_dim;
    int32_t  n_valid, budget, capacity;
    int32_t  n_sink, n_recent;               /* n_sink + n_recent <= budget                    */
} reform_evict_desc;

size_t reform_evict_topk_compact_workspace(const reform_evict_desc *desc);

reform_status reform_evict_topk_compact(const reform_evict_desc *desc,
                                        void *k, void *v, float *score,
                                        int32_t *pos, int32_t *kept_idx,
                                        void *workspace, size_t workspace_bytes,
                                        void *hip_stream);

/* Testing aid for the bounded waits above.  Sets, for later calls in this process, how many times a
 * workgroup polls for another one before it gives up (default 2^22; a negative value restores the
 * default).  0: every wait expires on its first poll.  In the in-place move publishing is off as
 * well, so the status word is set whenever the kept set makes one tile depend on another, and the
 * cache content after such a call is undefined; a selection stays exact.  Every kernel still runs
 * to its end.                                                                                   */
void reform_debug_set_move_spin_limit(int32_t polls);

/* reform_evict_topk_compact_static -- the same operation for callers that cannot allocate device
 * memory or carry a workspace: code running under HIP graph capture, tight serving loops,
 * harnesses that forbid hipMalloc.  It takes no workspace: the selection state, the staging rows
 * and the ordering flags live in a static device array of REFORM_STATIC_SCRATCH_BYTES that each
 * GPU the library runs on holds until the process ends.  Arguments, layouts, results and status
 * codes are those of reform_evict_topk_compact; the call allocates and frees nothing.
 *   - The device the work is meant for must be the current HIP device (the array's address on
 *     that device is looked up on the first call there).
 *   - A descriptor whose reform_evict_topk_compact_workspace() exceeds
 *     REFORM_STATIC_SCRATCH_BYTES is rejected with REFORM_ERR_WORKSPACE before any launch
 *     (8 KV heads x 65536 candidates -> 32768 of 256-byte rows needs about 5.3 MB).
 *   - Every call on a GPU shares that GPU's array, which still holds the previous call's
 *     contents; the call clears what it needs cleared itself.  Two such calls that overlap in
 *     time on one GPU (different streams or threads) race: serialise them.
 *   - The device-side status word described above is the first int32 of that array and is not
 *     reachable by the caller; use the workspace form to observe it.
 */
#define REFORM_STATIC_SCRATCH_BYTES (8u << 20)

reform_status reform_evict_topk_compact_static(const reform_evict_desc *desc,
                                               void *k, void *v, float *score,
                                               int32_t *pos, int32_t *kept_idx,
                                               void *hip_stream);

/* ------------------------------------------------------------------------------------------- */
/* reform_gather_topk
 *
 *     sim_qt   = <e_t, u_q> / max(|e_t| |u_q|, eps)              (Sec. 3.3, App. C.6)
 *     topk_q   = the k indices t with the largest sim_qt, ties to the lowest t, ascending
 *     union    = sorted unique { t + dlt : t in any topk_q, |dlt| <= radius, 0 <= t+dlt < n_ctx }
 *                united with the first n_head_keep and last n_tail_keep rows (Sec. 3.3 keeps
 *                the first and last tokens and widens hits to their neighbourhood)
 *
 *     emb         [n_ctx][dim], contiguous, dtype
 *     qry         [n_query][dim], contiguous, dtype
 *     topk_idx    [n_query][k] int32 out
 *     topk_score  [n_query][k] fp32 out (sim of the selected rows), may be NULL
 *     union_idx   [n_ctx] int32 out (first union_count entries), may be NULL (then no union)
 *     union_count one int32 in device memory, out, required iff union_idx != NULL
 * Supported: n_ctx <= 2^31 - 65536; dim % 8 == 0; any n_query >= 1 (up to 64 per pass over emb).
 * Rows of more than 8192 similarities are selected, where at most 64 workgroups suffice for all of
 * them, by several workgroups per row that wait for each other inside one launch (see
 * reform_evict_topk_compact).  The first int32 of the workspace is cleared by the call and set to
 * 1 if such a wait expired; the outputs are exact all the same.
 */
typedef struct {
    uint32_t struct_size;
    int32_t  dtype;
    int64_t  n_ctx;
    int32_t  dim, n_query, k;                /* 1 <= k <= n_ctx                                */
    int32_t  radius, n_head_keep, n_tail_keep;
    float    eps;                            /* > 0; 1e-8 in the tests                         */
} reform_gather_desc;

size_t reform_gather_topk_workspace(const reform_gather_desc *desc);

reform_status reform_gather_topk(const reform_gather_desc *desc,
                                 const void *emb, const void *qry,
                                 int32_t *topk_idx, float *topk_score,
                                 int32_t *union_idx, int32_t *union_count,
                                 void *workspace, size_t workspace_bytes,
                                 void *hip_stream);

/* Intermediate of reform_gather_topk, exposed for checking: only the similarity matrix,
 * sim [n_query][n_ctx] fp32 (device, out).  Same descriptor, k/radius/keeps ignored.           */
reform_status reform_gather_similarity(const reform_gather_desc *desc,
                                       const void *emb, const void *qry, float *sim,
                                       void *hip_stream);

/* ------------------------------------------------------------------------------------------- */
/* reform_gather_pooled -- the selection of Sec. 3.3 in the paper's own order
 *
 *     sim_qt   = cosine similarity as in reform_gather_topk                (Sec. 3.3, App. C.6)
 *     s_t      = max_q sim_qt                       (max-pool over the query tokens, Sec. 3.3)
 *     pooled_t = max { s_u : |u - t| <= (pool_window-1)/2, 0 <= u < n_ctx }
 *                (each token's score max-pooled with its adjacent tokens; the paper uses 128
 *                 neighbours = a window of 129, Sec. 4.5; the window is clipped at both ends)
 *     sel      = the `budget` tokens with the largest pooled_t, the first n_head_keep and the
 *                last n_tail_keep tokens always among them and counted inside the budget
 *                (Sec. 3.3 keeps the initial and final 256 tokens; Sec. 4 gives budgets of 8k and
 *                 16k), ties to the lowest index, ascending
 *
 *     emb      [n_ctx][dim], qry [n_query][dim]: contiguous, dtype
 *     sel_idx  [budget] int32 out
 *     pooled   [n_ctx] fp32 out, may be NULL (then it lives in the workspace only)
 * Supported: as reform_gather_topk; pool_window odd, 1 <= pool_window <= 1025;
 * n_head_keep + n_tail_keep <= budget <= n_ctx.
 * The one row of pooled scores is selected, when it has more than 8192 entries and at most 4
 * million, by up to 128 workgroups that wait for each other inside one launch (see
 * reform_evict_topk_compact).  The first int32 of the workspace is cleared by the call and set to
 * 1 if such a wait expired; the outputs are exact all the same.
 */
typedef struct {
    uint32_t struct_size;
    int32_t  dtype;
    int64_t  n_ctx;
    int32_t  dim, n_query, budget;
    int32_t  pool_window, n_head_keep, n_tail_keep;
    float    eps;
} reform_pooled_desc;

size_t reform_gather_pooled_workspace(const reform_pooled_desc *desc);

reform_status reform_gather_pooled(const reform_pooled_desc *desc,
                                   const void *emb, const void *qry,
                                   int32_t *sel_idx, float *pooled,
                                   void *workspace, size_t workspace_bytes,
                                   void *hip_stream);

/* ------------------------------------------------------------------------------------------- */
/* reform_embed_save_selected -- Alg. 1 `emb.SaveSelected(qkv)`, the selected heads of one tensor
 *
 *     emb[t][col + c] = x_t[c] / max(||x_t||, eps),  c in [0, head_dim)       (Sec. 3.2, the
 *     e_comb equation: the context embedding of a token is the concatenation of the
 *     L2-normalised Q/K/V states of the selected heads; one call writes n_heads adjacent
 *     segments for the n_rows tokens of a chunk: head h is read src_head_stride elements after
 *     head h-1 and written to columns [emb_col + h*head_dim, emb_col + (h+1)*head_dim))
 *
 *     src   the first selected head's state of the chunk's first token; token t's vector starts
 *           src_row_stride elements further on for each t (so a [heads][rows][d] or a
 *           [rows][heads][d] tensor can be addressed in place); dtype
 *     emb   embedding row of the chunk's first token in the [n_ctx][emb_dim] store
 *           (emb_row_stride = emb_dim elements); dtype; only columns
 *           [emb_col, emb_col + n_heads*head_dim) of the n_rows rows are written; with
 *           n_rows = 0 nothing is read or written and both pointers may be NULL
 * Supported: head_dim * sizeof(dtype) a multiple of 16 and at most 1024 bytes; strides and
 * emb_col multiples of 16 bytes; src and emb 16-byte aligned; 1 <= n_heads <= 65535.  Sums in
 * fp32.
 */
typedef struct {
    uint32_t struct_size;
    int32_t  dtype;
    int64_t  n_rows;
    int32_t  head_dim;
    int32_t  emb_col;
    int64_t  src_row_stride, emb_row_stride; /* in elements                                    */
    float    eps;                            /* > 0; 1e-12 in the tests                        */
    int32_t  n_heads;                        /* heads written by this call (adjacent columns)  */
    int64_t  src_head_stride;                /* in elements; ignored when n_heads == 1         */
} reform_embed_desc;

reform_status reform_embed_save_selected(const reform_embed_desc *desc,
                                         const void *src, void *emb, void *hip_stream);

/* ------------------------------------------------------------------------------------------- */
/* reform_rerotate_keys -- consecutive position ids after compression (Sec. 3.1)
 *
 * For a cache that stores rotary-embedded keys: after reform_evict_topk_compact the key at slot
 * r came from slot kept_idx[r] and is rotated by delta = r - kept_idx[r] positions, in place:
 *     a           = delta * theta^(-2c/rotary_dim),              c in [0, rotary_dim/2)
 *     k'[c]       = k[c] cos a - k[c + rotary_dim/2] sin a
 *     k'[c+rd/2]  = k[c + rotary_dim/2] cos a + k[c] sin a       (half-split pairing, as in the
 *                                                               models the paper evaluates)
 * Elements [rotary_dim, head_dim) and rows with delta = 0 are not touched; V is not rotated.
 *
 *     k         [n_kv_heads][capacity][head_dim], dtype, rows [0, n_rows) rotated in place
 *     kept_idx  [n_kv_heads][budget] int32 as written by reform_evict_topk_compact
 * Angles are formed in fp64 and reduced to a fraction of a turn before the fp32 sine/cosine.
 * Supported: rotary_dim even, rotary_dim/2 * sizeof(dtype) a multiple of 16; 0 <= n_rows <=
 * min(budget, capacity).
 */
typedef struct {
    uint32_t struct_size;
    int32_t  dtype;
    int32_t  n_kv_heads, head_dim, capacity;
    int32_t  n_rows, budget;
    int32_t  rotary_dim;                     /* <= head_dim                                    */
    float    theta;                          /* rotary base, > 1 (10000, 1e6, ...)             */
} reform_rope_desc;

reform_status reform_rerotate_keys(const reform_rope_desc *desc, void *k, const int32_t *kept_idx,
                                   void *hip_stream);

/* ------------------------------------------------------------------------------------------- */
/* reform_gather_rows -- the inputs that are recomputed (Sec. 3.3 "On-Demand Cache
 * Recomputation"; Alg. 1: the selected tokens' input embeddings are gathered and forwarded again)
 *
 *     out[i] = table[idx[i]],   i in [0, n)   with n = n_idx, or min(*count, n_idx) if count != NULL
 *
 *     table  [n_table][row_bytes] bytes, any element type
 *     idx    [n_idx] int32 (the union_idx of reform_gather_topk or the sel_idx of
 *            reform_gather_pooled)
 *     count  one int32 in device memory or NULL (the union_count of reform_gather_topk, so the
 *            caller needs no host round trip)
 *     out    [n_idx][row_bytes] bytes; rows >= n are not written
 *     err    one int32 in device memory or NULL; bit 0 is set if an index was outside the
 *            table (that row is then skipped, never read); the caller clears it
 * Supported: row_bytes a multiple of 16, table and out 16-byte aligned.
 */
typedef struct {
    uint32_t struct_size;
    int32_t  reserved;                       /* 0                                              */
    int64_t  n_table, n_idx, row_bytes;
} reform_rows_desc;

reform_status reform_gather_rows(const reform_rows_desc *desc, const void *table,
                                 const int32_t *idx, const int32_t *count, void *out,
                                 int32_t *err, void *hip_stream);

/* ------------------------------------------------------------------------------------------- */
/* reform_rotary_embed -- queries and keys to their positions, keys and values into the caches
 *
 * For token i at position pos[i] and pair c in [0, rotary_dim/2) with frequency f_c:
 *     a       = pos[i] * f_c                     (inverse = 1: -pos[i] * f_c)
 *     y[x]    = magnitude * (x cos a - x' sin a)     of every query and key head, where (x, x') are the
 *     y[x']   = magnitude * (x' cos a + x sin a)     elements of the pair: c and c + rotary_dim/2
 *               (REFORM_PAIRS_HALVES) or 2c and 2c + 1 (REFORM_PAIRS_ADJACENT)
 * Elements [rotary_dim, head_dim) and values are copied.  inverse = 1 is the transposed map: with the
 * same magnitude it takes the gradient of the rotated states to that of the unrotated ones; with
 * 1 / magnitude it takes the rotation back.
 *     f_c = theta^(-2c/rotary_dim)                                          REFORM_ROPE_PLAIN
 *         = theta^(-2c/rotary_dim) / factor                                 REFORM_ROPE_LINEAR
 *         = theta'^(-2c/rotary_dim), theta' = theta * factor^(rotary_dim/(rotary_dim-2))  REFORM_ROPE_BASE
 *         = f (1 - r_c) + f / factor * r_c, f = theta^(-2c/rotary_dim):     REFORM_ROPE_PARTS: r_c rises from 0
 *               at pair floor(p(turns_high)) to 1 at pair ceil(p(turns_low)), both kept within [0, rotary_dim-1],
 *               p(t) = rotary_dim ln(original_len / (2 pi t)) / (2 ln theta): the pair that turns t times
 *               within original_len
 *                                                                           REFORM_ROPE_BANDS: r_c falls from 1
 *               at turns_low to 0 at turns_high turns within original_len, linearly in the turns
 * Frequencies and angles are formed in fp64 and reduced to a fraction of a turn before the fp32
 * sine and cosine; products and sums in fp32, rounded once.
 *
 *     q, q_out    [n_q_heads][n_tokens][head_dim] by strides; NULL iff n_q_heads = 0
 *     k, v        [n_kv_heads][n_tokens][head_dim] by strides; k NULL iff n_kv_heads = 0, v may be NULL
 *                 (no values); input strides of 0 (one head or row for all) are allowed
 *     k_out,v_out slot == NULL: as k, row i for token i, strides kv_out_*.  Otherwise caches in n_blocks
 *                 blocks of block_len rows, block_stride elements apart: token i goes to row
 *                 slot[i] % block_len of block slot[i] / block_len, head h kv_out_head_stride elements
 *                 behind head h-1; a token whose slot is outside [0, n_blocks*block_len) is not stored
 *                 (padding).  Slots should differ: of two tokens with one slot the row holds either or a
 *                 mixture.  v_out may be NULL iff v is.
 *     pos         [n_tokens] int32, any sign
 *     slot        [n_tokens] int32 or NULL
 * q_out may be q, and without slots k_out may be k and v_out v, with the same strides (then rotated in
 * place); other overlaps of outputs with inputs or each other are not allowed.
 * Supported: head_dim <= 512 and a multiple of 16 bytes; rotary_dim even, at most head_dim, a multiple of 16
 * bytes (REFORM_PAIRS_ADJACENT) or of 32 (REFORM_PAIRS_HALVES); strides multiples of 16 bytes, pointers
 * 16-byte aligned; n_tokens times the 16-byte pieces of a row below 2^31; n_tokens = 0 does nothing.
 */
typedef enum { REFORM_PAIRS_HALVES = 0, REFORM_PAIRS_ADJACENT = 1 } reform_rope_pairs;
typedef enum {
    REFORM_ROPE_PLAIN = 0, REFORM_ROPE_LINEAR = 1, REFORM_ROPE_BASE = 2, REFORM_ROPE_PARTS = 3, REFORM_ROPE_BANDS = 4
} reform_rope_scaling;

typedef struct {
    uint32_t struct_size;
    int32_t  dtype;
    int32_t  n_tokens, n_q_heads, n_kv_heads, head_dim;
    int32_t  rotary_dim;
    int32_t  pairs;                          /* reform_rope_pairs                              */
    int32_t  inverse;                        /* 0 or 1                                         */
    int32_t  scaling;                        /* reform_rope_scaling                            */
    double   theta;                          /* > 1, finite                                    */
    double   factor;                         /* >= 1, finite; not read for REFORM_ROPE_PLAIN   */
    double   turns_high, turns_low;          /* 0 < turns_low < turns_high, finite, and ...    */
    int32_t  original_len;                   /* ... >= 1: read for PARTS and BANDS only        */
    float    magnitude;                      /* > 0, finite; 1 unless the model asks for another */
    int32_t  block_len, n_blocks;            /* read iff slot != NULL; block_len*n_blocks < 2^31 */
    int64_t  block_stride;                   /* all strides in elements                        */
    int64_t  q_head_stride, q_row_stride, k_head_stride, k_row_stride, v_head_stride, v_row_stride;
    int64_t  q_out_head_stride, q_out_row_stride, kv_out_head_stride, kv_out_row_stride;
} reform_rotary_desc;

reform_status reform_rotary_embed(const reform_rotary_desc *desc, const void *q, const void *k, const void *v,
                                  const int32_t *pos, const int32_t *slot,
                                  void *q_out, void *k_out, void *v_out, void *hip_stream);

/* ------------------------------------------------------------------------------------------- */
/* reform_prompt_attend -- causal attention over whole prompts of different lengths, packed
 *
 * Sequence s has query rows [cu_q[s], cu_q[s+1]) and key rows [cu_k[s], cu_k[s+1]) of packed tensors;
 * its last query row sees all of its keys and each row before it one key less:
 *     s_ij   = scale * <q_hi, k_gj>,  j in [0, nk - nq + i],  nq and nk the sequence's rows, g = h / G
 *     out_hi = sum_j softmax_j(s_ij) v_gj,      lse_hi = log sum_j exp(s_ij)
 * (with nk = nq plain causal attention, with nk > nq a prompt behind nk - nq cached rows).  A row that
 * sees no key (nk < nq) gets out = 0 and lse = -inf.  Rows of q that belong to no sequence keep what out and
 * lse held.
 *     q, out   [n_q_heads][n_q_rows][head_dim], k, v [n_kv_heads][n_k_rows][head_dim]: by strides, elements
 *              of a row contiguous (token-major tensors are addressed in place)
 *     cu_q     [n_seq + 1] int32 in device memory, ascending, 0 <= cu_q[s] <= n_q_rows
 *     cu_k     the same for the keys, or NULL for cu_q
 *     lse      [n_q_heads][n_q_rows] fp32, may be NULL
 * The lengths are read on the device, so a captured call follows them.  Boundaries outside [0, n_q_rows]
 * or [0, n_k_rows] are moved into it and a descending pair counts as an empty sequence, so that nothing
 * outside the tensors is read or written; sequences must not overlap in q.  (Beyond 1024 sequences a cu_q that
 * descends anywhere leaves it open which of its rows are computed, still with nothing outside touched.)
 * Arithmetic as in reform_chunk_attend_score, bitwise reproducible.  Keys and values that are not finite stay
 * within their sequence; there, rows before such a value may become NaN as well as those that see it (its
 * weight 0 is multiplied with it).  The same holds in reform_tree_attend for the nodes of one sequence.
 * Supported: REFORM_BF16 with head_dim 64 or 128; REFORM_F32 with head_dim % 4 == 0, <= 256; at most 65536
 * sequences; out and lse apart from the inputs; n_q_heads * n_q_rows / 16 + n_kv_heads * n_seq below 2^23, n_kv_heads * n_k_rows below 2^30; row
 * strides of k and v below 2^24.  n_q_rows = 0 does nothing.
 * The workspace takes partial results where few rows stand behind many keys, which are then shared out over workgroups; the query
 * gives 0 elsewhere.  Without it, or with less than the query asks for, the call returns REFORM_ERR_WORKSPACE.
 */
typedef struct {
    uint32_t struct_size;
    int32_t  dtype;
    int32_t  n_q_heads, n_kv_heads, head_dim;
    int32_t  n_seq, n_q_rows, n_k_rows;
    float    scale;                          /* > 0, finite                                    */
    int32_t  reserved;                       /* 0                                              */
    int64_t  q_head_stride, q_row_stride, k_head_stride, k_row_stride;   /* elements, multiples */
    int64_t  v_head_stride, v_row_stride, o_head_stride, o_row_stride;   /* of 16 bytes         */
} reform_prompt_desc;

size_t reform_prompt_attend_workspace(const reform_prompt_desc *desc);

reform_status reform_prompt_attend(const reform_prompt_desc *desc, const void *q, const void *k, const void *v,
                                   const int32_t *cu_q, const int32_t *cu_k, void *out, float *lse,
                                   void *workspace, size_t workspace_bytes, void *hip_stream);

/* ------------------------------------------------------------------------------------------- */
/* reform_tree_attend -- drafted tokens over a batch of caches
 *
 * Every sequence b of a batch has cached rows [0, L), L = cache_len[b], and behind them the rows of
 * its n = node_count[b] <= n_nodes drafted tokens (the caller writes them there, see reform_rotary_embed).
 * Node i sees all cached rows, itself and its ancestors:
 *     s_ij   = scale * <q_bhi, k_bgj>,  j in [0, L) or j - L in { i, parent[i], parent[parent[i]], ... }
 *     out, lse as in reform_chunk_attend_score
 *     q, out     [n_seq][n_q_heads][n_nodes][head_dim] by strides
 *     k, v       [n_seq][n_kv_heads][capacity][head_dim], rows contiguous, seq and head strides given
 *     cache_len  [n_seq] int32 in device memory; values outside [0, max_cache_len] are moved into it
 *     parent     [n_seq][n_nodes] int32 in device memory: a node before the node itself, or -1 (also for
 *                anything else) for one without a parent; NULL: each node's parent is the one before it, so
 *                that n_nodes = 1 is a generated token and NULL a short piece of text
 *     node_count [n_seq] int32 in device memory or NULL (all have n_nodes); values outside [0, n_nodes] are
 *                moved into it.  Rows of out and lse from node_count[b] on keep what they held.
 *     lse        [n_seq][n_q_heads][n_nodes] fp32, may be NULL
 * Supported: n_nodes in [1, 64]; types and head_dim as reform_prompt_attend, out and lse as there; max_cache_len + n_nodes at most
 * capacity and 2^31 - 512; n_seq * n_q_heads * n_nodes at most 2^22; with B = ceil(n_nodes * G / 16), n_seq * n_kv_heads * B *
 * ((max_cache_len + n_nodes) / 16 + 64) below 2^31.  n_seq = 0 does nothing.
 * The workspace takes partial results where long caches are shared out over workgroups.  Without it, or
 * with less than the query asks for, the call returns REFORM_ERR_WORKSPACE.  Results depend on the batch
 * that a sequence is computed in by rounding only (fp32 sums of the same terms in another order) and are
 * bitwise reproducible for the same arguments.
 */
typedef struct {
    uint32_t struct_size;
    int32_t  dtype;
    int32_t  n_seq, n_q_heads, n_kv_heads, head_dim;
    int32_t  n_nodes, max_cache_len, capacity;
    float    scale;                          /* > 0, finite                                    */
    int64_t  q_seq_stride, q_head_stride, q_row_stride, o_seq_stride, o_head_stride, o_row_stride;
    int64_t  kv_seq_stride, kv_head_stride;  /* elements, multiples of 16 bytes, as all strides */
} reform_tree_desc;

size_t reform_tree_attend_workspace(const reform_tree_desc *desc);

reform_status reform_tree_attend(const reform_tree_desc *desc, const void *q, const void *k, const void *v,
                                 const int32_t *cache_len, const int32_t *parent, const int32_t *node_count,
                                 void *out, float *lse, void *workspace, size_t workspace_bytes, void *hip_stream);

/* reform_tree_accept -- the drafted tokens that the model agrees with stay in the caches
 *
 * Node 0 is the last token that is certain already.  From it the path goes down as long as a child's drafted
 * token is the one the model chose after its parent (of several such children the first):
 *     path_0 = 0,   path_{m+1} = min { c > path_m : parent[c] = path_m, drafted[c] = target[path_m] }
 * Then row L + m of every cache becomes old row L + path_m, L = cache_len[b], m below the path's length, in
 * place; rows behind keep their content.
 *     parent, drafted, target  [n_seq][n_nodes] int32 in device memory; target[i]: the token the model chose
 *                  after node i.  parent NULL: a chain
 *     cache_len, node_count    as in reform_tree_attend; a sequence without nodes, or whose cache_len is
 *                  outside [0, capacity - nodes], is left alone (accepted 0, next_token -1)
 *     k, v         [n_layers] such caches, kv_layer_stride elements apart; both NULL: nothing moves
 *     path         [n_seq][n_nodes] int32 out, -1 behind the path, may be NULL
 *     accepted     [n_seq] int32 out: nodes on the path, may be NULL
 *     next_token   [n_seq] int32 out: target of the path's last node, may be NULL
 *     new_len      [n_seq] int32 out: cache_len + accepted, may be NULL; must not be cache_len itself
 * Outputs must not overlap the inputs or one another, nor the caches.
 * Supported: n_nodes in [1, 64]; head_dim * sizeof(element) a multiple of 16, at most 4096 bytes;
 * n_layers * n_seq * n_kv_heads at most 2^22.  n_seq = 0 does nothing.
 */
typedef struct {
    uint32_t struct_size;
    int32_t  dtype;
    int32_t  n_seq, n_kv_heads, head_dim;
    int32_t  n_nodes, capacity, n_layers;
    int64_t  kv_seq_stride, kv_head_stride, kv_layer_stride;   /* elements                     */
} reform_accept_desc;

reform_status reform_tree_accept(const reform_accept_desc *desc, const int32_t *parent, const int32_t *drafted,
                                 const int32_t *target, const int32_t *cache_len, const int32_t *node_count,
                                 void *k, void *v, int32_t *path, int32_t *accepted, int32_t *next_token,
                                 int32_t *new_len, void *hip_stream);

/* ------------------------------------------------------------------------------------------- */
/* reform_window_attend -- packed prompts whose rows see a sliding window and a few first keys
 *
 * As reform_prompt_attend, with fewer keys seen: row i of a sequence of nq query and nk key rows stands at
 * key t = nk - nq + i and sees
 *     j in [0, t] with j > t - window or j < n_sink
 * A window of nk keys or more gives reform_prompt_attend's results, up to rounding.  A row that sees no key (t < 0) gets out = 0 and lse = -inf.
 *     q, out, k, v, cu_q, cu_k, lse   as in reform_prompt_attend: layouts, lengths read on the device, boundaries that are out of
 *              place, rows of no sequence, arithmetic.  Keys and values that are not finite stay within their sequence; there, rows
 *              whose block goes through their tile of 64 keys may become NaN as well as those that see them
 * Supported: as reform_prompt_attend; window >= 1, n_sink >= 0; out and lse without a byte in common with the inputs or each other
 * (REFORM_ERR_INVALID_ARG).
 * No workspace is needed: the query gives 0, and what is passed is not looked at.  Few rows behind a wide window are not shared out over
 * workgroups, as reform_prompt_attend does it, which is the faster call there where the window covers all keys.
 */
typedef struct {
    uint32_t struct_size;
    int32_t  dtype;
    int32_t  n_q_heads, n_kv_heads, head_dim;
    int32_t  n_seq, n_q_rows, n_k_rows;
    float    scale;                          /* > 0, finite                                    */
    int32_t  window, n_sink;
    int32_t  reserved;                       /* 0                                              */
    int64_t  q_head_stride, q_row_stride, k_head_stride, k_row_stride;   /* elements, multiples */
    int64_t  v_head_stride, v_row_stride, o_head_stride, o_row_stride;   /* of 16 bytes         */
} reform_window_desc;

size_t reform_window_attend_workspace(const reform_window_desc *desc);

reform_status reform_window_attend(const reform_window_desc *desc, const void *q, const void *k, const void *v,
                                   const int32_t *cu_q, const int32_t *cu_k, void *out, float *lse,
                                   void *workspace, size_t workspace_bytes, void *hip_stream);

/* ------------------------------------------------------------------------------------------- */
/* reform_paged_attend -- one new token of each of a batch of sequences over caches in pages
 *
 * Sequence b has L = cache_len[b] keys, the new token's own (the last one) among them.  Key j lies in row j % page_len of page
 * page_table[b][j / page_len] of a pool that all sequences share (reform_rotary_embed writes there: slot = page * page_len +
 * row).  Seen are
 *     j in [0, L) with window = 0, or j >= L - window, or j < n_sink
 * and of these the ones whose page number lies in [0, n_pages): a page that was given back, or was never there, is -1 in the
 * table, and nothing of it is read.
 *     s_hj  = scale * <q_bh, k_j>,   out_bh = sum_j softmax_j(s_hj) v_j,   lse_bh = log sum_j exp(s_hj)
 *     score_bgj (+)= sum_{h in group g} softmax_j(s_hj): the attention that the key received (the eviction score of
 *              reform_paged_evict).  accumulate = 0: entries [0, L) are written, 0 for keys that are not seen.  accumulate = 1: keys
 *              that are seen get it added, the others keep what they have; but entry L - 1, the new token's, is written
 * A sequence that sees no key (L = 0, as padding of a batch) gets out = 0 and lse = -inf.
 *     q, out      [n_seq][n_q_heads][head_dim] by strides
 *     k, v        [n_pages][n_kv_heads][page_len][head_dim] by the strides of a page, a head and a row (a pool of
 *                 [pages][rows][heads][elements] is addressed in place), elements of a row contiguous
 *     page_table  [n_seq][max_pages] int32 in device memory, rows table_stride apart
 *     cache_len   [n_seq] int32 in device memory; values outside [0, max_len] are moved into it
 *     score       [n_seq][n_kv_heads][>= max_len] fp32 by strides, entries contiguous; may be NULL
 *     lse         [n_seq][n_q_heads] fp32, may be NULL
 * out, lse and score have no byte in common with the inputs or one another (REFORM_ERR_INVALID_ARG; they may lie between one another's rows).
 * Arithmetic: products and sums in fp32; for bf16 the probabilities of the P.V product are taken in two bf16 parts (16 bits), the score sums the
 * unrounded fp32 ones.  Bitwise reproducible for the same arguments; results depend on the batch and on max_len by rounding only.
 * Keys and values that are not finite matter where they are seen only, and there stay within their sequence and KV head (an infinite
 * value may give NaN), in the score within the keys that are seen.  Rows behind L are never looked at.
 * Supported: types and head_dim as reform_prompt_attend; any page_len >= 1; n_pages * page_len below 2^31; max_len at most
 * max_pages * page_len and 2^31 - 65536; row stride of k and v below 2^24; n_seq * n_q_heads at most 2^22; with B = ceil(n_q_heads /
 * n_kv_heads / 16), n_seq * n_kv_heads * B * (max_len / 16 + 64) below 2^31.  n_seq = 0 does nothing.
 * The workspace takes partial results of caches that are shared out over workgroups, and the logits of all keys if the score is asked
 * for (4 bytes a key that can be seen and query head); the query wants to know whether it is: want_score.  Without it, or with less than the
 * query asks for, the call returns REFORM_ERR_WORKSPACE.  The host knows max_len and not the lengths: that decides the workspace's size, how
 * the keys are shared out, and whether K and V go past the caches' order of replacement (64 MB and more of them), so a bound that fits the batch
 * is the faster one.
 * The score is that of generated tokens: the calls on prompts add nothing to it, and the first eviction after a prompt ranks its keys by what the
 * tokens since then gave them.  A program that wants more in it before writes that into score.
 */
typedef struct {
    uint32_t struct_size;
    int32_t  dtype;
    int32_t  n_seq, n_q_heads, n_kv_heads, head_dim;
    int32_t  page_len, n_pages, max_pages, max_len;
    int32_t  window, n_sink;                 /* window >= 0 (0: all keys), n_sink >= 0         */
    int32_t  want_score;                     /* 1 iff score is not NULL                        */
    int32_t  accumulate;                     /* 0: score = ..., 1: score += ...                */
    float    scale;                          /* > 0, finite                                    */
    int32_t  reserved;                       /* 0                                              */
    int64_t  q_seq_stride, q_head_stride, o_seq_stride, o_head_stride;   /* elements, multiples of 16 bytes */
    int64_t  kv_page_stride, kv_head_stride, kv_row_stride;              /* likewise           */
    int64_t  table_stride, score_seq_stride, score_head_stride;          /* elements           */
} reform_paged_desc;

size_t reform_paged_attend_workspace(const reform_paged_desc *desc);

reform_status reform_paged_attend(const reform_paged_desc *desc, const void *q, const void *k, const void *v,
                                  const int32_t *page_table, const int32_t *cache_len, float *score,
                                  void *out, float *lse, void *workspace, size_t workspace_bytes, void *hip_stream);

/* ------------------------------------------------------------------------------------------- */
/* reform_paged_evict -- caches in pages go back to their budget
 *
 * The rule of reform_evict_topk_compact for every sequence b of a batch and every KV head: of L = cache_len[b] > budget keys those
 * `budget` are kept whose score is largest (ties: the lowest index), the first n_sink and the last n_recent always
 * among them.  Then row r of the head becomes old row kept_idx[r], r < budget, in ascending order, for k, v, score and pos
 * alike, in place.  A sequence of L <= budget keys stays as it is (kept_idx[r] = r).  Rows behind keep what they held.
 * new_len[b] = min(L, budget): pages behind it can be given back.
 *     k, v, page_table, cache_len   as in reform_paged_attend; the pages of sequences that outgrew their budget must be their
 *              own: a page that is in the table twice holds undefined rows afterwards.  Rows whose page number lies outside
 *              [0, n_pages) are neither read nor written: what would come from there leaves the row it would go to as it is
 *     score    [n_seq][n_kv_heads][>= max_len] fp32 by strides, entries contiguous, in/out; must be finite (no NaN/Inf)
 *     pos      like score, with its strides, int32 that travel with the rows, in/out; may be NULL
 *     kept_idx [n_seq][n_kv_heads][budget] int32 out, contiguous, the first new_len entries of a head; may be NULL
 *     new_len  [n_seq] int32 out, may be NULL
 * k, v, score, pos, kept_idx and new_len have no byte in common with one another or the inputs (REFORM_ERR_INVALID_ARG; k and v may be
 * parts of one pool).
 * The workspace takes the kept keys, and rows that are set aside where few heads have many; the query gives 0 where max_len is within
 * the budget.  Without it, or with less than the query asks for, the call returns REFORM_ERR_WORKSPACE.
 * Supported: head_dim * sizeof(element) a multiple of 16 up to 4096; strides of k and v multiples of 16 bytes; page_len, n_pages,
 * max_pages, max_len as in reform_paged_attend; budget at least 1; n_seq * n_kv_heads * (row bytes / 64 + 4) below 2^22.  n_seq = 0 does
 * nothing.
 */
typedef struct {
    uint32_t struct_size;
    int32_t  dtype;
    int32_t  n_seq, n_kv_heads, head_dim;
    int32_t  page_len, n_pages, max_pages, max_len;
    int32_t  budget, n_sink, n_recent;       /* n_sink + n_recent <= budget                    */
    int64_t  kv_page_stride, kv_head_stride, kv_row_stride;              /* elements           */
    int64_t  table_stride, score_seq_stride, score_head_stride;
} reform_paged_evict_desc;

size_t reform_paged_evict_workspace(const reform_paged_evict_desc *desc);

reform_status reform_paged_evict(const reform_paged_evict_desc *desc, void *k, void *v, float *score, int32_t *pos,
                                 const int32_t *page_table, const int32_t *cache_len, int32_t *kept_idx, int32_t *new_len,
                                 void *workspace, size_t workspace_bytes, void *hip_stream);

/* ------------------------------------------------------------------------------------------- */
/* Measurement aids (no step of the method): what this machine sustains on the resources the
 * kernels above are bound by, so a benchmark can quote a kernel against the measured ceiling as
 * well as against the data-sheet one.
 *
 * reform_probe_mfma_bf16: `workgroups` workgroups of 8 waves each run `iters` trips of 16
 *   v_mfma_f32_16x16x32_bf16 (4 x 4 operand registers, all combinations) and nothing else;
 *   executed flop = workgroups * 8 * iters * 16 * 16384.  `operands`: 64 KiB of device memory
 *   holding the bf16 values to multiply (random data heats the chip like real inputs, zeros do
 *   not); `sink`: 16 bytes of device memory that is practically never written.
 * reform_probe_stream: reads `bytes` (a multiple of 16) from src with 16-byte loads and, if dst is
 *   not NULL, stores them to dst (a plain copy: bytes read + bytes written); with dst == NULL it
 *   is a read-only stream.  `sink` as above.
 * Both only enqueue one kernel on hip_stream.                                                   */
reform_status reform_probe_mfma_bf16(const void *operands, float *sink, int32_t iters,
                                     int32_t workgroups, void *hip_stream);
reform_status reform_probe_stream(const void *src, void *dst, size_t bytes, void *sink,
                                  void *hip_stream);

const char *reform_status_string(reform_status status);

/* Library version, major*10000 + minor*100 + patch.                                            */
int32_t reform_version(void);

#ifdef __cplusplus
}
#endif
#endif /* REFORM_H */
