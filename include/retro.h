/*
 * retro.h — C ABI of an MI355X (gfx950) library for one decode step of
 * retrospective sparse attention ("Retrospective Sparse Attention for
 * Efficient Long-Context Generation", Alg. 1 without its UpdateKV step).
 *
 * One step of one attention layer, for a batch of sequences:
 *   1. append the step's key/value to a paged KV cache and keep per-page key
 *      min/max digests (Sec. 2.1, "Dynamic Sparse Attention");
 *   2. score every page against the current query, eq. (quest_score), and keep
 *      the top-k pages under a token budget (PageSelect);
 *   3. record, per KV head and page, the last step the page was loaded, and hand
 *      the previous value to the attention kernel (Alg. 2, UpdateAndBuildMask);
 *   4. one attention pass over the selected pages for the current query and the
 *      W past queries of the retrospective window, a past query taking only the
 *      pages it has not seen (eq. update-org, eq. update-sup, "Retrospective
 *      Mask" paragraph);
 *   5. merge the past queries' supplementary outputs into an output cache of
 *      (output, log-sum-exp) per past query, eq. (merged_attn_general), and
 *      return the finished output of the query leaving the window.
 *
 * Window convention: W counts PAST queries.  A step processes W+1 queries:
 * row r of the window is the query of step tau = t - W + r, row W the current
 * one.  (The paper's window w counts the current query too: W = w - 1.)
 * W = 0 is plain query-aware sparse attention without retrospection.
 *
 * Conventions for every entry point
 *   - All buffers are caller-owned DEVICE memory, contiguous, row-major, with
 *     the layouts given below.  The library allocates nothing and keeps no state
 *     between calls; scratch lives in the caller's `workspace`.
 *   - Work is enqueued on `stream` (a hipStream_t; NULL = the default stream)
 *     and is asynchronous: no call synchronises the host.
 *   - Argument errors are detected on the host before anything is enqueued and
 *     return RETRO_EINVAL / RETRO_EUNSUPPORTED / RETRO_EWORKSPACE; a failed
 *     launch returns RETRO_EHIP.  No C++ exception crosses the ABI.
 *   - Device-side contract (not checkable on the host): seq_lens, page_table,
 *     selections and the mask hold values produced by this library or obeying
 *     the ranges documented here.  Out-of-range page numbers are skipped by the
 *     kernels instead of being dereferenced.
 *   - Calls that share buffers must be ordered by the caller (same stream).
 */
#ifndef RETRO_H
#define RETRO_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef enum {
  RETRO_OK = 0,
  RETRO_EINVAL = -1,        /* null pointer, negative size, inconsistent dimension */
  RETRO_EUNSUPPORTED = -2,  /* well-formed but outside the supported shapes */
  RETRO_EHIP = -3,          /* a HIP launch or query failed */
  RETRO_EWORKSPACE = -4,    /* workspace null or smaller than retro_workspace_size() */
  RETRO_ESCRATCH = -5       /* retro_step_noalloc: the step needs more than the library's
                               static scratch, or a clear of it would be captured */
} retro_status;

typedef enum { RETRO_F32 = 0, RETRO_BF16 = 1 } retro_dtype;

/* Bits of retro_dims.flags.  0 lets retro_step choose its launches (the normal
 * case); RETRO_FLAG_KV_MX4 says how the cache is held; the other bits select a launch
 * sequence explicitly or test the failure path, with the same results. */
typedef enum {
  /* retro_step: the page scores take a launch of their own even where the
   * scores, selection and attention fit in one launch */
  RETRO_FLAG_SEPARATE_SCORES = 1,
  /* retro_step: the selection follows the scores, ahead of the attention launch
   * (implies a separate score launch) */
  RETRO_FLAG_SELECT_IN_SCORES = 2,
  /* tests of the failure path only: every bounded wait between the workgroups
   * of a launch gives up after a few polls, as if its producers never came */
  RETRO_FLAG_TEST_WAIT_TIMEOUT = 4,
  /* the cache's keys and values are held in 4 bits (see "The cache in 4 bits" below) */
  RETRO_FLAG_KV_MX4 = 16
} retro_flag;

/* Problem statement of one layer.  Supported: head_dim 64 or 128; page_size
 * 16 or 32; 1 <= group <= 16; 0 <= window <= 64; (window+1)*group <= 1024;
 * page_size <= budget_tokens; 0 <= budget_permille <= 1000; max_pages <= 16384;
 * flags a combination of retro_flag bits. */
typedef struct retro_dims {
  int32_t batch;           /* sequences in the batch                                   */
  int32_t num_kv_heads;    /* h_k                                                      */
  int32_t group;           /* G query heads per KV head; h_q = h_k * G (GQA)            */
  int32_t head_dim;        /* d                                                        */
  int32_t page_size;       /* P tokens per page                                        */
  int32_t budget_tokens;   /* B; each step keeps k = min(B_t / P, pages of the sequence) */
  int32_t window;          /* W past queries revisited per step                        */
  int32_t max_pages;       /* length of a page-table row (logical pages per sequence)  */
  int32_t num_phys_pages;  /* physical pages in k_cache / v_cache / digest             */
  int32_t dtype;           /* retro_dtype of queries, keys, values and digests         */
  float sm_scale;          /* softmax scale applied to q.k; 0 selects 1/sqrt(d)         */
  int32_t budget_permille; /* relative budget (Sec. 4 ablation; Table 1's setting of
                              0.15 = 150): B_t = max(B, floor(L * budget_permille /
                              1000)) tokens for a sequence of L tokens (the step's
                              token included); 0: B_t = B.  k_max covers the largest
                              B_t of a full page-table row.                          */
  int32_t flags;           /* retro_flag bits; 0 for normal use                        */
  int32_t reuse_interval;  /* top-k selection reuse, the baseline of the paper's
                              motivational study (Appendix, Table 4) as an alternative
                              PageSelect: with f = reuse_interval >= 2, steps t with
                              t mod f != 0 keep the selection (rows and counts) that
                              `sel` holds from the previous step, unscored, and run
                              UpdateAndBuildMask (Alg. 2) on it; steps with t mod f
                              == 0 select as usual.  0 or 1: every step selects.    */
} retro_dims;

/* The paged KV cache of one layer (Sec. 2.1; pages as in a vLLM-style pool), in dtype; with
 * RETRO_FLAG_KV_MX4 the pages of keys and values are in 4 bits instead.
 *   k_cache     [num_phys_pages][h_k][P][d]   dtype  key page, token-major
 *   v_cache     [num_phys_pages][h_k][d][P]   dtype  value page, stored transposed
 *                                                    (d-major) so that the token
 *                                                    contraction reads contiguously
 *   digest      [batch][h_k][max_pages][2][d] dtype  per LOGICAL page of each sequence:
 *                                                    [0] = element-wise key minimum,
 *                                                    [1] = maximum over the page's
 *                                                    stored tokens (Quest digest); a
 *                                                    head's digests are one contiguous
 *                                                    stream for the page scan
 *   page_table  [batch][max_pages]            int32  logical page -> physical page
 *   seq_lens    [batch]                       int32  tokens stored per sequence
 *   last_loaded [batch][h_k][max_pages]       int32  A of Alg. 2: last decode step in
 *                                                    which each logical page was
 *                                                    loaded; the caller initialises it
 *                                                    to -1 before the first step.
 * Slots beyond seq_lens are never read as keys; their values are zeroed before use. */
typedef struct retro_kv_cache {
  void* k_cache;
  void* v_cache;
  void* digest;
  const int32_t* page_table;
  int32_t* seq_lens;
  int32_t* last_loaded;
} retro_kv_cache;

/* Output of page selection (PageSelect + UpdateAndBuildMask).
 *   selected     [batch][h_k][k_max]  int32  logical page ids in ascending order,
 *                                            -1 after the first num_selected entries
 *   mask         [batch][h_k][k_max]  int32  M of Alg. 2: last_loaded of each selected
 *                                            page before this step (-1 padding)
 *   num_selected [batch][h_k]         int32
 * with k_max = retro_k_max(dims). */
typedef struct retro_selection {
  int32_t* selected;
  int32_t* mask;
  int32_t* num_selected;
} retro_selection;

/* The attention output cache (Sec. 2.3, "Attention Output Cache"): for each of the
 * last W steps tau, the output of tau's query merged over every supplement so
 * far, in ring slot tau mod W.
 *   o_cache   [batch][W][h_q][d]  fp32
 *   lse_cache [batch][W][h_q]     fp32 natural-log normaliser (log of alpha)
 * Slots are only read after the step that wrote them; no initialisation needed.
 * Both may be NULL when W == 0. */
typedef struct retro_output_cache {
  float* o_cache;
  float* lse_cache;
} retro_output_cache;

/* Library version string. */
const char* retro_version(void);

/* Human-readable name of a status code. */
const char* retro_status_string(int32_t status);

/* Validate dims; on success write k_max = min(budget_tokens / page_size, max_pages). */
retro_status retro_k_max(const retro_dims* dims, int32_t* k_max);

/* Bytes of scratch the select / attend / step calls need for these dims.  The
 * workspace holds, besides scratch, the words through which the workgroups of
 * one launch hand work to each other and a sticky error word: zero-fill it once
 * before its first use and let one call at a time use it (calls sharing a
 * workspace are ordered on one stream).  Use it with the dims it was sized for:
 * a one-launch step (see retro_step) on a workspace last used by a one-launch
 * step of another geometry sets the error word instead of running (its outputs
 * are NaN) until the workspace is zero-filled again. */
retro_status retro_workspace_size(const retro_dims* dims, size_t* bytes);

/* Bulk-store n_tokens tokens of sequence `seq` at positions start_pos ..
 * start_pos+n_tokens-1 (k_src, v_src: [n_tokens][h_k][d] dtype, device) and
 * rebuild the digests of the pages they touch.  start_pos must equal the
 * sequence's current seq_lens entry, which becomes start_pos + n_tokens.  For the
 * prefill that precedes the first decode step: last_loaded is not touched. */
retro_status retro_prefill_kv(const retro_dims* dims, const retro_kv_cache* cache, int32_t seq,
                              int32_t start_pos, int32_t n_tokens, const void* k_src,
                              const void* v_src, void* stream);

/* AppendKV (Alg. 1) of one token per sequence (k_new, v_new: [batch][h_k][d] dtype)
 * at position seq_lens[b], which is then incremented.  The page's digest widens to
 * the new key (or starts at it for the page's first slot), and last_loaded of that
 * page is set to step-1 for every head: Alg. 2's current-page rule, applied when a
 * page receives a key newer than every past query.  May be called several times
 * per step (several tokens per step).  A token whose logical page is not mapped
 * (page_table entry < 0 or >= num_phys_pages, or position >= max_pages*P) is
 * dropped and seq_lens is left unchanged. */
retro_status retro_append_kv(const retro_dims* dims, int32_t step, const retro_kv_cache* cache,
                             const void* k_new, const void* v_new, void* stream);

/* AppendKV (Alg. 1) of n_tokens tokens per sequence in order, with the result of
 * n_tokens calls of retro_append_kv (token j of sequence b at position
 * seq_lens[b] + j, digests widened, last_loaded of every page receiving a key set
 * to step-1 for every head), in one launch per 64 tokens: for steps that add
 * several tokens (e.g. the tokens before the last of a multi-token step, whose
 * last token goes through retro_step).  k_new / v_new [n_tokens][batch][h_k][d]
 * (dtype), device memory, read only.  The first token whose logical page is not
 * mapped (page_table entry < 0 or >= num_phys_pages, or position >= max_pages*P)
 * is dropped with every later token of the call, and seq_lens[b] advances by
 * the number appended.  n_tokens = 0 does nothing; n_tokens < 0 or a null
 * k_new / v_new (n_tokens > 0) is RETRO_EINVAL. */
retro_status retro_append_kv_tokens(const retro_dims* dims, int32_t step,
                                    const retro_kv_cache* cache, int32_t n_tokens,
                                    const void* k_new, const void* v_new, void* stream);

/* UpdateKV (Alg. 1; Sec. 3.3, retrospective KV cache update): the keys and values
 * of the n_tokens most recent stored tokens of every sequence b (positions
 * seq_lens[b] - n_tokens .. seq_lens[b] - 1; those below 0 are skipped) are
 * overwritten with k_upd / v_upd [batch][n_tokens][h_k][d] (dtype; row j is
 * position seq_lens[b] - n_tokens + j), e.g. re-embedded from the previous
 * layer's updated outputs, and the digest of every page they touch is recomputed
 * as the element-wise min / max over its stored keys.  Called before the step's
 * append (Alg. 1 order), with n_tokens = W for the window's past tokens.
 * last_loaded and seq_lens are unchanged.  n_tokens = 0 does nothing. */
retro_status retro_update_kv(const retro_dims* dims, const retro_kv_cache* cache,
                             int32_t n_tokens, const void* k_upd, const void* v_upd,
                             void* stream);

/* PageSelect + UpdateAndBuildMask (Alg. 1, Alg. 2) for the current query
 * q_cur [batch][h_q][d] (dtype).
 *   score of page p of KV head h = sum over the G query heads g of h of
 *     sum_i max(q_gi * Kmin_pi, q_gi * Kmax_pi)                  eq. (quest_score)
 *   evaluated in fp32: products rounded to fp32, the d terms summed as a perfect
 *   binary tree over index order, the G head sums added in order, then + 0.0f.
 *   The k = min(B_t/P, ceil(seq_len/P)) best pages by (score descending, page index
 *   ascending) are written in ascending order; then for each selected page p, in
 *   order: mask = last_loaded[p]; last_loaded[p] = step.
 * Page selection is exact: it depends on no floating-point reduction order other
 * than the one stated. */
/* (With dims->reuse_interval = f >= 2 and step mod f != 0 no score is computed:
 * the rows and counts `sel` holds are kept, and only the mask / last_loaded
 * loop above runs on them; q_cur is not read.) */
retro_status retro_select_pages(const retro_dims* dims, int32_t step, const void* q_cur,
                                const retro_kv_cache* cache, const retro_selection* sel,
                                void* workspace, size_t ws_bytes, void* stream);

/* Attention of the W+1 window queries q_window [batch][W+1][h_q][d] (dtype; row W
 * is step t) over the selected pages.  Row r (tau = t-W+r) uses page p iff tau >= 0
 * and (r == W or mask[p] < tau); every stored token of a used page counts.
 * Output per row and query head: o_part [batch][W+1][h_q][d] fp32 (softmax-weighted
 * values) and lse_part [batch][W+1][h_q] fp32 = ln sum exp(sm_scale * q.k);
 * an empty set gives (0, -inf).  A NaN score, or one of +inf, makes its row's
 * outputs and log-normaliser NaN (also through retro_step and
 * retro_merge_output_cache).  A NaN or infinite value of a selected page can reach
 * every row of its KV head, also rows that do not use the page: a zero weight
 * times it is NaN.  Reads only; writes o_part, lse_part, workspace. */
retro_status retro_decode_attend(const retro_dims* dims, int32_t step, const void* q_window,
                                 const retro_kv_cache* cache, const retro_selection* sel,
                                 float* o_part, float* lse_part, void* workspace,
                                 size_t ws_bytes, void* stream);

/* The attention pass of retro_decode_attend alone, as one kernel launch: each
 * split's partial (O, LSE) stays in the workspace (library-private layout) and
 * nothing else is written.  Meant for timing the page-gather attention kernel in
 * isolation (the paper's kernel-level breakdown separates it from the merge);
 * callers wanting outputs use retro_decode_attend or retro_step. */
retro_status retro_decode_attend_partials(const retro_dims* dims, int32_t step,
                                          const void* q_window, const retro_kv_cache* cache,
                                          const retro_selection* sel, void* workspace,
                                          size_t ws_bytes, void* stream);

/* The kernel launch of retro_step that ends in the attention partials, alone:
 * page scores (eq. quest_score), selection (top-k + UpdateAndBuildMask's mask,
 * Alg. 2) and attention, with the sequence lengths of `cache` (no token is
 * appended).  Where retro_step scores in a launch of its own (see retro_step),
 * the launch starts from the page scores the last retro_step or
 * retro_select_pages call with this workspace left in it.  Writes the page
 * scores, sel's rows, mask and count (mask values from last_loaded as it
 * stands, which this call does not update) and the splits' partials in the
 * workspace.  Meant for timing the step's dominant kernel in isolation;
 * returns RETRO_EUNSUPPORTED where retro_step selects outside the attention
 * launch (max_pages > 6144). */
retro_status retro_step_attend_partials(const retro_dims* dims, int32_t step,
                                        const void* q_window, const retro_kv_cache* cache,
                                        const retro_selection* sel, void* workspace,
                                        size_t ws_bytes, void* stream);

/* The page scores, eq. (quest_score) in the fp32 order of retro_select_pages,
 * that the last retro_step, retro_step_attend_partials or retro_select_pages
 * call with this workspace computed: copied (asynchronously, on `stream`) to
 * scores [batch][h_k][max_pages] fp32, device memory.  Entries of pages at or
 * past a sequence's page count are unspecified.  Meant for checking the scores
 * bit for bit; workspace as sized by retro_workspace_size for these dims. */
retro_status retro_copy_scores(const retro_dims* dims, const void* workspace, size_t ws_bytes,
                               float* scores, void* stream);

/* MergeOutput + CacheOutput (Alg. 1; eq. merged_attn_general) for step t.
 * For each query head and row r with tau = t-W+r >= 0:
 *   r == W   : out = part; pushed to slot t mod W;
 *   0 < r < W: out = merge(slot tau mod W, part); written back to the slot;
 *   r == 0   : out = merge(slot, part) is final (the query leaves the window), and
 *              the slot (t-W) mod W = t mod W is then reused by row W;
 * where merge((O_a,Z_a),(O_b,Z_b)) = ((e^Za O_a + e^Zb O_b)/(e^Za + e^Zb),
 * ln(e^Za + e^Zb)), a -inf side contributing nothing.  Rows with tau < 0 give
 * o_out = 0, lse_out = -inf and touch no slot.
 *   o_out [batch][W+1][h_q][d] fp32, lse_out [batch][W+1][h_q] fp32. */
retro_status retro_merge_output_cache(const retro_dims* dims, int32_t step, const float* o_part,
                                      const float* lse_part, const retro_output_cache* ocache,
                                      float* o_out, float* lse_out, void* stream);

/* One whole step: retro_append_kv(k_new, v_new), retro_select_pages(row W of
 * q_window), retro_decode_attend, retro_merge_output_cache, with the same
 * semantics, without materialising o_part / lse_part.
 * One launch where every workgroup of it fits on the GPU at once (as the
 * occupancy of its kernel times the compute units tells; up to 4480 pages per
 * sequence and 160 per workgroup, (window + 1) * group <= 128 rows, at most 64
 * KV heads and 1024 workgroups):
 * page scores (with the append), selection, attention, combine + merge, the
 * last_loaded update and the seq_lens advance, the workgroups of a KV head
 * handing each other scores and partial results through tagged words in
 * `workspace` (each word carries the launch's epoch; no counters, no fences).
 * That needs every workgroup resident at once: work of other streams or
 * processes holding compute units delays it until they free them; a wait that
 * runs past its bound (tens of milliseconds) sets the sticky error word in
 * `workspace`: the outputs of that step and of every later step with this
 * workspace are then NaN, and the output cache, last_loaded and seq_lens are
 * left as they were, until the workspace is zero-filled again
 * (RETRO_FLAG_TEST_WAIT_TIMEOUT in dims->flags makes every such wait give up
 * at once, for tests of that path).
 * Otherwise, or with RETRO_FLAG_SEPARATE_SCORES, three launches: the scores
 * (with the append), then attention with every attention workgroup selecting
 * in front of it, then combine + merge; with RETRO_FLAG_SELECT_IN_SCORES or
 * for max_pages > 6144, the selection runs right after the scores, in a launch
 * of its own, instead.  Steps
 * that keep an earlier selection (top-k reuse, retro_dims.reuse_interval) run
 * the append, Alg. 2 on the kept rows, attention and combine + merge as four
 * launches. */
retro_status retro_step(const retro_dims* dims, int32_t step, const void* q_window,
                        const void* k_new, const void* v_new, const retro_kv_cache* cache,
                        const retro_selection* sel, const retro_output_cache* ocache,
                        float* o_out, float* lse_out, void* workspace, size_t ws_bytes,
                        void* stream);

/* The number of kernel launches retro_step makes for these dims on the current
 * device in a step that selects (1: scores, selection, attention and merge in
 * one launch; 3 or 4: see retro_step; 4 or 5 over a cache in 4 bits; a top-k reuse
 * step always makes 4), in *launches.  Host only: nothing is enqueued. */
retro_status retro_step_launches(const retro_dims* dims, int32_t* launches);

/* How the attention of these dims is launched on the current device: *row_tiles
 * = the tiles of 16 window rows that a workgroup of the streamed kernel takes, or
 * 0 where the kernel that stages chunks through LDS takes the call (fp32, and
 * small calls for which it is the faster one); *splits = the parts of the
 * selection per KV head.  selects == 0: retro_decode_attend and the attention
 * launch of steps without a selection in front of it; else the attention of a
 * step of three launches.  Over a cache in 4 bits *row_tiles is 1 or 2 and `selects`
 * makes no difference.  Host only: nothing is enqueued. */
retro_status retro_attend_plan(const retro_dims* dims, int32_t selects, int32_t* row_tiles,
                               int32_t* splits);

/* retro_step for callers that cannot allocate (code under HIP graph capture,
 * tight serving loops, harnesses that forbid allocation): the same step and
 * results, with the workspace in a static device array of the library (64 MiB
 * per GPU, held until the process ends) instead of a caller's buffer; the
 * caller still passes every input and output.  No allocation is made.
 * Steps whose retro_workspace_size exceeds 64 MiB return RETRO_ESCRATCH.
 * Every call on a GPU shares that GPU's array, which keeps the last call's
 * contents: a call whose dims (flags aside) differ from the previous call's on
 * the device first clears the part it uses, with a kernel on `stream`; if that
 * stream is being captured the call returns RETRO_ESCRATCH instead (make the
 * first call of a geometry outside the capture).  Calls that overlap on one
 * GPU (other streams or host threads) race on the array.  After a wait that
 * gives up (see retro_step), later calls fail until the dims change. */
retro_status retro_step_noalloc(const retro_dims* dims, int32_t step, const void* q_window,
                                const void* k_new, const void* v_new,
                                const retro_kv_cache* cache, const retro_selection* sel,
                                const retro_output_cache* ocache, float* o_out,
                                float* lse_out, void* stream);

/* ---- Projections of the multi-layer decode with re-embedding (Sec. 3.3) --------
 * Every layer projects the W+1 window rows of every sequence (rows = batch*(W+1),
 * at most 112) to queries, keys and values, and its merged outputs back to the
 * model width; the past rows are re-embedded from the layer below's updated
 * outputs, their new keys and values then go to retro_update_kv.  With so few
 * rows the products are bound by reading the weights, which are therefore kept
 * pre-tiled for the matrix cores.  bf16 weights and inputs, fp32 accumulation,
 * bf16 results rounded to nearest even.  Every pointer is a device address,
 * 16-byte aligned; the caller owns every buffer. */

/* Tiles a weight w [k][n] bf16 (row-major, y = x . w) into w_packed (k*n bf16, a
 * separate buffer): element (i, j) goes to [j/16][i/32][(i%32)/8][j%16][i%8].
 * Weights that share an input (query, key and value) are packed as one [k][n]
 * matrix with their columns side by side.  k % 32 == 0 and n % 16 == 0, else
 * RETRO_EUNSUPPORTED. */
retro_status retro_pack_weight(const void* w, int32_t k, int32_t n, void* w_packed,
                               void* stream);

/* q = x . Wq, k_out = x . Wk, v = x . Wv for x [rows][k] bf16 and a packed
 * [k][n_q + 2 n_kv] weight whose columns are Wq's, then Wk's, then Wv's; outputs
 * bf16 [rows][n_q], [rows][n_kv], [rows][n_kv] (for the window rows of a
 * decoder: [batch][W+1][h_q][d] and [batch][W+1][h_k][d]).  Supported: 1 <= rows
 * <= 112, k % 1024 == 0, n_q % 16 == n_kv % 16 == 0 (else RETRO_EUNSUPPORTED);
 * rows == 0 does nothing. */
retro_status retro_project_qkv(const void* x, int32_t rows, int32_t k, const void* w_packed,
                               int32_t n_q, int32_t n_kv, void* q, void* k_out, void* v,
                               void* stream);

/* retro_project_qkv for the window rows of one decoder layer (rows = batch *
 * (W+1), x [batch][W+1][k] bf16, a packed [k][(h_q + 2 h_k) d] weight) with the
 * layer's UpdateKV folded in (Alg. 1; Sec. 3.3): q [batch][W+1][h_q][d] receives
 * every row's query; k_new, v_new [batch][h_k][d] the newest row's key and value
 * (for retro_step, which appends them); the keys and values of the n_update rows
 * before the newest overwrite the sequence's last n_update stored tokens, as
 * retro_update_kv would (positions seq_lens[b] - n_update .. seq_lens[b] - 1,
 * those below 0 skipped), and the digests of the pages they touch are
 * recomputed.  Call it before the step, whose append advances seq_lens.  bf16
 * dims only; 0 <= n_update <= W; rows <= 112, k % 1024 == 0 (else
 * RETRO_EUNSUPPORTED). */
retro_status retro_project_qkv_update(const retro_dims* dims, const retro_kv_cache* cache,
                                      const void* x, int32_t k, const void* w_packed,
                                      int32_t n_update, void* q, void* k_new, void* v_new,
                                      void* stream);

/* The output projection and the residual add: y = bf16(o) . Wo for o [rows][k]
 * fp32 (a decoder's merged outputs o_out, k = h_q * d) and a packed [k][n]
 * weight, rounded to bf16; then h[r][j] += y[r][j] in fp32 (h [rows][n], the
 * residual stream, updated in place) and x_next = bf16(h) [rows][n] (the next
 * layer's input).  Supported shapes as for retro_project_qkv. */
retro_status retro_project_out(const float* o, int32_t rows, int32_t k, const void* w_packed,
                               int32_t n, float* h, void* x_next, void* stream);

/* The projections of the multi-layer decode (Sec. 3.3) for fp32 stacks:
 * y = x . w (accumulate == 0) or y += x . w (accumulate != 0: the output
 * projection added into the residual stream in place) for x [rows][k] and w
 * [k][n] fp32 row-major (not packed), y [rows][n] fp32; x and y must not
 * overlap.  Each output element is one fp32 fused multiply-add chain over
 * i = 0 .. k-1 in order, so results repeat exactly from run to run.  rows == 0
 * does nothing; rows > 65535 or rows * n >= 2^31 is RETRO_EUNSUPPORTED. */
retro_status retro_project_f32(const float* x, int32_t rows, int32_t k, const float* w,
                               int32_t n, float* y, int32_t accumulate, void* stream);

/* ---- Prompts, chunks of prompts and rotated positions ---------------------------
 * What precedes and surrounds the retrospective steps in a model whose keys and
 * queries carry their positions: per-head norms and the rotation, the storage of
 * a ragged batch of rows with both applied on the way, and the attention of these
 * rows over everything stored.  Of retro_dims these calls use batch,
 * num_kv_heads, group, head_dim, page_size, max_pages, num_phys_pages, dtype and
 * sm_scale (the others have to be valid).  Rows are tokens: queries [rows][h_q][d], keys and values
 * [rows][h_k][d] in dtype, where `*_stride` elements lie between the rows of an
 * input (parts of one projection's output: its row length; else heads * d).
 * Outputs are contiguous.  Every pointer is a device address, 16-byte aligned
 * except the arrays of int32 and lse, and every stride a multiple of 16 bytes and
 * no less than heads * d (RETRO_EINVAL otherwise). */

/* Norm and rotation.  For a head's vector x at position p:
 *   y = x * (mean(x^2) + eps)^(-1/2) * weight      (weight NULL: y = x)
 * and, with (c, s) = table[p][i], pair i of y's first rot_dim elements becomes
 *   (a, b) -> (a c - b s, b c + a s)
 * in fp32, rounded once to dtype.  rot_dim: a multiple of 16 up to d; 0 leaves
 * the rotation out (table may be NULL then). */
typedef struct retro_rotary {
  const float* table;   /* [positions][rot_dim / 2][2] cosine, sine (retro_rotary_table)  */
  int32_t positions;    /* rows of table                                                */
  int32_t rot_dim;      /* rotated elements of a head, the leading ones                  */
  int32_t interleaved;  /* 0: pair i is (i, i + rot_dim / 2); 1: it is (2 i, 2 i + 1)     */
  float eps;            /* >= 0, finite                                                 */
  const void* q_norm;   /* [d] dtype, weights of the queries' norm; NULL: none           */
  const void* k_norm;   /* [d] dtype, weights of the keys' norm; NULL: none              */
} retro_rotary;

/* A ragged batch of rows: sequence b has the rows row_start[b] .. row_start[b+1]-1
 * (ascending, row_start[0] >= 0, row_start[batch] <= n_rows; an empty range is a
 * sequence that takes no part), row row_start[b] + j at position start_pos[b] + j.
 * A sequence with start_pos[b] < 0 takes no part.  Rows that belong to no
 * sequence (in front of row_start[0], at or behind row_start[batch]) are not read
 * and their outputs stay as they were, so that a captured call can be replayed
 * for fewer rows.  n_rows: rows that the buffers hold; what reaches past it is cut.
 * longest only helps retro_chunk_attend choose between two kernels that both take any
 * lengths: results are right whatever it says, but where it is unknown every sequence is
 * taken to have a row, and a chunk of a few hundred rows beside as many empty ranges may
 * take two to three times as long. */
typedef struct retro_chunk {
  const int32_t* row_start;  /* [batch + 1] */
  const int32_t* start_pos;  /* [batch]; not the cache's seq_lens array */
  int32_t n_rows;
  int32_t longest;           /* most rows of a sequence, where the host knows; <= 0: unknown */
} retro_chunk;

/* Fills table [positions][rot_dim / 2][2] fp32 with cosine and sine of
 * p * base^(-2 i / rot_dim), computed in fp64 and rounded once.  rot_dim a
 * multiple of 16 in 16 .. 128, base > 0 and finite (RETRO_EINVAL otherwise).  A program
 * whose frequencies are scaled in some other way fills its own table. */
retro_status retro_rotary_table(float* table, int32_t positions, int32_t rot_dim, double base,
                                void* stream);

/* Norm and rotation of the queries and keys of `rows` rows at `positions` [rows]
 * int32: q -> q_out [rows][h_q][d], k -> k_out [rows][h_k][d].  q or k may be NULL
 * (then its output is not looked at).  q_out may be q, and k_out k, where their
 * strides are h_q * d and h_k * d.  A row of negative position is not written; the
 * rotated elements of one at or past rotary->positions become NaN.  positions may
 * be NULL where rot_dim is 0.  rows == 0 does nothing; rows >= 2^31 - 4 is
 * RETRO_EUNSUPPORTED.  E.g. for the window rows of a step: rotated queries for
 * retro_step, rotated keys for retro_update_kv. */
retro_status retro_rotate_qk(const retro_dims* dims, const retro_rotary* rotary,
                             const int32_t* positions, int32_t rows, const void* q,
                             int64_t q_stride, const void* k, int64_t k_stride, void* q_out,
                             void* k_out, void* stream);

/* AppendKV (Alg. 1) of a ragged batch: what retro_append_kv does for row after
 * row of every sequence, with keys normalised and rotated as `rotary` says (and
 * the digests those of the stored keys), and queries likewise into q_out
 * [n_rows][h_q][d] (q NULL: no queries).  start_pos[b] must equal seq_lens[b]
 * for every sequence with rows; seq_lens[b] becomes start_pos[b] + the rows
 * appended, and last_loaded of the pages that receive a key becomes step - 1 for
 * every head (step 0, for a prompt before the first decode step, leaves it at its
 * initial -1).  The first row whose page is not mapped is dropped with every
 * later row of its sequence (slots past the new seq_lens, and digests and last_loaded of
 * pages past it, are then unspecified).  Queries are written for dropped rows
 * too (NaN past rotary->positions); q_out may be q where q_stride is h_q * d.  With rot_dim > 0,
 * rotary->positions must be at least max_pages * P (RETRO_EINVAL).  n_rows == 0 does nothing. */
retro_status retro_append_kv_rotary(const retro_dims* dims, int32_t step,
                                    const retro_kv_cache* cache, const retro_chunk* chunk,
                                    const retro_rotary* rotary, const void* q, int64_t q_stride,
                                    const void* k, int64_t k_stride, const void* v,
                                    int64_t v_stride, void* q_out, void* stream);

/* Bytes of workspace that retro_chunk_attend needs for up to n_rows rows, whatever
 * the lengths.  Zero-fill it once before its first use (the parts of a tile are
 * counted there; a call leaves the counts at zero) and let one call at a time use
 * it; calls of other dims may, one after the other. */
retro_status retro_chunk_workspace_size(const retro_dims* dims, int32_t n_rows, size_t* bytes);

/* Dense causal attention of a ragged batch over the paged cache: row at position
 * p of sequence b, query head g of KV head h, takes every stored token i of the
 * sequence with i <= p and i < seq_lens[b]:
 *   out = sum_i softmax_i(sm_scale q . k_i) v_i,  lse = ln sum_i exp(sm_scale q . k_i)
 * out [n_rows][h_q][d] dtype, lse [n_rows][h_q] fp32 (may be NULL); out may be q where
 * q_stride is h_q * d (RETRO_EINVAL otherwise).  A row that no token is left for gives
 * (0, -inf).  The chunk's own keys and values are stored
 * first (retro_append_kv_rotary, retro_prefill_kv, retro_append_kv_tokens); one row per
 * sequence is dense decoding.  Tokens of pages that are not mapped are left out.
 * Products and sums in fp32; for bf16 the softmax weights are rounded to bf16 for
 * their product with the values (2^-8 of a weight at most), where a sequence has few
 * rows as two bf16 halves (sums and log-normalisers take the unrounded ones).  Which of
 * the two a sequence of more than 32 / G rows gets, and the order of its sums, depend on
 * the call's other sequences too; the same call gives the same bits.
 * NaN and infinities as in retro_decode_attend: a NaN score, or one of +inf,
 * makes its row NaN; a NaN or infinite value of a stored token can make every
 * row of its sequence and KV head in the same call NaN, also rows in front of it;
 * slots past seq_lens never count, whatever they hold.  Reads the cache only.
 * n_rows == 0 does nothing; n_rows * h_q * d >= 2^40 or n_rows * G >= 2^31 - 256
 * is RETRO_EUNSUPPORTED. */
retro_status retro_chunk_attend(const retro_dims* dims, const retro_kv_cache* cache,
                                const retro_chunk* chunk, const void* q, int64_t q_stride,
                                void* out, float* lse, void* workspace, size_t ws_bytes,
                                void* stream);

/* ---- The cache in 4 bits ---------------------------------------------------------
 * With RETRO_FLAG_KV_MX4 in dims->flags a cache's keys and values are held in 4.25 bits
 * an element (the elements and scales of the OCP Microscaling Formats specification's
 * MXFP4), a quarter (1 / 3.8) of bf16's bytes.  With the digests, which stay in dtype, a cache of bf16
 * keys of 128 holds 3.2 times the tokens in the same memory with pages of 16, 3.5 with 32.  A head's
 * vector is cut into blocks of 32 elements.  A block has one exponent byte e and 32 codes: a sign bit and the
 * magnitudes 0, 0.5, 1, 1.5, 2, 3, 4, 6 in the order of the other three bits; an element stands for
 * its code's value times 2^(e - 127), which is exact in bf16.  Storing an element x of dtype (a key
 * as the other format would hold it, normalised, rotated and rounded):
 *   with m the largest magnitude of the block and 2^f <= m < 2^(f + 1),
 *   e = 127 + f - 2 for m < 1.75 * 2^f, one more from there on, cut to 2 .. 252;
 *   the code is the one nearest to x / 2^(e - 127), of two equally near ones that with an
 *   even last bit, and 6 for what lies beyond.
 * A block with a NaN or an infinity gets e = 255: all of it stands for NaN.  (A cache that
 * another program has filled holds no other exponents either; slots past seq_lens may.)
 * k_cache and v_cache are then bytes, [num_phys_pages][h_k][P d / 2 + P d / 32], a page of
 * a KV head being its codes (element 2 i in the low half of a byte, 2 i + 1 in the high
 * one), then its exponents:
 *   keys    codes [P][d], exponents [P][d / 32]
 *   values  codes [P / 4][16][4][d / 16]: of four tokens the 16 parts of the vector in
 *           turn, of a part the tokens in turn; exponents [P / 4][d / 32][4]
 * digest and the queries stay in dtype; a digest holds the minimum and maximum of what the
 * page's keys stand for, so that pages are scored as they will be attended.
 * Every call takes such dims but retro_project_qkv_update and retro_step_attend_partials
 * (RETRO_EUNSUPPORTED), with the semantics that it has for a cache whose keys and values are what
 * the codes stand for; queries, keys and values that it is given, the outputs of attention,
 * k_cache and v_cache have to be 16-byte aligned (RETRO_EINVAL).  retro_step is four or five
 * launches then (the append, the scores, the selection, which is a launch of its own for
 * large tables, the attention, combine + merge; nothing that an earlier call has left in the
 * workspace is read), and retro_chunk_attend takes bf16 rows' weights in tiles of 32 rows (always for sequences of up to
 * 32 / G rows) as two bf16 halves and in tiles of 256 as one, retro_decode_attend and retro_step as three, fp32 rows always as three. */

/* Rows of the cache as keys and values: row j of sequence b, as `chunk` lays them out, is
 * the token at position start_pos[b] + j; k_out, v_out [n_rows][h_k][d] dtype (either may
 * be NULL).  For every format of the cache.  Rows of positions at or past seq_lens[b], or
 * whose page is not mapped, become zeros; rows that belong to no sequence stay as they
 * were.  Reads the cache only.  n_rows == 0 does nothing. */
retro_status retro_read_kv(const retro_dims* dims, const retro_kv_cache* cache,
                           const retro_chunk* chunk, void* k_out, void* v_out, void* stream);

#ifdef __cplusplus
}
#endif

#endif /* RETRO_H */
