/*
 * vlac.h -- C ABI of the VLA-Cache control-step library (CUDA, sm_100a).
 *
 * One control step of a vision-language-action decoder with cross-frame K/V reuse
 * (VLA-Cache, arxiv 2502.02175): choose which vision tokens may keep last step's K/V
 * (Algorithm 1 and Sec. 3.4), run every decoder layer over the remaining positions only
 * (Algorithm 2, Sec. 4.1, Appendix "Inference Detail"), then generate the action tokens.
 *
 * General conventions
 *   - Every pointer named "device" is a raw CUDA device pointer on the current device; "host"
 *     pointers are ordinary host memory.  The library never takes ownership of caller memory.
 *   - Work is enqueued on the CUDA stream passed as `void* stream` (a cudaStream_t; NULL is the
 *     default stream).  Results are valid once the caller has synchronised that stream.
 *   - Every call returns VLAC_OK (0) or a negative VLAC_ERR_* code; nothing throws or aborts.
 *   - A context serves one call at a time; calls on the same context must be stream-ordered.
 *   - The sequence is [n_text_pre text][n_cams*grid*grid vision][n_text_post text]; position p of
 *     sequence b is row b*L+p of a [batch][L][hidden] buffer.  Vision token v (camera c, block
 *     row i, block column j: v = c*grid*grid + i*grid + j) sits at position n_text_pre + v.
 *   - bf16 means the upper 16 bits of an IEEE fp32.
 */
#ifndef VLAC_H_
#define VLAC_H_

#ifdef __cplusplus
extern "C" {
#endif

#define VLAC_OK                0
#define VLAC_ERR_INVALID_ARG  -1
#define VLAC_ERR_BAD_STATE    -2
#define VLAC_ERR_OOM          -3
#define VLAC_ERR_CUDA         -4
#define VLAC_ERR_TIMEOUT      -5
#define VLAC_ERR_TOO_LARGE    -6   /* a size exceeds a fixed capacity stated beside the call */

#define VLAC_MAX_LAYERS 64

typedef struct vlac_ctx   vlac_ctx;    /* configuration, borrowed weight pointers, workspace         */
typedef struct vlac_cache vlac_cache;  /* per-sequence K/V, previous frame, saved attention, selection */

/* Decoder and sequence shape.  n_kv_heads must equal n_heads; head_dim must be 64 or 128 (the
 * tensor-memory kernels take no other), hidden and ffn multiples of 8; n_layers <= VLAC_MAX_LAYERS;
 * patch*3 even; max_batch <= 8. */
typedef struct {
  int n_layers, hidden, n_heads, n_kv_heads, head_dim, ffn, vocab;
  int n_cams, grid, patch;            /* L_v = n_cams*grid*grid; a frame is (grid*patch)^2 RGB8 */
  int n_text_pre, n_text_post;
  int n_action;                       /* action tokens generated per step (the paper uses 7)    */
  float rms_eps, rope_theta;          /* rope_theta is informational: the tables are inputs      */
  int max_batch;
} vlac_config;

/* One layer's weights: device bf16, row-major [out_features][in_features], each matrix 16-byte
 * aligned (they are read through TMA tensor maps); gains [hidden]. */
typedef struct {
  const void *wq, *wk, *wv, *wo, *w_gate, *w_up, *w_down, *g_attn, *g_mlp;
} vlac_layer_w;

/* Whole model.  `layers` is a HOST array of n_layers structs (copied at create); all other
 * pointers are device memory that must outlive the context.  rope_cos/rope_sin are fp32
 * [L + n_action][head_dim/2]: cos/sin(pos * theta^(-2i/head_dim)), rotate-half pairing. */
typedef struct {
  const vlac_layer_w* layers;
  const void *embed;      /* bf16 [vocab][hidden]            */
  const void *proj;       /* bf16 [hidden][hidden], vision feature projector */
  const void *g_final;    /* bf16 [hidden]                   */
  const void *lm_head;    /* bf16 [vocab][hidden]            */
  const float *rope_cos, *rope_sin;
} vlac_weights;

/* Hyper-parameters of Algorithm 1 and Eq. (reuse_ratio).  Paper defaults (Appendix
 * "Experimental Settings"): tau 0.996, top_k 100, tau_task 0.5.
 *   task_mode 0: tau_task is a rank fraction -- the L_v - floor(tau_task*L_v) tokens with the
 *                highest task-relevance score are recomputed;  1: the printed test S >= tau_task.
 *   k_ent:       the k of Eq. (reuse_ratio) (the paper gives no value).
 *   alpha_override: HOST pointer to n_layers doubles replacing the entropy-derived ratios, or NULL.
 *   layer_mask:  bit l set = layer l enters the task-relevance mean (Sec. 3.3 "selected layers");
 *                0 means all layers. */
typedef struct {
  double tau;
  int    top_k;
  double tau_task;
  int    task_mode;
  double k_ent;
  const double* alpha_override;
  unsigned long long layer_mask;
} vlac_select_params;

/* Views into the cache's selection state (device memory owned by the cache; valid until the
 * cache is freed, contents overwritten by the next select/step).
 *   M[b][l]            rows recomputed by layer l of sequence b
 *   rows[b][l][0..M)   their positions, ascending; entries beyond M are unspecified
 *   *_mask[b][v]       1/0 per vision token: P_static (Eq. topk), P_task (Eq. ptask), P_final (Eq. pfinal)
 *   sim[b][v]          Eq. (sim);  S[b][v] task-relevance score (Sec. 3.3)
 *   alpha[b][l]        reuse ratio actually applied (running maximum of Eq. reuse_ratio, or the override) */
typedef struct {
  int batch, n_layers, seq_len, n_vision;
  int* M;
  int* rows;
  unsigned char *static_mask, *task_mask, *final_mask;
  double *sim, *S, *alpha;
} vlac_selection;

/* Which part of a cache vlac_cache_read / vlac_cache_write address. */
#define VLAC_PART_K          0   /* bf16 [max_seq][n_heads][head_dim] of (seq, layer), keys after rotation */
#define VLAC_PART_V          1   /* same layout                                                           */
#define VLAC_PART_PREV_FRAME 2   /* uint8 [n_cams][H][W][3] of seq (layer ignored)                         */
#define VLAC_PART_ATTN_PREV  3   /* fp32 [n_layers][n_heads][L_v] of seq: scores saved by the previous step */
#define VLAC_PART_ATTN_NEXT  4   /* same layout: scores being written by the current prefill               */
#define VLAC_PART_WARM       5   /* int32 [1] of seq: 0 = cold (next select reuses nothing)                */
#define VLAC_PART_PREV_FRAME_BF16 6 /* bf16 [n_cams][H][W][3] of seq: previous frame of vlac_select_bf16   */

/* Create a context.  Copies `cfg` and the layer table, borrows every weight pointer, allocates the
 * workspace for max_batch sequences.  Errors: INVALID_ARG (a shape the kernels do not take, a NULL or
 * a weight matrix that is not 16-byte aligned), OOM, CUDA.
 *
 * Environment switches, read here once per context (off by default):
 *   VLAC_NO_GRAPH=1     vlac_step launches its kernels one by one instead of replaying a captured graph
 *                       (same results; used to profile single kernels)
 *   VLAC_VERBOSE=1      CUDA errors noted by the library are also printed to stderr
 *
 * vlac_destroy releases the context.  Every cache allocated from it must have been freed first:
 * BAD_STATE otherwise, and nothing is released. */
int vlac_create(const vlac_config* cfg, const vlac_weights* w, vlac_ctx** out);
int vlac_destroy(vlac_ctx* ctx);

/* Allocate the persistent state of `batch` (1..max_batch) independent sequences: per layer K/V
 * caches of L + n_action positions (bf16, keys stored after rotation), the previous frame, the
 * text-to-vision attention scores saved by the previous step (Sec. 3.3), and the selection buffers.
 * The cache starts cold.  Library-owned device memory; release with vlac_cache_free. */
int vlac_cache_alloc(vlac_ctx* ctx, int batch, vlac_cache** out);
/* Make sequence `seq` (or all if seq < 0) cold: its next step recomputes every position. */
int vlac_cache_reset(vlac_cache* cache, int seq, void* stream);
int vlac_cache_free(vlac_cache* cache);
/* Copy one part of the cache to / from caller DEVICE memory (device-to-device, stream-ordered).
 * `bytes` must equal the part's size, else INVALID_ARG. */
int vlac_cache_read (vlac_cache* cache, int part, int seq, int layer, void* dst_device, unsigned long long bytes, void* stream);
int vlac_cache_write(vlac_cache* cache, int part, int seq, int layer, const void* src_device, unsigned long long bytes, void* stream);

/* Token selection: Algorithm 1 (patch similarity Eq. sim, threshold + top-k Eq. topk, task
 * relevance Eq. avistext/ptask from the saved scores, eviction Eq. pfinal) followed by the
 * per-layer reuse ratio of Sec. 3.4 / Eq. (reuse_ratio) and the row lists each layer recomputes.
 *   frames: device uint8 [batch][n_cams][H][W][3], the current camera frames (16-byte aligned).
 * A cold sequence gets M = L for every layer.  `out` (may be NULL) receives views of the result.
 * Runs entirely on the device; no host synchronisation. */
int vlac_select(vlac_ctx* ctx, vlac_cache* cache, const unsigned char* frames,
                const vlac_select_params* params, vlac_selection* out, void* stream);

/* The same selection from frames given as bf16 values (normalised pixels, the form a vision encoder takes; the
 * Appendix "Experimental Settings" lowers tau to 0.85 for noisy real-robot frames).  Eq. (sim) is evaluated on those
 * values with fp32 sums in a fixed order, so the similarities are reproducible but not exact: they agree with exact
 * arithmetic to about 1e-6, and a caller who needs index sets that do not depend on the last bits keeps tau and the
 * top-k boundary 1e-5 away from any similarity.  The previous frame is the cache part VLAC_PART_PREV_FRAME_BF16
 * (written by the caller with vlac_cache_write; vlac_step maintains only the byte frame).
 *   frames_bf16: device bf16 [batch][n_cams][H][W][3]. */
int vlac_select_bf16(vlac_ctx* ctx, vlac_cache* cache, const void* frames_bf16,
                     const vlac_select_params* params, vlac_selection* out, void* stream);

/* Install a caller-made selection instead: HOST arrays M[batch][n_layers] and
 * rows[batch][n_layers][L] (ascending positions).  For each sequence the row sets must shrink with
 * depth (rows of layer l+1 a subset of layer l) and contain every text position; INVALID_ARG otherwise. */
int vlac_select_import(vlac_ctx* ctx, vlac_cache* cache, const int* M_host, const int* rows_host, void* stream);

/* One decoder layer over the selected rows only (Algorithm 2; Sec. 4.1; Appendix "Token Reuse
 * Mechanism"): gather the rows of `hidden`, RMSNorm, Q/K/V projection, rotation at the rows' own
 * positions, overwrite those positions of the layer's K/V cache, causal attention of the new
 * queries over all cached positions (fresh and reused), output projection, SwiGLU MLP, both with
 * residual; results are written back to the same rows of `hidden`.  Other rows are untouched.
 * Also records, for the prompt-text queries behind the vision block, the mean attention
 * probability on every vision key (readable as VLAC_PART_ATTN_NEXT).
 *   hidden: device bf16 [batch][L][hidden], updated in place.
 * Uses the selection currently held by the cache (from vlac_select / vlac_select_import);
 * BAD_STATE if there is none. */
int vlac_layer_forward(vlac_ctx* ctx, vlac_cache* cache, int layer, void* hidden, void* stream);

/* One control step for every sequence of the cache: selection (skipped if force_full != 0 or the
 * sequence is cold), input rows (token embeddings; projected vision features), all layers via the
 * partial forward above, greedy first action token from the last prompt position, then
 * n_action - 1 ordinary single-row passes that append K/V behind the prompt (Sec. 3.1).  Finally
 * the frame and the recorded attention become "previous" and the sequences become warm.
 *   frames        device uint8 [batch][n_cams][H][W][3]
 *   vision_feats  device bf16  [batch][L_v][hidden]
 *   prompt_ids    device int32 [batch][n_text_pre + n_text_post]
 *   force_full    1 = recompute every position (the no-reuse step of the same library)
 *   action_tokens device int32 [batch][n_action], ties in the argmax go to the lower id
 *   all_logits    device fp32  [batch][n_action][vocab] or NULL: logits behind each action token
 *   forced_tokens device int32 [batch][n_action] or NULL: tokens to feed back instead of the
 *                 library's own choices (action_tokens still reports the library's choices).
 * Stream behaviour: on an ordinary (created) stream the step is captured once into a CUDA graph and
 * replayed; caller buffers are staged through library buffers around the replay.  On the NULL /
 * legacy default stream, inside a caller's own stream capture, with VLAC_NO_GRAPH=1 or while
 * vlac_profile is on, the ~1300 kernels of a step are launched one by one: same results, but about
 * three times slower at batch 1 (launch gaps, no overlap across kernel boundaries). */
int vlac_step(vlac_ctx* ctx, vlac_cache* cache, const unsigned char* frames, const void* vision_feats,
              const int* prompt_ids, const vlac_select_params* params, int force_full,
              int* action_tokens, float* all_logits, const int* forced_tokens, void* stream);

/* One control step whose action tokens all come from ONE parallel pass (the paper applies the method
 * to OpenVLA-OFT, a decoder that emits its action chunk in one pass: Sec. 5 main LIBERO results and
 * Table 2; it prints no equations for that decoder, so the reading taken is stated here).  Selection, input rows
 * and the partial prefill are those of vlac_step.  Then n_action placeholder rows at positions
 * L .. L+n_action-1, whose input is act_embed[i] for every sequence, go through all layers together:
 * each sees the whole prompt (reused or fresh K/V, as the prefill left it) and every row of the
 * chunk, in both directions.  Their K/V are written behind the prompt and overwritten by the next
 * step.  Token i is the argmax (ties to the lower id) of the logits of row L+i; the prompt's last-row
 * logits are not formed and nothing is fed back.
 *   act_embed     device bf16 [n_action][hidden], caller-owned, must stay alive and unchanged while a
 *                 captured step that read it may be replayed (as for the weights)
 *   action_tokens device int32 [batch][n_action];  all_logits device fp32 [batch][n_action][vocab] or NULL
 * The rows of one sequence's chunk are the columns of the single-row kernels, so n_action <= 8 is
 * required (INVALID_ARG otherwise); sequences of a batch are taken one after the other.  Other
 * arguments, errors and stream behaviour as for vlac_step. */
int vlac_step_chunk(vlac_ctx* ctx, vlac_cache* cache, const unsigned char* frames, const void* vision_feats,
                    const int* prompt_ids, const vlac_select_params* params, int force_full, const void* act_embed,
                    int* action_tokens, float* all_logits, void* stream);

/* Comparison baseline, not part of the method: one control step WITHOUT reuse across frames in which, instead, vision
 * tokens that receive little attention are dropped inside the frame after layer prune_layer - 1 (the FastV row of the
 * paper's Table 2; Sec. 5 "Baselines"; the paper prints no equations for it, the reading is that of the FastV method).
 * Layers 0 .. prune_layer-1 run over the whole sequence.  Each vision token is then scored by the text-to-vision
 * attention it received in layer prune_layer-1 of this step (mean over heads and over the prompt-text queries behind the
 * vision block, the scores of Eq. avistext that every prefill records); the n_keep best stay (ties to the lower
 * index).  From layer prune_layer on the other vision tokens are gone: their rows are not computed and no query attends to
 * their positions, in the prefill and in the single-row passes; kept tokens keep their positions.  prune_layer >= n_layers
 * or n_keep >= L_v gives the plain no-reuse step.  Afterwards vlac_selection_view shows the rows per layer, and the cache
 * is warm as after vlac_step.  prune_layer < 1: INVALID_ARG.  Other arguments and stream behaviour as for vlac_step. */
int vlac_step_pruned(vlac_ctx* ctx, vlac_cache* cache, const unsigned char* frames, const void* vision_feats,
                     const int* prompt_ids, int prune_layer, int n_keep, int* action_tokens, float* all_logits,
                     const int* forced_tokens, void* stream);

/* Views of the selection held by the cache (after select / select_import / step). */
int vlac_selection_view(vlac_cache* cache, vlac_selection* out);

/* Number of kernels the library launched since the context was created (monotonic). */
unsigned long long vlac_launch_count(const vlac_ctx* ctx);

/* Measurement aid (the paper has no counterpart): while enabled, the library brackets every launch of
 * its single-row matrix-vector kernel (the kernel that streams the weights during the action-token
 * passes) with CUDA events on the caller's stream, up to 4096 launches.  vlac_profile(ctx, 1) clears
 * the record and starts; vlac_profile(ctx, 0) stops.  vlac_profile_read waits for the recorded events
 * and returns the summed device time (ms), the summed weight bytes those launches streamed, and their
 * count. */
int vlac_profile(vlac_ctx* ctx, int enable);
int vlac_profile_read(vlac_ctx* ctx, double* ms_total, unsigned long long* bytes_total, int* n_launches);
/* Device time (ms) of the parts of the last step run while profiling was on, in order: selection,
 * input rows, all prefill layers, first action token, then one entry per single-row pass.  Writes at
 * most `cap` entries and their count to *n.  (A profiled step launches its kernels one by one; the
 * graph replay is not used, so the parts include launch gaps the replay does not have.) */
int vlac_profile_segments(vlac_ctx* ctx, double* ms, int cap, int* n);

/* Nonzero if a device-side bounded wait gave up since the context was created (reads one int
 * back; synchronises the stream). */
int vlac_device_error(vlac_ctx* ctx, void* stream);

/* Self-test of the bounded device-side waits (the paper has no counterpart).  Every wait on a
 * shared-memory barrier inside the library's kernels polls against the GPU's wall clock and gives up
 * after a fixed time, recording a code in the context's device error word instead of hanging.  This
 * call runs that same wait, in a one-CTA kernel, on a barrier that nothing ever signals, with a limit
 * of limit_us microseconds (1..100000), then synchronises the stream and returns what
 * vlac_device_error returns: VLAC_ERR_TIMEOUT when the mechanism works.  The error word stays set for
 * the life of the context, so use a context made for the purpose. */
int vlac_selftest_wait_expiry(vlac_ctx* ctx, unsigned int limit_us, void* stream);

/* Greedy token choice that allocates nothing (the paper has no counterpart; it is the last step of
 * vlac_step offered on its own).  For each of `rows` logits rows it returns the index of the largest
 * value, equal values (-0 and +0 are equal) going to the lower index, exactly as vlac_step picks
 * action tokens.
 *
 * It exists for callers that may not allocate device memory at the time of the call: a control loop
 * that reserved its whole memory budget at start-up and must not hit cudaMalloc (or the device-wide
 * synchronisation it implies) afterwards, or a process whose GPU memory belongs to one pool.  It takes
 * no context: its only scratch is a 32 KB array built into the library, which every GPU that loads
 * the library holds until the process exits.  No cudaMalloc/cudaFree or allocating routine is called.
 *
 *   logits      device fp32, row r starts at logits + r*row_stride (row_stride >= vocab, in elements)
 *   rows        1..64; more returns VLAC_ERR_TOO_LARGE and does nothing
 *   tokens      device int32 [rows]
 * The first call on each device looks up the array's device address (one runtime query); make that
 * first call outside any stream capture.  The address is remembered per device ordinal and belongs to
 * the device's primary context: after cudaDeviceReset, or from a context the caller made through the
 * driver API, it is not valid.  All calls share the array and it keeps the previous call's
 * contents; every slot is rewritten before it is read, so nothing needs clearing, but two calls whose
 * kernels overlap on the GPU (different streams, no ordering) race on it: order them. */
int vlac_greedy_tokens_static(const float* logits, int rows, int vocab, long long row_stride,
                              int* tokens, void* stream);

/* ------------------------------------------------------------------------------------------------
 * Paged K/V pool and attention over a shared prefix
 *
 * The cache above holds one dense sequence per control loop.  Several sequences that begin with the same
 * rows -- action candidates sampled from one prompt, several loops under one instruction -- can share those
 * rows in a pool of pages.  The pool is caller-owned device memory described by this struct (no handle, no
 * allocation in the library); its tables are device data, so that every call below can be captured into a
 * CUDA graph and none waits for the device.
 *
 *   k, v    16-bit elements (dtype) [n_layers][n_pages][page_size][n_kv_heads][head_dim], 16-byte aligned,
 *           keys stored after rotation as in the cache
 *   table   int32 [n_slots][max_pages]: the pages of each slot's sequence in order, -1 behind the last
 *   len     int32 [n_slots]: rows held by the slot (0: empty)
 *   refs    int32 [n_pages], 16-byte aligned: slots that hold the page; 0 = free
 *   work    scratch of vlac_pages_work_bytes(p) bytes, 16-byte aligned, contents without meaning between calls
 * A fresh pool has table = -1, len = 0, refs = 0.
 * page_size: a power of two, 8..256.  head_dim: 64 or 128.  n_pages*page_size and max_pages*page_size < 2^31.
 *
 * Rules of all calls below
 *   - Lists (slots, lengths, status) are device int32 arrays of n entries, n <= VLAC_PAGES_MAX_LIST (TOO_LARGE
 *     beyond; n = 0 does nothing).  The call returns INVALID_ARG for what the host can see; what only the
 *     device can see is reported per entry in status[n] (0 or a VLAC_ERR_* code), and an entry that is refused
 *     changes nothing unless stated otherwise.
 *   - status INVALID_ARG: a slot outside [0, n_slots), a target slot that an earlier entry of the list names
 *     (the first stands), a target that another entry reads, a length or position outside its range.
 *     status BAD_STATE: a length or a page number in the slot's own tables outside its range.
 *   - Pages are taken lowest number first, entries in list order; when they do not suffice, an entry and every later
 *     one that needs a page get OOM.  Results depend on the tables alone, never on timing.
 *   - A sequence's last page is never shared while it is partly filled, so rows are appended in place.
 *   - Calls that change a pool, and calls that read it, must be stream-ordered with one another (they share work too). */
#define VLAC_BF16 0
#define VLAC_FP16 1
#define VLAC_PAGES_MAX_LIST 1024
typedef struct {
  void *k, *v;
  int dtype, n_layers, n_pages, page_size, n_kv_heads, head_dim;
  int n_slots, max_pages;
  int *table, *len, *refs;
  void* work;
  unsigned long long work_bytes;
} vlac_pages;

/* Scratch bytes for a pool of this shape (only n_pages, n_slots and max_pages are read); 0 for a NULL or
 * impossible shape. */
unsigned long long vlac_pages_work_bytes(const vlac_pages* p);

/* Give slot seqs[i] the length lens[i] (0..max_pages*page_size): pages are taken behind the last row, or given back from the
 * end (before any are taken); rows that stay keep their pages and contents, new rows are undefined until written.
 * BAD_STATE also for a cut inside a page that another slot holds (vlac_pages_compact with the rows to keep does that). */
int vlac_pages_resize(const vlac_pages* p, const int* seqs, const int* lens, int n, int* status, void* stream);
/* Give all pages of these slots back: resize to 0. */
int vlac_pages_free(const vlac_pages* p, const int* seqs, int n, int* status, void* stream);

/* Make slot dst[i] hold the rows of slot src[i].  deep = 0: the full pages are shared and the rows of a partly filled last
 * page are copied, all layers; deep = 1: every row is copied into pages of its own (rows that a later step overwrites).  A
 * target that holds a sequence gives it back first; after OOM it is left empty.  A source may appear several times; a target
 * must not be the source of any entry. */
int vlac_pages_fork(const vlac_pages* p, const int* src, const int* dst, int n, int deep, int* status, void* stream);

/* Make slot dst[i] hold the rows keep[keep_ptr[i] .. keep_ptr[i+1]) of slot src[i] (positions, strictly ascending,
 * INVALID_ARG otherwise), in that order and without gaps, all layers: pruned tokens leave the cache.  Leading pages that stay
 * whole are shared, the other rows gathered into fresh pages.  dst[i] == src[i] prunes in place (its old pages are given
 * back after the new ones are taken; OOM leaves it as it was); otherwise targets are treated as in vlac_pages_fork.
 *   keep_ptr  device int32 [n + 1], 0 <= keep_ptr[i] <= keep_ptr[i+1] <= n_keep;  keep  device int32 [n_keep] */
int vlac_pages_compact(const vlac_pages* p, const int* src, const int* dst, int n, const int* keep_ptr, const int* keep, int n_keep,
                       int* status, void* stream);

/* Write rows row_ptr[i] .. row_ptr[i+1] of k_rows / v_rows into one layer of slot seqs[i], from position start[i] on
 * (start = NULL: the last rows of the slot).  The positions must lie inside the slot's length (vlac_pages_resize first) and in
 * pages that no other slot holds (BAD_STATE otherwise: vlac_pages_fork with deep = 1).
 *   row_ptr         device int32 [n + 1], 0 <= row_ptr[i] <= row_ptr[i+1] <= rows
 *   k_rows, v_rows  device, the pool's type, row r at r*k_stride / r*v_stride elements (multiples of 8, at least
 *                   n_kv_heads*head_dim), 16-byte aligned; none of the rows of the pool that the call writes */
int vlac_pages_write(const vlac_pages* p, int layer, const int* seqs, const int* start, const int* row_ptr, int n, int rows,
                     const void* k_rows, long long k_stride, const void* v_rows, long long v_stride, int* status, void* stream);

/* Copy positions 0 .. n_rows-1 of sequence seq of a control-step cache into slot `slot`, all layers: the prompt that a step left
 * becomes a prefix that candidates share.  Shapes must agree (bf16 pool of the cache's layers, heads and head_dim, n_rows <= the
 * cache's L + n_action), the slot must already have n_rows rows in pages of its own.  status: device int32 [1]; BAD_STATE also where
 * vlac_step_pruned has dropped one of these positions and no step has recomputed every position of the sequence since (the layers behind the
 * pruning have no row there; vlac_cache_write does not change what counts as dropped). */
int vlac_pages_from_cache(const vlac_pages* p, vlac_cache* cache, int seq, int slot, int n_rows, int* status, void* stream);

/* Attention of new rows over paged sequences, the common prefix read once for all that share it.
 *
 * Row q_ptr[i] + j of q is the j-th of the nq_i = q_ptr[i+1] - q_ptr[i] newest rows of slot seqs[i], at position
 * len - nq_i + j, and sees the positions 0 .. len - nq_i + j of that slot (its own K/V rows are already written).  Query head h
 * reads K/V head h / (n_heads / n_kv_heads).  out = softmax(scale * q K^T) V, lse = log sum exp of the scaled scores (natural
 * logarithm); a row that sees nothing (position < 0) gets zeros and -inf.  Values at positions a row does not see never reach it,
 * infinities and NaN included.
 *
 * vlac_prefix_plan finds, from the tables, which neighbours of the list hold the same leading pages and divides the work; it is
 * called once whenever tables, lengths or q_ptr changed (once per token) and serves the attention of every layer.  Both calls want
 * max_pages*page_size < 2^31 - 1024 (INVALID_ARG otherwise).  List
 * sequences that share most next to one another.  A slot may be listed twice.  Status per entry as above; the rows of a refused
 * entry, and rows behind q_ptr[n], are left as they are.
 *   plan     n (<= VLAC_PAGES_MAX_LIST), rows of q, n_heads (a multiple of n_kv_heads, n_heads*rows < 2^29), and mem: device
 *            memory of vlac_prefix_bytes(p, n, rows, n_heads) bytes, 16-byte aligned, that holds the plan and the partial sums; a plan
 *            is made before its first attention call (or its first 256 bytes are zero: then nothing is computed), with the pool and the
 *            struct that the attention calls get (a call with another table or shape computes nothing, see vlac_prefix_error), and serves
 *            one of them at a time (two captured graphs that may overlap need two)
 *   scale    finite, also times log2(e)
 *   q, out   device, the pool's type, row r at r*q_stride / r*out_stride elements (multiples of 8, at least n_heads*head_dim), 16-byte
 *            aligned;  lse  device fp32 [rows][n_heads] or NULL.  No row of out shares memory with a row of q (queries are still read while results
 *            are written; columns of one buffer are fine), nor with lse or K and V of the pool (INVALID_ARG) */
typedef struct {
  int n, rows, n_heads;
  void* mem;
  unsigned long long bytes;
} vlac_prefix;
unsigned long long vlac_prefix_bytes(const vlac_pages* p, int n, int rows, int n_heads);
int vlac_prefix_plan(const vlac_pages* p, const vlac_prefix* plan, const int* seqs, const int* q_ptr, int* status, void* stream);
int vlac_prefix_attention(const vlac_pages* p, int layer, const vlac_prefix* plan, const void* q, long long q_stride, float scale,
                          void* out, long long out_stride, float* lse, void* stream);
/* VLAC_ERR_TIMEOUT if a device-side bounded wait of an attention call gave up since the plan was made (its output is then not
 * valid), as vlac_device_error does for a context; INVALID_ARG if a call came with another pool or struct than the plan was made with (its
 * output was left as it was).  Reads one int back and synchronises the stream. */
int vlac_prefix_error(const vlac_prefix* plan, void* stream);

/* Self-test of those waits: vlac_prefix_attention whose loads of common pages (more than 16 stacked rows) begin delay_us microseconds late
 * (0..100000) and whose waits give up after limit_us (1..100000).  Where the limit covers the delay and the call's own latencies the results are
 * the ordinary ones; with a longer delay vlac_prefix_error answers TIMEOUT until the next plan, and the output is not valid. */
int vlac_selftest_prefix_wait(const vlac_pages* p, int layer, const vlac_prefix* plan, const void* q, long long q_stride, float scale,
                              void* out, long long out_stride, float* lse, unsigned int delay_us, unsigned int limit_us, void* stream);

/* ------------------------------------------------------------------------------------------------
 * Speculative decoding over the paged pool: a tree of drafted tokens behind each sequence in one pass
 *
 * A token step of a caller's decoder: vlac_pages_resize makes room for the drafted rows, vlac_tree_plan and vlac_prefix_plan look at
 * the trees and tables once; per layer vlac_pages_append rotates the new rows and puts their K and V into the pool and
 * vlac_tree_attention lets each see the sequence and its own ancestors; vlac_logits_adjust applies penalties, biases and the grammar and
 * picks a token for every row; vlac_tree_accept finds the path that the decoder would have taken itself, and vlac_pages_compact drops the
 * other rows.  Nothing waits for the device; the whole step can be captured.  The rules of the paged calls hold here too; an
 * ordinary token is a tree of one row.
 *
 * Rotary tables for any positions, fp32, made in 64 bits (as vlac_weights.rope_cos / rope_sin, and for vlac_pages_append):
 *     f_i = theta^(-2i/rot_dim), i < rot_dim/2;  turns_i = original_len * f_i / (2 pi)
 *     g_i = clamp((turns_i - turns_low) / (turns_high - turns_low), 0, 1), 0 if original_len is 0
 *     cos[p][i] = amplitude * cos((first + p) * f_i * (g_i + (1 - g_i) / factor)),  sin alike
 * factor stretches the positions (1: none): all frequencies alike with original_len = 0, otherwise only those that turn seldom over the
 * length that the weights were trained for (the interpolation by parts of the YaRN paper, arXiv 2309.00071, whose attention temperature is the
 * amplitude; it blends by turns, and the tables of code that blends linearly over the index i between two dimensions cannot be had from this call).
 *   rot_dim  even, 2..256;  theta > 0, factor > 0, original_len >= 0, amplitude finite; turns_low < turns_high where original_len > 0; no frequency
 *            of 65536 turns a position or more (an angle is right to its own size times 2^-59, a g_i between 0 and 1 to
 *            turns_i / (turns_high - turns_low) times that)
 *   first >= 0, n_pos >= 0, first + n_pos <= 2^31 - 1;  cos, sin  device fp32 [n_pos][rot_dim/2] */
typedef struct {
  int rot_dim;
  double theta, factor, original_len, turns_low, turns_high, amplitude;
} vlac_rope_scaling;
int vlac_rope_tables(const vlac_rope_scaling* r, int first, int n_pos, float* cos, float* sin, void* stream);

/* How vlac_pages_append treats a head's query or key before it is stored, in this order and rounded once at the end:
 *   q_gain, k_gain  device [head_dim] of the pool's type, or NULL: x -> x / sqrt(mean(x^2) + eps) * gain over the head's dimensions (16-byte aligned; sums
 *                   in fp32: components beyond 10^18 overflow them, and with eps = 0 a head of none beyond 10^-19 is lost in them; eps >= 0)
 *   rot_dim         0 or a multiple of 16 up to head_dim: the first rot_dim dimensions are rotated, pairs (i, i + rot_dim/2), or with
 *                   interleaved = 1 (2i, 2i + 1):  (x, y) -> (x cos - y sin, x sin + y cos)
 *   cos, sin        device fp32 [n_pos][rot_dim/2], 16-byte aligned (not read with rot_dim = 0) */
typedef struct {
  const float *cos, *sin;
  int n_pos, rot_dim, interleaved;
  const void *q_gain, *k_gain;
  float eps;
} vlac_rope;

/* vlac_pages_write with the norm and rotation of `rope` on the way, for the queries of the same rows too: row r of q goes to row r of
 * q_out, row r of k_rows and v_rows (v as it is) into the pool.
 *   pos    device int32 [rows], the position that row r is rotated to, or NULL: the position it is written to.  An entry with a
 *          position outside [0, n_pos) is refused (INVALID_ARG); without rotation positions are not looked at
 *   q      n_heads heads of head_dim a row (n_heads = 0: none, q and q_out are not looked at); strides and alignment as k_rows.  q_out may be q
 *          itself (same stride); no other row of q_out shares memory with rows of q, k_rows or v_rows, and none with K or V of the pool
 *          (INVALID_ARG).  q, like k_rows and v_rows, none of the rows of the pool that the call writes
 * A row_ptr that falls refuses all.  Other arguments, codes and refusals as vlac_pages_write; rows of refused entries and rows behind row_ptr[n] stay as they were, in q_out too. */
int vlac_pages_append(const vlac_pages* p, int layer, const int* seqs, const int* start, const int* row_ptr, int n, int rows, const vlac_rope* rope,
                      const int* pos, int n_heads, const void* q, long long q_stride, void* q_out, long long q_out_stride, const void* k_rows,
                      long long k_stride, const void* v_rows, long long v_stride, int* status, void* stream);

/* Trees of drafted tokens, one per entry of a list.
 *   q_ptr    device int32 [n + 1]: rows q_ptr[i] .. q_ptr[i+1] (at most max_rows, 1..VLAC_TREE_MAX_ROWS) are the nq_i newest rows of slot seqs[i]
 *   parent   device int32 [rows]: the row's parent within its entry, a row in front of it; -1: none (what it extends is the sequence)
 * and what vlac_tree_plan makes of them (a caller may write mask itself: any bits, of its own rows too; vlac_logits_adjust goes by entry then as well):
 *   mask     device uint32 [rows][ceil(max_rows/32)]: bit j = the row sees row j of its entry (its ancestors and itself)
 *   pos      device int32 [rows]: len - nq_i + depth, the position to rotate to;  entry  device int32 [rows]: the row's entry
 * Status as for the paged calls, INVALID_ARG also for a parent out of range and nq_i > len, TOO_LARGE for nq_i > max_rows; rows of refused
 * entries and of none get mask 0, pos -1, entry -1.  A falling q_ptr refuses all.  p and seqs may both be NULL: pos is then the depth.  mask, pos
 * and entry serve one step at a time (two captured graphs that may overlap need two). */
#define VLAC_TREE_MAX_ROWS 1024
typedef struct {
  int n, rows, max_rows;
  const int *q_ptr, *parent;
  unsigned* mask;
  int *pos, *entry;
} vlac_tree;
int vlac_tree_plan(const vlac_pages* p, const vlac_tree* tree, const int* seqs, int* status, void* stream);

/* vlac_prefix_attention, on the same plan, with the tree's mask among the newest rows: row j of entry i sees the positions in front of
 * len - nq_i and those len - nq_i + b whose bit b is set in its mask (b < nq_i).  tree->n and rows are the plan's; the mask is read, the rest of the
 * tree is not.  An entry that the plan refused keeps its rows of out; one that vlac_tree_plan refused sees only what lies in front of the tree. */
int vlac_tree_attention(const vlac_pages* p, int layer, const vlac_prefix* plan, const vlac_tree* tree, const void* q, long long q_stride, float scale,
                        void* out, long long out_stride, float* lse, void* stream);

/* Logits before a token is picked.  For row r and token t, in this order, fp32, every step rounded once:
 *   made = how often t was generated: in tokens[span[r][1] .. span[r][2]), and (with a tree) among drafted[] of the rows that row r sees in its mask
 *   seen = made > 0 or t in the prompt tokens[span[r][0] .. span[r][1])
 *   x = logits[r][t];  if seen: x = x > 0 ? x / repetition[r] : x * repetition[r]
 *   x = x - frequency[r] * made;  if made: x = x - presence[r];  x = x + bias of t;  x = -infinity where t is not allowed
 * out[r][t] is x in the type of the logits; picked[r] the lowest index of the largest x (before that rounding) among the allowed tokens, a NaN
 * counting as the largest; -1 if none is allowed.
 *   tokens      device int32 [n_tokens] (up to 2^30, n_bias too).  Spans of rows may overlap.  Here, in bias_token and in drafted, numbers outside the
 *               vocabulary are passed over (padding)
 *   span        device int32 [rows][3], or NULL: no history
 *   repetition, frequency, presence   device fp32 [rows], each or NULL (not applied)
 *   bias        entries bias_ptr[r] .. bias_ptr[r+1] of bias_token, bias (int32 [rows + 1], int32 / fp32 [n_bias]) for row r; of several for a token
 *               the last stands; bias_ptr NULL: none
 *   allow       device uint32 [n_allow][ceil(vocab/32)], bit t % 32 of word t / 32: 1 = allowed; allow_row[r] (int32 [rows]) says which one row r
 *               goes by, -1 none; allow_row NULL: row r the r-th (n_allow >= rows).  allow NULL: all tokens are allowed
 *   tree, drafted   the rows are the tree's (tree->rows == rows) and drafted  device int32 [rows] their tokens; both or neither
 * The host refuses what it can see (INVALID_ARG).  status[r]: INVALID_ARG for a span, bias_ptr or allow_row out of range; such a row's out and picked
 * stay as they were. */
#define VLAC_FP32 2
typedef struct {
  const int* tokens; int n_tokens;
  const int* span;
  const float *repetition, *frequency, *presence;
  const int *bias_ptr, *bias_token; const float* bias; int n_bias;
  const unsigned* allow; const int* allow_row; int n_allow;
  const vlac_tree* tree; const int* drafted;
} vlac_logits_rules;
/* logits, out  device, dtype VLAC_FP32, VLAC_BF16 or VLAC_FP16, row r at r*stride / r*out_stride elements (at least vocab; any alignment of the element;
 *              rows of out that lie as their logits do to 16 bytes are faster); out NULL: only tokens are picked; out may be logits itself (same stride), other overlaps are refused
 * picked, status  device int32 [rows]; picked may be NULL.  rows 0..65535 (TOO_LARGE beyond), vocab 1..2^30 */
int vlac_logits_adjust(int rows, int vocab, int dtype, const void* logits, long long stride, const vlac_logits_rules* rules, void* out,
                       long long out_stride, int* picked, int* status, void* stream);

/* The path of each tree that the decoder confirms: from the entry's first row on, to the first child whose drafted token is the token chosen at the
 * row (drafted, chosen  device int32 [rows]; a negative number is no token and confirms nothing).
 *   count   [n]: rows on the path (0 for an empty or refused entry);  path  [rows]: the path's rows within the entry from q_ptr[i] on, -1 behind;
 *   tokens  [rows]: the tokens chosen at them (the last is new), -1 behind
 *   keep_ptr [n + 1], keep [n_keep]: the positions of slot seqs[i] that stay, for vlac_pages_compact (the rows in front of the tree, then the path;
 *           all rows of a refused entry whose slot is sound).  keep_ptr runs on beyond n_keep where the list does not fit: those entries get
 *           TOO_LARGE, and vlac_pages_compact refuses them.  0 <= n_keep < 2^31 - 1
 * Status otherwise as vlac_tree_plan; of the tree only n, rows, max_rows, q_ptr and parent are looked at. */
int vlac_tree_accept(const vlac_pages* p, const vlac_tree* tree, const int* seqs, const int* drafted, const int* chosen, int* count, int* path, int* tokens,
                     int* keep_ptr, int* keep, int n_keep, int* status, void* stream);

const char* vlac_status_string(int status);

#ifdef __cplusplus
}
#endif
#endif  /* VLAC_H_ */
