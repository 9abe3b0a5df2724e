/*
 * hill.h -- C ABI of libhill.so: GB300 (sm_103a) kernels for the per-decode-
 * step token-importance evaluation of HillInfer (arxiv 2602.18750).
 *
 * One decode step of one layer: score the current query against every cached
 * key (Eq. 1, Sec. 2.1), aggregate the scores per token over all query heads
 * (Sec. 4.1 column-sum of attention weights, or the raw inner product of
 * Sec. 4.4), optionally add them to a running per-token importance, select
 * the top-k tokens per sequence (Sec. 3.1, Sec. 4.2), and run the decode
 * attention over the selected tokens only (Sec. 4.1, workflow step 6).
 *
 * Conventions shared by every call
 * --------------------------------
 * - All tensor pointers are DEVICE pointers owned by the caller; the library
 *   never allocates, frees or retains them.  Scratch space comes from the
 *   caller's workspace `ws` (size from hill_workspace_bytes; 16-byte aligned;
 *   its contents need no initialisation and are not preserved between calls).
 * - Calls are asynchronous on `stream` (a cudaStream_t; NULL = legacy default
 *   stream).  A returned HILL_OK means the work was enqueued.  Two calls that
 *   share a workspace must be ordered on the GPU (same stream).
 * - Kernels are launched as programmatic dependents of the previous kernel on
 *   the stream.  Any kernel of a call may read the call's inputs before its
 *   dependency wait -- the scoring calls q, the 16-bit K cache and lens,
 *   hill_topk_select(_bkp) and hill_evict_step_end lens and k,
 *   hill_gather_sparse_attn q -- so those must be complete when the call is
 *   issued in stream order: work that writes them must not be a kernel that
 *   triggers its dependents early (griddepcontrol.launch_dependents) and
 *   writes them afterwards.  Ordinary kernels and copies satisfy this.  What
 *   an earlier call of this library writes (scores, accum, hits, idx, count,
 *   the E4M3 shadow, workspaces) is read after the wait, and outputs and
 *   workspace are written only after it.  The calls that write 16-bit K rows
 *   (hill_cache_insert, hill_cache_read_q4, hill_paged_read, hill_paged_write
 *   into 16-bit pools) do not trigger their dependents early.
 * - Host-side validation failures return immediately and launch nothing.
 *   Launch failures return HILL_ERR_CUDA.  Conditions only visible on the
 *   device (a budget larger than max_k, a selected index outside the cache, a
 *   copy that never completed) set a device error word; hill_sync_status()
 *   reports and clears it.  No kernel traps or spins without a bound.
 * - Layouts (element strides, the head dimension contiguous):
 *     q        [B][H][d]          strides q_sb, q_sh
 *     k_cache  [B][Hkv][cap][d]   strides k_sb, k_sh, k_sn
 *     v_cache  [B][Hkv][cap][d]   strides v_sb, v_sh, v_sn
 *     lens, k, count  [B] int32;  scores, accum  [B][cap] float32 (row = cap);
 *     idx      [B][max_k] int32;  out  [B][H][d] float32, contiguous.
 *   Every stride must be a multiple of 8 elements and q/k/v 16-byte aligned.
 *   Query head h reads KV head h / (H / Hkv) (contiguous grouping).
 * - lens[b] counts the cached tokens of sequence b including the token
 *   generated this step (the caller appends its K/V first); it is clamped to
 *   [0, cap] on the device.  Entries of scores/accum at j >= lens[b] are not
 *   touched.  k[b] is clamped to [0, lens[b]].
 * - Supported: head_dim 128; any H and Hkv with H a multiple of Hkv (MHA,
 *   GQA with any group size G = H / Hkv, MQA); B <= 512; fp16 or bf16 q/K/V;
 *   capacities up to 385024 tokens (the keys that a selection holds on chip).
 *   Groups of more than 8 query heads are scored in passes of at most 8 over
 *   the same keys, except with at most 4 KV heads (MQA-like), where one pass
 *   scores up to 32 query heads of each KV head from every key tile; the
 *   attention takes up to 16 query heads per pass over the gathered rows.
 *   More than 32 KV heads are scored in passes of at most 32 (e.g. 40 KV
 *   heads: two passes of 20), each pass streaming only its own heads' keys.
 */
#ifndef HILL_H_
#define HILL_H_

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef enum {
  HILL_OK = 0,
  HILL_ERR_INVALID_ARG = 1,  /* bad pointer, size, stride or alignment       */
  HILL_ERR_UNSUPPORTED = 2,  /* valid but not built (head_dim, group size)    */
  HILL_ERR_WORKSPACE = 3,    /* ws NULL or smaller than hill_workspace_bytes */
  HILL_ERR_CUDA = 4,         /* a CUDA runtime call or launch failed          */
  HILL_ERR_TIMEOUT = 5,      /* a bounded device wait expired (device word)   */
  HILL_ERR_DEVICE = 6        /* a device-side argument check fired (device word) */
} hill_status;

typedef enum { HILL_F16 = 0, HILL_BF16 = 1 } hill_dtype;

/* Importance rule.  ATTN (the paper's definition, Sec. 4.1): per (b, h) the
 * softmax of z = q.K/sqrt(d) over j < lens[b], summed over all H query heads.
 * RAW (Sec. 4.4 "Algorithmic Simplification"): the sum over heads of z itself
 * (no softmax); the 1/sqrt(d) scale is kept. */
typedef enum { HILL_SCORE_ATTN = 0, HILL_SCORE_RAW = 1 } hill_score_mode;

typedef struct {
  int32_t batch;         /* B  >= 0                                   */
  int32_t num_q_heads;   /* H  >= 1                                   */
  int32_t num_kv_heads;  /* Hkv >= 1, H % Hkv == 0                    */
  int32_t head_dim;      /* d (128)                                   */
  int32_t capacity;      /* cap: allocated tokens per (b, kv head)    */
  int32_t dtype;         /* hill_dtype of q, K and V                  */
  int64_t q_sb, q_sh;             /* element strides of q             */
  int64_t k_sb, k_sh, k_sn;       /* element strides of k_cache       */
  int64_t v_sb, v_sh, v_sn;       /* element strides of v_cache       */
} hill_desc;

/* Bytes of workspace that any call below needs for this descriptor, mode and
 * index width (the maximum over the four calls).  Returns 0 for an invalid
 * descriptor.  Queries the current device's SM count. */
size_t hill_workspace_bytes(const hill_desc* desc, hill_score_mode mode, int32_t max_k);

/* Per-token importance (Eq. 1 with Sec. 4.1 or Sec. 4.4):
 *   ATTN: scores[b][j] = sum_h softmax_{j'<lens[b]}(q_h . K_{g(h),j'} / sqrt(d))[j]
 *   RAW : scores[b][j] = sum_h q_h . K_{g(h),j} / sqrt(d)
 * for j < lens[b].  If accum != NULL it is also updated: accum[b][j] +=
 * scores[b][j] (running importance across decode steps; a newly appended
 * token must hold 0 in accum before its first step).  scores is required. */
hill_status hill_score(const hill_desc* desc, const void* q, const void* k_cache,
                       const int32_t* lens, hill_score_mode mode, float* scores,
                       float* accum, void* ws, size_t ws_bytes, void* stream);

/* Top-k selection (Sec. 3.1 top-alpha retention, Sec. 4.2 global top-alpha):
 * for each b, the first n_b = min(k[b], lens[b]) tokens j < lens[b] in the
 * order (scores[b][j] descending, j ascending) -- a lower index wins a tie --
 * written to idx[b][0..n_b) in ascending index order, idx[b][n_b..max_k) =
 * -1, count[b] = n_b.  If n_b > max_k, count[b] = max_k and the device error
 * word records HILL_ERR_DEVICE.  -0.0 ranks equal to +0.0; keys must be
 * finite. */
hill_status hill_topk_select(const hill_desc* desc, const float* scores, const int32_t* lens,
                             const int32_t* k, int32_t max_k, int32_t* idx, int32_t* count,
                             void* ws, size_t ws_bytes, void* stream);

/* Decode attention over the selected tokens only (Sec. 4.1, workflow step 6; Eq. 1
 * restricted to the selected set, softmax renormalised over it):
 *   out[b][h][:] = sum_{t<count[b]} p_t V[b][g(h)][idx[b][t]][:],
 *   p = softmax_t(q_h . K[b][g(h)][idx[b][t]] / sqrt(d)).
 * count[b] == 0 gives zeros.  count[b] is clamped to [0, max_k]; an index
 * outside [0, cap) is skipped and recorded as HILL_ERR_DEVICE. */
hill_status hill_gather_sparse_attn(const hill_desc* desc, const void* q, const void* k_cache,
                                    const void* v_cache, const int32_t* idx, const int32_t* count,
                                    int32_t max_k, float* out, void* ws, size_t ws_bytes,
                                    void* stream);

/* The whole step for one layer, in the order of the evaluation workflow of
 * Sec. 4.1 (steps 4-6: score the cached keys against the current query,
 * keep the top-alpha critical tokens, attend over those only): hill_score,
 * then hill_topk_select on accum (if given) else on this step's scores, then
 * (if out != NULL) hill_gather_sparse_attn over the selection.  scores may be
 * NULL (then the step's scores live in the workspace).  Results equal those
 * of the three separate calls. */
hill_status hill_evict_step(const hill_desc* desc, const void* q, const void* k_cache,
                            const void* v_cache, const int32_t* lens, const int32_t* k,
                            int32_t max_k, hill_score_mode mode, float* accum, float* scores,
                            int32_t* idx, int32_t* count, float* out, void* ws,
                            size_t ws_bytes, void* stream);

/* BKP bookkeeping (Sec. 4.2, Bidirectional KV Cache Pools), applied to the
 * kept set of one HBM tier.  Two metrics decide which tokens stay:
 *  - temporal-aware pinning: the W = min(recent, lens[b]) most recent tokens
 *    [lens[b] - W, lens[b]) are always kept;
 *  - the older tokens [0, lens[b] - W) are ranked as in hill_topk_select and
 *    the first min(k[b], lens[b] - W) of them are kept;
 *  - frequency-aware tracking: hits (nullable, [B][cap] uint16, caller-
 *    owned and persistent across steps; the paper's 2-byte-per-token hit-rate
 *    table) gains +1, saturating at 65535, at every kept token.
 * idx[b] lists the kept tokens in ascending order (the window last), count[b]
 * = kept tokens.  If the window plus the ranked tokens exceed max_k, the
 * window keeps its max_k most recent tokens, the ranked part gets what is
 * left, and HILL_ERR_DEVICE is recorded.  recent < 0 is HILL_ERR_INVALID_ARG;
 * recent = 0 with hits = NULL is exactly hill_topk_select. */
hill_status hill_topk_select_bkp(const hill_desc* desc, const float* scores, const int32_t* lens,
                                 const int32_t* k, int32_t recent, int32_t max_k, int32_t* idx,
                                 int32_t* count, uint16_t* hits, void* ws, size_t ws_bytes,
                                 void* stream);

/* hill_evict_step with the BKP selection of hill_topk_select_bkp in place of
 * the plain top-k (same other arguments; recent = 0 with hits = NULL is
 * exactly hill_evict_step). */
hill_status hill_evict_step_bkp(const hill_desc* desc, const void* q, const void* k_cache,
                                const void* v_cache, const int32_t* lens, const int32_t* k,
                                int32_t recent, int32_t max_k, hill_score_mode mode, float* accum,
                                float* scores, int32_t* idx, int32_t* count, uint16_t* hits, float* out,
                                void* ws, size_t ws_bytes, void* stream);

/* The same step in two calls, for the layer-pipelined evaluation of Sec. 4.3
 * (the evaluation of layer i + 1 overlaps the rest of layer i): while the
 * normalisation and selection of one layer run on a second stream, the K
 * stream of the next layer proceeds on the first.
 *
 * hill_evict_step_begin launches the scoring kernel: it streams the K cache
 * once and writes, in ATTN mode, the logits and per-CTA softmax partials into
 * the workspace, in RAW mode the per-token sums into scores (and accum +=).
 * It reads q, k_cache and lens.
 *
 * hill_evict_step_end completes the step from the workspace: in ATTN mode the
 * normalisation (scores, accum += as in hill_score), then the top-k selection
 * of hill_topk_select_bkp (recent = 0 and hits = NULL: exactly
 * hill_topk_select) on accum if given, else on this step's scores.  It reads
 * no keys.  Its kernels run beside a scoring kernel of another layer: the
 * normalisation's finalize fits next to a scoring CTA on one SM, and the
 * selection uses the SMs the scoring grid of begin leaves free.
 *
 * Both calls of one step take the same desc, lens, max_k, mode, accum,
 * scores and ws (sized by hill_workspace_bytes); end may be issued on another
 * stream than begin, after an event recorded behind begin.  The workspace
 * belongs to the step from begin until end has completed: a pipeline over
 * layers rotates n >= 2 workspaces and issues begin of layer l + n only after
 * end of layer l.  One workspace per layer leaves the K stream without any
 * wait inside a decode step (fastest); two or three bound the memory.  The
 * scoring kernel of begin takes 17/20 of the SMs, so that end's kernels have
 * room beside it.  Results equal those of
 * hill_evict_step_bkp without attention, the ATTN scores within rounding (the
 * smaller scoring grid and the two-kernel normalisation combine the softmax
 * partials in another order); the selection follows the same rule on the
 * step's own scores.  Attention: hill_gather_sparse_attn on idx and count
 * afterwards. */
hill_status hill_evict_step_begin(const hill_desc* desc, const void* q, const void* k_cache,
                                  const int32_t* lens, int32_t max_k, hill_score_mode mode, float* accum,
                                  float* scores, void* ws, size_t ws_bytes, void* stream);
/* hill_evict_step_begin with the keys scored from their E4M3 shadow (k8,
 * kscale as in hill_score_f8 below): the split form of hill_evict_step_f8's
 * evaluation, completed by hill_evict_step_end in the same way. */
hill_status hill_evict_step_begin_f8(const hill_desc* desc, const void* q, const uint8_t* k8, const float* kscale,
                                     const int32_t* lens, int32_t max_k, hill_score_mode mode, float* accum,
                                     float* scores, void* ws, size_t ws_bytes, void* stream);
hill_status hill_evict_step_end(const hill_desc* desc, const int32_t* lens, const int32_t* k, int32_t recent,
                                int32_t max_k, hill_score_mode mode, float* accum, float* scores,
                                int32_t* idx, int32_t* count, uint16_t* hits, void* ws, size_t ws_bytes,
                                void* stream);

/* Per-KV-head selection (a variant of the evaluation: the paper evaluates at
 * token level for every head topology, Sec. 5.3; here each KV head keeps its
 * own set).  The importance is aggregated over the G query heads of each KV
 * head only,
 *   ATTN: s[b][g][j] = sum_{h in group g} softmax_{j'<lens[b]}(z[b,h,j'])[j]
 *   RAW : s[b][g][j] = sum_{h in group g} z[b,h,j],
 * written to scores [B][Hkv][cap] (caller-owned, required unless accum
 * [B][Hkv][cap] is given; then accum += s and the ranking uses accum).  The
 * top min(k[b], lens[b]) tokens of every (b, g) go to idx [B][Hkv][max_k]
 * (ascending, -1 padded) and count [B][Hkv], and if out != NULL the query
 * heads of KV head g attend over idx[b][g] only.  B * Hkv <= 512. */
hill_status hill_evict_step_kvh(const hill_desc* desc, const void* q, const void* k_cache,
                                const void* v_cache, const int32_t* lens, const int32_t* k, int32_t max_k,
                                hill_score_mode mode, float* accum, float* scores, int32_t* idx,
                                int32_t* count, float* out, void* ws, size_t ws_bytes, void* stream);

/* Asymmetric-precision scoring (Sec. 4.4, CEC): the evaluation ranks tokens
 * with low-precision inner products, while the attention keeps the original
 * 16-bit keys and values.  On this GPU the low precision is OCP FP8 E4M3
 * (its tensor-core rate is ~14x that of INT8 here), one scale per key row:
 *   k8     [B][Hkv][cap][128] uint8 E4M3 codes, dense, 16-byte aligned;
 *   kscale [B][Hkv][cap32] float32, cap32 = cap rounded up to 32, dense.
 * A row's codes are e4m3(K_i * (448 / amax)) with amax = max_i |K_i| (float32
 * product, round to nearest even, saturating) and its scale is amax / 448.
 * The query is cast the same way per (b, h) inside the scoring kernel, and
 *   z8 = (sum_i e4m3(q)_i e4m3(K)_i) * s_q * s_k / sqrt(d)
 * replaces the logit of Eq. 1 in the importance (ATTN or RAW, as hill_score).
 *
 * hill_quantize_k writes the shadow of rows [row_begin[b], row_end[b]) of
 * every KV head (device arrays [B], clamped to [0, cap]); max_rows bounds
 * row_end - row_begin over b (e.g. 1 to add this step's token, cap to build
 * the whole shadow). */
hill_status hill_quantize_k(const hill_desc* desc, const void* k_cache, const int32_t* row_begin,
                            const int32_t* row_end, int32_t max_rows, uint8_t* k8, float* kscale,
                            void* stream);

/* hill_score on the E4M3 shadow (same outputs and workspace as hill_score). */
hill_status hill_score_f8(const hill_desc* desc, const void* q, const uint8_t* k8, const float* kscale,
                          const int32_t* lens, hill_score_mode mode, float* scores, float* accum,
                          void* ws, size_t ws_bytes, void* stream);

/* hill_evict_step with the scoring on the E4M3 shadow; the sparse attention
 * (out != NULL) reads the original k_cache and v_cache.  k_cache and v_cache
 * may be NULL when out is NULL. */
hill_status hill_evict_step_f8(const hill_desc* desc, const void* q, const uint8_t* k8, const float* kscale,
                               const void* k_cache, const void* v_cache, const int32_t* lens,
                               const int32_t* k, int32_t max_k, hill_score_mode mode, float* accum,
                               float* scores, int32_t* idx, int32_t* count, float* out, void* ws,
                               size_t ws_bytes, void* stream);

/* Synchronises `stream`, then returns and clears the device error word of the
 * current device: HILL_ERR_TIMEOUT if a bounded wait expired, HILL_ERR_DEVICE
 * if a device-side argument check fired, HILL_ERR_CUDA if the synchronisation
 * itself failed, else HILL_OK. */
hill_status hill_sync_status(void* stream);

/* Static, human-readable name of a status. */
const char* hill_status_string(hill_status status);

/* Largest scratch, in bytes, that hill_score_noalloc may use: 16 MiB. */
#define HILL_SCORE_NOALLOC_MAX_SCRATCH (16u << 20)

/* hill_score for callers that cannot allocate device memory.  (The paper
 * has no counterpart; this is a deployment convenience.)  Some callers have
 * no way to obtain a workspace: a plug-in running inside a host application
 * that owns the whole device-memory budget and forbids its own cudaMalloc, a
 * latency-critical decode loop where an allocation could block or fail at an
 * unpredictable moment, or a binding from a language without a CUDA
 * allocator.  This entry point takes the same arguments as hill_score minus
 * the workspace and computes exactly what hill_score computes; its scratch is
 * a fixed HILL_SCORE_NOALLOC_MAX_SCRATCH-byte array built into the library,
 * which every GPU that loads the library holds until the process exits.
 *  - It allocates nothing: no cudaMalloc, cudaFree or allocating library call.
 *  - The first call on each device looks up that array's device address
 *    (cudaGetSymbolAddress, no allocation); make that first call on a device
 *    before any stream capture.
 *  - A call needing more scratch than the array holds returns
 *    HILL_ERR_WORKSPACE without launching anything.  ATTN mode needs
 *    4*B*H*cap bytes of logits, 8*B*H*P bytes of softmax partials and
 *    8*B*H bytes of statistics, each rounded up to 256 bytes; P = min(SMs,
 *    B * ceil(cap / 32)) * W partial slots, W = 8 / Hkv rounded down when
 *    Hkv <= 4 and H / Hkv >= 5, else 1 (SMs = the device's multiprocessor
 *    count).  RAW mode needs none.
 *  - All calls share the array, and it keeps whatever the last call left;
 *    no entry of it needs to start at zero (a call reads only what it wrote).
 *    Calls that overlap on the GPU (two streams, or two host threads without
 *    ordering) race on it: order them on one stream. */
hill_status hill_score_noalloc(const hill_desc* desc, const void* q, const void* k_cache,
                               const int32_t* lens, hill_score_mode mode, float* scores,
                               float* accum, void* stream);

/* ---------------------------------------------------------------------------
 * A cache of bounded size.  The calls above leave every token in the cache
 * and pass a kept set along; a program that evicts for good keeps a cache of
 * `cap` slots instead, whose slots are taken again by accumulated attention
 * weight (the importance of Sec. 4.1, summed over the steps).  Per decode
 * step and layer: hill_cache_insert puts the new token in, then
 * hill_window_attn attends over what is held and adds the step's weights to
 * accum.  Both have a form for a cache held in 4 bits.
 *
 * State, caller-owned, per row = per sequence, or with kvh != 0 per
 * (sequence, KV head), each KV head then keeping tokens of its own:
 *   seen   [B] or [B][Hkv] int32         tokens inserted so far, 0 at first; the
 *                                        row holds min(seen, cap) tokens, in the
 *                                        slots from 0 on
 *   pos    [B][cap] or [B][Hkv][cap] int32     the position (0-based count of the
 *                                        sequence's tokens) that a slot holds
 *   accum  [B][cap] or [B][Hkv][cap] float32   the slot's accumulated weight
 * seen serves as `lens` of the attention: lens is clamped to [0, cap].
 *
 * 4-bit caches: a row of d = 128 channels is 64 bytes of codes (byte i:
 * channel 2i in the low half, 2i + 1 in the high half) with a scale and a
 * minimum in desc's 16-bit type, value = min + scale * code:
 *   k4, v4  [B][Hkv][cap][64] uint8, dense, 16-byte aligned;
 *   params  [B][Hkv][cap32][4] 16-bit (K scale, K min, V scale, V min), cap32 =
 *           cap rounded up to 32, dense, 16-byte aligned.
 * Finite rows give scale = (max - min) / 15 rounded to the 16-bit type and
 * code = (x - min) / scale rounded to nearest even, clamped to [0, 15] (0 when
 * the scale rounds to 0).  A row with a NaN or an infinity, or whose max - min
 * float32 does not hold, stands for no finite value.  desc gives the sizes and the type; its K and V
 * strides are not used for 4-bit caches.
 *
 * These calls read all their inputs after the dependency wait (see above). */

/* Bytes of workspace of hill_window_attn and hill_window_attn_q4, with or
 * without an accum.  Returns 0 for an invalid descriptor. */
size_t hill_window_workspace_bytes(const hill_desc* desc, int32_t with_accum);

/* Decode attention over the visible part of the cache: of the n = lens[row]
 * tokens held (clamped to [0, cap]) the first `sinks` slots and the newest
 * `window`, slots j < n with j < sinks or j >= n - window (Eq. 1 restricted to
 * them):
 *   out[b][h] = sum_j p_j V[b][g(h)][j],  p = softmax_j(q_h . K[b][g(h)][j] / sqrt(d)).
 * A window of cap or more shows everything; with nothing visible the output
 * is zero.  sinks and window count slots, so they are for caches in order of
 * position (ones that have not evicted).  If accum is given, accum[row][j] +=
 * sum of p_j over the row's query heads, for visible j only.
 * lens and accum: [B] and [B][cap], kvh != 0: [B][Hkv] and [B][Hkv][cap] (B * Hkv
 * <= 2048).  What lies in slots that are not visible does not matter, NaN
 * included; a query, key or value that is seen and not finite leaves the
 * outputs (and weights) that it enters not finite, as the formula has it.
 * Logits and sums are float32.  A weight meets V as the sum of two numbers of
 * the cache's type: in bf16 it is off by at most 2^-16 of itself, in fp16 by
 * 2^-22 of itself and 2^-32 of the head's largest weight.
 * q, K, V as in the calls above; out 16-byte aligned. */
hill_status hill_window_attn(const hill_desc* desc, const void* q, const void* k_cache, const void* v_cache,
                             const int32_t* lens, int32_t sinks, int32_t window, int32_t kvh, float* accum,
                             float* out, void* ws, size_t ws_bytes, void* stream);

/* hill_window_attn over a 4-bit cache: K and V are the values that the rows
 * stand for (not rounded to 16 bits).  A token's weight times its V scale is
 * off by at most 2^-21 of itself and 2^-32 of the head's largest such product.
 * Scales are at least 0; with scales and minima up to 2^90 no sum overflows. */
hill_status hill_window_attn_q4(const hill_desc* desc, const void* q, const uint8_t* k4, const uint8_t* v4,
                                const void* params, const int32_t* lens, int32_t sinks, int32_t window, int32_t kvh,
                                float* accum, float* out, void* ws, size_t ws_bytes, void* stream);

/* New tokens of every sequence, in order of position. */
typedef struct {
  const void* k;              /* [B][Hkv][max_new][d] in desc's type          */
  const void* v;              /* the same                                     */
  int64_t k_sb, k_sh, k_sn;   /* element strides, multiples of 8; d contiguous */
  int64_t v_sb, v_sh, v_sn;
  int32_t max_new;            /* new tokens per sequence, at most             */
  const int32_t* count;       /* [B] how many of them (clamped), or NULL: all */
  const float* weight;        /* [B][max_new] (kvh: [B][Hkv][max_new]) their
                                 first accumulated weights, or NULL: 0        */
} hill_new_rows;

/* Inserts the new tokens: token i of a row gets position seen[row] + i and a
 * slot, its rows are written there for the row's KV heads, pos and accum of
 * the slot are set, and seen[row] grows by the number of new tokens.
 * While slots are free, tokens take them in order.  The e tokens that find none
 * take, in ascending order, the slots that are given up: among the held slots
 * with a position p, sinks <= p < seen + new - recent (seen before the call),
 * the last e in the order (accum descending, slot ascending).  So the first
 * `sinks` tokens of the sequence and the `recent` newest, the new ones among
 * them, stay.  slots [B][max_new] (kvh: [B][Hkv][max_new]) receives every new
 * token's slot, -1 past a sequence's own.
 * sinks + max(recent, max_new) must not exceed cap.  If pos names fewer slots
 * that may go than are needed (positions that no insert made), none of them is
 * given up: the tokens that found no free slot are dropped (slot -1) and
 * HILL_ERR_DEVICE is recorded.  -0.0 ranks
 * equal to +0.0; weights must be finite. */
hill_status hill_cache_insert(const hill_desc* desc, const hill_new_rows* rows, void* k_cache, void* v_cache,
                              int32_t* seen, int32_t* pos, float* accum, int32_t sinks, int32_t recent, int32_t kvh,
                              int32_t* slots, void* stream);

/* hill_cache_insert into a 4-bit cache. */
hill_status hill_cache_insert_q4(const hill_desc* desc, const hill_new_rows* rows, uint8_t* k4, uint8_t* v4,
                                 void* params, int32_t* seen, int32_t* pos, float* accum, int32_t sinks,
                                 int32_t recent, int32_t kvh, int32_t* slots, void* stream);

/* The values of slots [row_begin[b], row_end[b]) of every KV head of a 4-bit
 * cache, rounded to desc's type, into 16-bit caches of desc's strides (for the
 * calls that read those); max_rows bounds row_end - row_begin over b. */
hill_status hill_cache_read_q4(const hill_desc* desc, const uint8_t* k4, const uint8_t* v4, const void* params,
                               const int32_t* row_begin, const int32_t* row_end, int32_t max_rows, void* k_cache,
                               void* v_cache, void* stream);

/* ---------------------------------------------------------------------------
 * Prompts.  Before the decode steps a program runs its prompts through the same
 * cache: attention of all their queries, and the importance (Sec. 4.1) that
 * their tokens start with.  Rows of several sequences are packed: sequence b has
 * the query rows [q_start[b], q_start[b+1]) of q and the key rows [k_start[b],
 * k_start[b+1]) of k and v (device arrays [B + 1], int32, ascending).  With n
 * queries and m keys, query i of a sequence is at position i + m - n: the keys
 * before its prompt are its context, and a query sees key j where
 *   j <= pos  and  (j < sinks or j > pos - window).
 * Rows that belong to no sequence are neither read into a result nor written;
 * offsets that descend or leave the tensors are clamped and recorded as
 * HILL_ERR_DEVICE.
 *     q [q_rows][H][d], k and v [k_rows][Hkv][d], strides *_st (row), *_sh (head)
 * in elements, multiples of 8; 16-byte aligned; d contiguous.  At most 2^30 rows, 512 sequences.
 * (A stride of 0, of rows or heads that are one and the same, is HILL_ERR_UNSUPPORTED.)
 * These calls read all their inputs after the dependency wait (see above). */
typedef struct {
  int32_t batch;         /* B >= 0, at most 512                       */
  int32_t num_q_heads;   /* H >= 1                                    */
  int32_t num_kv_heads;  /* Hkv >= 1, H % Hkv == 0                    */
  int32_t head_dim;      /* d (128)                                   */
  int32_t dtype;         /* hill_dtype of q, k, v and out             */
  int32_t q_rows, k_rows;
  int64_t q_st, q_sh, k_st, k_sh, v_st, v_sh;
} hill_packed;

/* Attention of every query over the keys that it sees (Eq. 1):
 *   out[i][h] = sum_j p_ij v_j,  p_ij = exp(z_ij - lse[i][h]),
 *   z_ij = q_i . k_j / sqrt(d),  lse[i][h] = ln sum_j exp(z_ij).
 * out [q_rows][H][d] in desc's type, dense, 16-byte aligned; lse [q_rows][H]
 * float32, dense, or NULL.  A query that sees nothing has zeros and -infinity.  What lies in keys and
 * values that a query does not see does not matter to it, NaN included.
 * Logits, sums and outputs are held in float32; a weight meets v rounded to the
 * type of v (half a step of that type), and the output is rounded once. */
hill_status hill_prompt_attn(const hill_packed* desc, const void* q, const void* k, const void* v,
                             const int32_t* q_start, const int32_t* k_start, int32_t sinks, int32_t window,
                             void* out, float* lse, void* stream);

/* Bytes of workspace of hill_prompt_importance.  Returns 0 for an invalid descriptor. */
size_t hill_prompt_workspace_bytes(const hill_packed* desc);

/* The weights of those queries summed for each key, added to a running importance:
 *   accum[b][j] += sum_h sum_i exp(z_ij - lse[i][h])
 * over the `newest` last queries of sequence b (all, if it has no more) that
 * see key j.  lse is that of hill_prompt_attn.  accum [B][cap] (kvh: [B][Hkv][cap], each KV
 * head the sum over its own query heads), float32, dense.  Keys past cap are left out
 * and recorded as HILL_ERR_DEVICE.  Sums are float32, in a fixed order. */
hill_status hill_prompt_importance(const hill_packed* desc, const void* q, const void* k, const float* lse,
                                   const int32_t* q_start, const int32_t* k_start, int32_t sinks, int32_t window,
                                   int32_t newest, int32_t kvh, float* accum, int32_t cap, void* ws,
                                   size_t ws_bytes, void* stream);

/* ---------------------------------------------------------------------------
 * A cache in pages.  Position p of sequence b lies in page table[b][p / page],
 * slot p % page of the pools
 *   k, v    [pages][Hkv][page][d], dense, 16-byte aligned, in desc's type, or (scales
 *           given) as E4M3 codes, one byte each;
 *   scales  [pages][Hkv][page][2] float32 (K scale, V scale), dense, 16-byte aligned, or NULL.
 * A row of codes is e4m3(x * (448 * (1 / amax))) with amax = max |x|, its scale amax * (1 / 448)
 * (float32 steps, round to nearest even), and it stands for code * scale; rows with amax below
 * 2^-119 stand for zeros.  `page` is a multiple of 16; table [B][cols] covers cols * page
 * positions.  A page number outside [0, pages) stands for nothing: entries of
 * positions that a call does not touch may hold any; one that it
 * touches is recorded as HILL_ERR_DEVICE, reads as zeros and is not written.
 * These calls read all their inputs after the dependency wait (see above). */
typedef struct {
  void* k;
  void* v;
  float* scales;
  const int32_t* table;
  int32_t pages, page, cols;
} hill_pages;

/* hill_window_attn over a cache in pages: the same visible positions, outputs,
 * importance and workspace (hill_window_workspace_bytes).  desc->capacity =
 * cols * page; its K and V strides are not used.  E4M3: K and V are the values that the rows stand for; a
 * token's weight times its V scale is off by at most 2^-21 of itself and 2^-32
 * of the head's largest such product. */
hill_status hill_paged_attn(const hill_desc* desc, const void* q, const hill_pages* pages, const int32_t* lens,
                            int32_t sinks, int32_t window, int32_t kvh, float* accum, float* out, void* ws,
                            size_t ws_bytes, void* stream);

/* New rows of several sequences, packed: [rows][Hkv][d] in desc's type, strides in
 * elements, multiples of 8; 16-byte aligned; d contiguous. */
typedef struct {
  const void* k;
  const void* v;
  int64_t k_st, k_sh, v_st, v_sh;
  int32_t rows;
} hill_rows;

/* New rows into their pages, quantised where the pools hold codes: row t of sequence b
 * (starts[b] <= t < starts[b+1], device array [B + 1]) becomes position begin[b] + t - starts[b].
 * Rows before the first sequence or behind the last go nowhere.  Positions below 0 or past the
 * table are dropped and recorded as HILL_ERR_DEVICE.  No two rows of a call may
 * have the same place.  desc gives batch, num_kv_heads and dtype. */
hill_status hill_paged_write(const hill_desc* desc, const hill_pages* pages, const hill_rows* rows,
                             const int32_t* starts, const int32_t* begin, void* stream);

/* Positions [row_begin[b], row_end[b]) (clamped to the table and to desc's capacity) of every KV
 * head into 16-bit caches of desc's strides, for the calls that read those: copied, or
 * code * scale rounded to desc's type.  max_rows bounds row_end - row_begin over b.  (A stride
 * of 0, of rows that would lie in one place, is HILL_ERR_INVALID_ARG.) */
hill_status hill_paged_read(const hill_desc* desc, const hill_pages* pages, const int32_t* row_begin,
                            const int32_t* row_end, int32_t max_rows, void* k_cache, void* v_cache, void* stream);

/* Number of kernels this library has launched (or recorded into a CUDA graph
 * under stream capture) in this process so far, over all devices.  Lets a
 * caller count the kernels one call or one captured graph contains. */
uint64_t hill_kernel_launches(void);

/* Self-test of the bounded waits every kernel uses (no counterpart in the
 * paper): launches one warp that waits on a barrier nothing will complete,
 * for limit_us microseconds (1 .. 1e6), then gives up.  The wait expiring is
 * recorded like any other: the next hill_sync_status() returns
 * HILL_ERR_TIMEOUT, and the stream and context stay usable. */
hill_status hill_selftest_wait(uint32_t limit_us, void* stream);

/* ABI version of this header (major * 100 + minor). */
int32_t hill_abi_version(void);

#ifdef __cplusplus
}
#endif

#endif /* HILL_H_ */
