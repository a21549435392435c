/*
 * specvocab.h -- C ABI of the SpecVocab draft-step library for AMD MI355X (gfx950).
 *
 * The library computes the draft model's output distribution over a per-step speculative
 * vocabulary (arxiv 2602.13836, Section 3): it scores the whole vocabulary with a low-rank
 * selector and keeps the k best tokens (Section 3.3, Steps 1-2), computes the exact logits of
 * those k tokens only by reading their rows of the output embedding once (Section 3.3, Step 3,
 * and "Custom kernel" in Section 3.5), and turns them into the subset softmax and the top-kd
 * draft tokens.  A full-vocabulary projection (Section 3.1) is exported as the baseline.
 *
 * Conventions shared by every entry point
 * ---------------------------------------
 * Memory.   Every pointer named "device" is GPU memory of the current HIP device, owned by the
 *           caller for the whole call and until the stream has finished the enqueued work.  The
 *           library allocates nothing, frees nothing and keeps no pointer after returning.
 * Layout.   Matrices are row-major.  ld* arguments are row strides in ELEMENTS.  h, U, W_down and
 *           W_vocab of one call share one storage type `dt`: SV_F32 (IEEE float32) or SV_BF16
 *           (bfloat16).  Logits, scores and probabilities are float32; token ids are int32.
 * Alignment.Base pointers of h, U, W_down, W_vocab and the workspace are 16-byte aligned; a row
 *           of h / U / W_down / W_vocab is a whole number of 16-byte units (d, d_prime multiples
 *           of 8 for bf16, of 4 for float32) and so are the row strides.
 * Stream.   `stream` is a hipStream_t passed as void* (NULL = the default stream).  Calls only
 *           enqueue work: they do not synchronise, do not read device memory on the host, and can
 *           be captured into a HIP graph.  Outputs are valid once the stream reaches that point.
 *           The first call on a device also runs a one-time device set-up (see specvocab_init); a
 *           caller whose first call would fall inside a stream capture calls specvocab_init before.
 * Workspace.`ws` is device scratch of at least specvocab_workspace_bytes(...) bytes for the same
 *           shape (may be NULL when that is 0).  Its contents need not be initialised and are
 *           undefined afterwards.  Calls that share a workspace must be ordered on one stream.
 * Errors.   Every entry point returns an sv_status.  Arguments are validated on the host before
 *           anything is enqueued; on any status other than SV_OK nothing has been launched.
 *           Index CONTENTS (range, uniqueness) are the caller's contract and are not checked --
 *           except in the debug mode switched on by the environment variable SPECVOCAB_VALIDATE=1:
 *           every call that takes an index list then first runs a range check over it, waits for
 *           the stream (so the call is no longer asynchronous nor capturable), and returns
 *           SV_ERR_INDEX without launching the operation if an entry lies outside [0, V) (a padding
 *           slot, -1, is accepted in lists passed with SV_IDX_PADDED) or if a list declared with
 *           SV_IDX_SORTED descends.
 * Precision.Products of the stored values are accumulated in float32 (order unspecified).
 *           With SV_BF16 storage the intermediate h' of the selector is rounded to bfloat16
 *           (round-to-nearest-even) before the second projection; with SV_F32 it stays float32.
 * Ties.     Wherever "largest" decides, equal values are ordered by smaller token id first.
 * Threads.  Entry points may be called from several host threads; the library keeps no per-call
 *           state on the host (only the per-device set-up, done once under a lock and read-only
 *           afterwards).  specvocab_select_static is the exception: see there.
 */
#ifndef SPECVOCAB_H
#define SPECVOCAB_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

#define SPECVOCAB_VERSION 100 /* major*10000 + minor*100 + patch */

typedef enum {
    SV_OK = 0,
    SV_ERR_NULL = 1,        /* a required pointer is NULL */
    SV_ERR_SHAPE = 2,       /* a size is out of range or sizes disagree (k > V, kd > k, ld < d ...) */
    SV_ERR_DTYPE = 3,       /* unknown sv_dtype / sv_idx_mode / sv_op value */
    SV_ERR_ALIGN = 4,       /* pointer or stride not 16-byte aligned */
    SV_ERR_WORKSPACE = 5,   /* workspace missing or too small */
    SV_ERR_UNSUPPORTED = 6, /* legal in principle, not handled by this build (see each function) */
    SV_ERR_INDEX = 7,       /* debug mode only: an index lies outside [0, V) */
    SV_ERR_HIP = 8          /* a HIP runtime call (kernel launch, device query) failed */
} sv_status;

/* SV_E4M3 names rows in 8 bits (see specvocab_quantize_rows); only specvocab_workspace_bytes takes it. */
typedef enum { SV_F32 = 0, SV_BF16 = 1, SV_E4M3 = 2 } sv_dtype;

/* SV_IDX_PER_ROW: idx is [rows x k], row r of h uses idx[r, :].
 * SV_IDX_PER_STEP: idx is [k], one set shared by every row of the step. */
typedef enum { SV_IDX_PER_ROW = 0, SV_IDX_PER_STEP = 1 } sv_idx_mode;

/* Subset sizes that differ from row to row inside fixed-size lists (Section 3.3 Step 2 lets k vary).
 * OR this flag into idx_mode to say that the index list may hold PADDING SLOTS: entries equal to -1
 * name no token.  A padding slot reads no row of U, its logit is -inf and its probability 0; the real
 * entries of the row are computed exactly as without padding, and the draft top-kd behaves as on the
 * compacted list of real entries (if a row has fewer than kd of them, the remaining tok_out entries
 * are -1 with probability 0; a row of padding only gets all probabilities 0).  With one hidden
 * row (and wherever the row-gather kernel serves the call) a padded list costs nothing extra; where
 * the matrix cores multiply (several bf16 hidden rows) the gathering calls need extra workspace
 * (specvocab_workspace_bytes with the flagged idx_mode) and two small extra launches.  Lists
 * without the flag must not contain -1. */
#define SV_IDX_PADDED 4

/* OR this flag into idx_mode to DECLARE that every list is sorted by ascending id (repeats allowed), which is how
 * specvocab_select emits its lists.  A declaration, not a request: the library does not sort, and a list that is
 * not sorted then gives wrong logits (never an access out of bounds; the debug mode reports SV_ERR_INDEX).  It
 * matters for a large batch: with more than 64 bf16 hidden rows, one list per row and rows * k >= 2 V -- sets that
 * together cover the vocabulary -- the gathering calls read all of U once, tile by tile, and store only the
 * entries each row asks for.  Lists in any order take the same route between a pass that groups every list by
 * tile and one that puts the logits back into the caller's order (two more small launches, 3 rows * k more words
 * of workspace, about a tenth more time at 512 rows); the declaration saves both.  Ignored together with
 * SV_IDX_PADDED and wherever it makes no difference. */
#define SV_IDX_SORTED 8

typedef enum {
    SV_OP_SELECT = 0,
    SV_OP_SUBSET_LOGITS = 1,
    SV_OP_DRAFT_TOPK = 2,
    SV_OP_DENSE_LOGITS = 3,
    SV_OP_DRAFT_STEP = 4,
    SV_OP_INDEXED_HEAD_NAIVE = 5,
    SV_OP_AUX_LOG_SOFTMAX = 6,
    SV_OP_QUANTIZED_DENSE_LOGITS = 7,  /* dt: what h is, SV_BF16 or SV_E4M3 */
    SV_OP_QUANTIZED_SUBSET_LOGITS = 8, /* the same */
    SV_OP_QUANTIZED_SAMPLE_STEP = 9,   /* the same; k: 0 for the whole vocabulary */
    SV_OP_SAMPLE = 10,                 /* k: logits of a row (n) */
    SV_OP_TOKEN_LOGPROBS = 11,         /* k: logits of a row (n); kd: alternatives (top); dt: type of the logits */
    SV_OP_DISTILL = 12                 /* k: logits of a row (n); dt: type of the logits */
} sv_op;

/* What a teacher's list holds (specvocab_distill). */
typedef enum {
    SV_TEACHER_LOGITS = 0,   /* logits: its probabilities are their softmax over the list, at the call's temperature */
    SV_TEACHER_LOGPROBS = 1, /* log probabilities at that temperature; the mass that the list leaves counts nothing */
    SV_TEACHER_REST = 2      /* the same; the mass that the list leaves counts as one more token */
} sv_teacher;

/* Largest kd the draft top-kd accepts. */
#define SPECVOCAB_MAX_KD 64
/* Most alternatives and most given tokens of a row in specvocab_token_logprobs, and most entries of a teacher's list. */
#define SPECVOCAB_MAX_TOP 64
#define SPECVOCAB_MAX_GIVEN 64
#define SPECVOCAB_MAX_TEACHER 512

/* SPECVOCAB_VERSION of the loaded library. */
int specvocab_version(void);

/* One-time set-up of the current HIP device: device attributes, the opt-in of the kernels that use more
 * than 64 KiB of LDS, and the device address of the static scratch array of specvocab_select_static.
 * Every entry point does this by itself on its first call on a device; call specvocab_init explicitly,
 * once per device and outside any stream capture, when that first call would otherwise happen while a
 * stream is being captured.  Idempotent and thread-safe.  Returns SV_OK or SV_ERR_HIP. */
int specvocab_init(void);

/* Static, NUL-terminated description of an sv_status value. */
const char* specvocab_status_string(int status);

/* Bytes of device workspace the given operation needs for the given shape, written to
 * *bytes_out (host pointer).  Arguments an operation does not have are ignored (pass 0).
 * 0 is a valid answer.  Returns SV_ERR_SHAPE / SV_ERR_DTYPE on sizes the operation rejects. */
int specvocab_workspace_bytes(int op, int64_t rows, int64_t d, int64_t V, int64_t k,
                              int64_t d_prime, int64_t kd, int dt, int idx_mode,
                              size_t* bytes_out);

/* Section 3.3, Steps 1 and 2: the candidate vocabulary of every row.
 *     h'[r, :] = W_down h[r, :]          W_down  device [d_prime x d], row stride d
 *     s[r, :]  = W_vocab h'[r, :]        W_vocab device [V x d_prime], row stride d_prime
 *     idx_out[r, :] = token ids of the k largest s[r, :], in ascending id order
 * h: device [rows x d], row stride ldh.  idx_out: device [rows x k] int32.
 * scores_out: device [rows x k] float32 receiving s[r, idx_out[r, j]], or NULL.
 * Requires 1 <= k <= V, 1 <= d_prime, rows >= 1; V above 4194304 is SV_ERR_UNSUPPORTED.
 * Cost.  Rows of up to 16384 tokens: s lies in the workspace, and one launch selects from it (bf16, exactly 16384:
 * up to 64 rows, up to 256 with d_prime > 256).  With bf16, scores_out == NULL, no threshold, d_prime <= 512 and
 * 16384 <= V <= 393216, a call of more than a handful of hidden rows keeps less than s in memory; the result is the
 * same exact top-k.
 *   Two bytes per score: d_prime <= 256 and 9 to 64 rows (d_prime > 128 and less than 24 rows: k <= V / 4, V > 98304:
 *   V / 8); d_prime <= 128, 2 to 8 rows, k <= V / 8 (up to 4 rows and V > 196608: V / 16); 128 < d_prime <= 256, 65
 *   to 128 rows, rows * ceil(V / 32768) <= 256; d_prime > 256, 65 to 128 rows, up to 16.8 million scores, to 256 rows
 *   up to 10 million.  A sample of the scores brackets each row's k-th: of every 32 tokens those whose id modulo 32
 *   is 0 or 16, V <= 65536 also 10 or 26, V <= 32768 also 2, 8, 18 or 24.  Likeness of neighbouring tokens does not
 *   mislead it, and chance one row in hundreds of millions; scores that depend on the id modulo 32 do.  Such a row
 *   takes up to 20 us more at 40000 tokens, 37 at 128256, 57 at 262144 (all rows of 64: 66), and the call as long as
 *   its slowest row.  The two bytes hold a score's distance from a score near the row's median in 11 bits, and the
 *   tokens that share the k-th one's (a dozen) are computed again: more of them where a row's scores lie in groups
 *   far apart against their width and the k-th in the one that the median is not in (200 standard deviations apart:
 *   30 to 100 us more).
 *   One byte per score: every other shape of 65 rows and more.  The scores of 4096 evenly spaced tokens (ids floor(j
 *   V / 4096)) decide how a row's scores map to bytes, and those that share the k-th one's are computed again.  Where
 *   the sample misleads (about 1e-5 of rows on scores that do not depend on the token id modulo the sampling stride;
 *   certain for inputs built so that the sampled tokens score unlike all others) a row takes tens of microseconds
 *   more, up to a few milliseconds.
 * From 65 hidden rows and 32768 tokens on wider selectors keep only the few per cent of scores inside a bracket from
 * 8192 sampled tokens (ids floor(j V / 8192)); a row whose bracket misses is recomputed by a slow exact path, about a
 * millisecond per such row.  Every other shape, every call with scores_out and every threshold materialises s in the
 * workspace, which is the same size either way: 12 bytes per score and some kilobytes per row. */
int specvocab_select(const void* h, int64_t rows, int64_t d, int64_t ldh,
                     const void* W_down, int64_t d_prime,
                     const void* W_vocab, int64_t V,
                     int dt, int64_t k,
                     int32_t* idx_out, float* scores_out,
                     void* ws, size_t ws_bytes, void* stream);

/* specvocab_select for callers that cannot allocate device memory or pass a workspace: code running under
 * HIP graph capture, tight serving loops, harnesses that forbid hipMalloc.  Same arguments, results and
 * kernels as specvocab_select, but the scratch memory is a static device array inside the library
 * (SPECVOCAB_STATIC_SCRATCH_BYTES per GPU the library runs on, held until the process ends) instead of a
 * workspace argument; the call allocates nothing and frees nothing.  Shapes whose
 * specvocab_workspace_bytes(SV_OP_SELECT, ...) exceeds SPECVOCAB_STATIC_SCRATCH_BYTES return
 * SV_ERR_WORKSPACE (8 MiB holds one hidden row at V up to about 600000, or four rows at V = 128256).
 * All calls on one GPU share that GPU's array, which keeps the previous call's contents (the kernels
 * clear what must start at zero): calls that overlap on one GPU -- different streams or host threads
 * without ordering between them -- race; order them on one stream. */
#define SPECVOCAB_STATIC_SCRATCH_BYTES (8u << 20)
int specvocab_select_static(const void* h, int64_t rows, int64_t d, int64_t ldh,
                            const void* W_down, int64_t d_prime,
                            const void* W_vocab, int64_t V,
                            int dt, int64_t k,
                            int32_t* idx_out, float* scores_out, void* stream);

/* specvocab_select with a score threshold: of the k best tokens of a row only those with
 * s[r, v] >= tau stay; the others become padding slots in place (idx_out = -1, scores_out = -inf),
 * so that the list keeps its length k and its ascending id order and can be passed on with
 * SV_IDX_PADDED.  tau = -INFINITY is specvocab_select; NaN is SV_ERR_SHAPE.  Workspace as for
 * SV_OP_SELECT. */
int specvocab_select_threshold(const void* h, int64_t rows, int64_t d, int64_t ldh,
                               const void* W_down, int64_t d_prime,
                               const void* W_vocab, int64_t V,
                               int dt, int64_t k, float tau,
                               int32_t* idx_out, float* scores_out,
                               void* ws, size_t ws_bytes, void* stream);

/* Section 3.3, Step 3 (the fused indexed LM head of Section 3.5, "Custom kernel"):
 *     logits_out[r, j] = < U[idx(r, j), :], h[r, :] >
 * without materialising U[idx, :]; each needed row of U is read from memory once per use.
 * h: device [rows x d] stride ldh.  U: device [V x d] stride ldu.
 * idx: device int32, [rows x k] (SV_IDX_PER_ROW) or [k] (SV_IDX_PER_STEP), any order; every
 * entry must lie in [0, V) (caller's contract, unchecked) or, with SV_IDX_PADDED, be -1.
 * Duplicates just repeat the value.
 * logits_out: device [rows x k] float32.
 * With several hidden rows and one set per row (a draft tree) the union of the sets is formed in
 * the workspace and each needed row of U is read once per step rather than once per asking row;
 * specvocab_workspace_bytes(SV_OP_SUBSET_LOGITS, ...) says how much that needs (0 otherwise). */
int specvocab_subset_logits(const void* h, int64_t rows, int64_t d, int64_t ldh,
                            const void* U, int64_t V, int64_t ldu, int dt,
                            const int32_t* idx, int64_t k, int idx_mode,
                            float* logits_out,
                            void* ws, size_t ws_bytes, void* stream);

/* Subset softmax (Section 3.3, q_K = softmax(z')) and the top-kd draft tokens of every row
 * (inference hyper-parameter "Top-k", 10 in the paper's appendix):
 *     q[r, j]      = exp(logits[r, j] - max_j) / sum_l exp(logits[r, l] - max_j)
 *     tok_out[r,t] = idx(r, j_t), prob_out[r, t] = q[r, j_t], where j_0, j_1, ... order the row by
 *                    descending logit, equal logits by ascending token id
 * logits: device [rows x k] float32 (finite).  idx: as in specvocab_subset_logits; token ids of
 * one row must be unique.  tok_out: device [rows x kd] int32.  prob_out: device [rows x kd]
 * float32.  probs_full_out: device [rows x k] float32 receiving q, or NULL.
 * Requires 1 <= kd <= min(k, SPECVOCAB_MAX_KD), else SV_ERR_SHAPE / SV_ERR_UNSUPPORTED. */
int specvocab_draft_topk(const float* logits, const int32_t* idx, int idx_mode,
                         int64_t rows, int64_t k, int64_t kd,
                         int32_t* tok_out, float* prob_out, float* probs_full_out,
                         void* ws, size_t ws_bytes, void* stream);

/* The whole draft step after selection: specvocab_subset_logits followed by specvocab_draft_topk on
 * the logits it produced (Section 3.3 Step 3 and q_K = softmax(z'), then the top-kd tokens), with the
 * same arguments, results and tie rule as those two calls, enqueued back to back on `stream`.
 * (Two kernels on purpose: on this multi-die GPU a kernel boundary is the cheapest device-wide
 * synchronisation; a single-launch version with an in-kernel hand-over measured slower.)
 * logits_out: device [rows x k] float32, required (the top-kd stage reads it). */
int specvocab_draft_step(const void* h, int64_t rows, int64_t d, int64_t ldh,
                         const void* U, int64_t V, int64_t ldu, int dt,
                         const int32_t* idx, int64_t k, int idx_mode, int64_t kd,
                         float* logits_out, int32_t* tok_out, float* prob_out, float* probs_full_out,
                         void* ws, size_t ws_bytes, void* stream);

/* Comparator, not part of the method: the indexed LM head done the naive way the paper's kernel
 * replaces (Section 3.5 "Custom kernel", Figure 3a): U' = U[idx, :] is first materialised in the
 * workspace (k rows read and written), then logits_out = U' h is computed over the copy (k rows read
 * again).  Same arguments and results as specvocab_subset_logits; exists so that the benchmark can
 * put the fused gather next to the three-times-the-traffic path on the same GPU.
 * One index set per hidden row or per step; the workspace holds rows x k x d (or k x d) elements. */
int specvocab_indexed_head_naive(const void* h, int64_t rows, int64_t d, int64_t ldh,
                                 const void* U, int64_t V, int64_t ldu, int dt,
                                 const int32_t* idx, int64_t k, int idx_mode,
                                 float* logits_out,
                                 void* ws, size_t ws_bytes, void* stream);

/* Static-vocabulary mode (the fixed sub-vocabularies the paper compares against: Section 2 "Static
 * sub-vocabularies", the 32K-token baselines of Section 4): packs U' = U[idx, :] into a dense matrix
 * once, when the static vocabulary is chosen,
 *     U_packed[j, :] = U[idx[j], :]            j < k
 * after which every draft step is specvocab_dense_logits over U_packed (V = k) followed by
 * specvocab_draft_topk with the same idx as the token ids (SV_IDX_PER_STEP).
 * idx: device [k] int32, entries in [0, V) (caller's contract).  U_packed: device [k x d] in `dt`, row
 * stride d, 16-byte aligned, written completely; it must not overlap U. */
int specvocab_pack_rows(const void* U, int64_t V, int64_t d, int64_t ldu, int dt,
                        const int32_t* idx, int64_t k, void* U_packed, void* stream);

/* Section 3.4 (training side, forward only): the vocabulary speculator's own output distribution over
 * the ENTIRE vocabulary, q_aux = softmax(s) with s = W_vocab (W_down h) as in specvocab_select, returned
 * as natural-log probabilities (what a cross-entropy style distillation loss consumes):
 *     logq_out[r, v] = s[r, v] - log sum_u exp(s[r, u])
 * Arguments as in specvocab_select; logq_out: device [rows x V] float32.  No limit on V beyond int32. */
int specvocab_aux_log_softmax(const void* h, int64_t rows, int64_t d, int64_t ldh,
                              const void* W_down, int64_t d_prime,
                              const void* W_vocab, int64_t V, int dt,
                              float* logq_out,
                              void* ws, size_t ws_bytes, void* stream);

/* Measurement aid, not part of the method: one plain streaming read of buf (device, 16-byte aligned, `bytes` a
 * multiple of 16): every lane loads 16 bytes per instruction, consecutive lanes consecutive addresses, nothing
 * is written.  Timed over a buffer much larger than the caches it gives the read bandwidth a kernel can reach on
 * the machine, which the benchmark quotes beside the published HBM peak.  ws: 262144 bytes of device scratch. */
int specvocab_stream_read_probe(const void* buf, size_t bytes, void* ws, size_t ws_bytes, void* stream);

/* Section 3.1, the full-vocabulary baseline:  logits_out[r, v] = < U[v, :], h[r, :] >.
 * logits_out: device [rows x V] float32. */
int specvocab_dense_logits(const void* h, int64_t rows, int64_t d, int64_t ldh,
                           const void* U, int64_t V, int64_t ldu, int dt,
                           float* logits_out,
                           void* ws, size_t ws_bytes, void* stream);

/* ---- From a layer's output to a token, with the output embedding in 8 bits ------------------------------------------------
 *
 * Rows in 8 bits: a row of d values (d a multiple of 16) is d e4m3 codes and, in another array, one byte per block of 128 values,
 * the exponent of the block's scale: 2^(byte - 127), 255 for NaN (e8m0).  Value i of the row is scale[i / 128] * code[i].  A row has
 * 4 * ceil(d / 512) scale bytes (whole words; bytes past the last block are 127).  Row strides: of codes at least d and a multiple of
 * 16, of scales at least that number and a multiple of 4, bases aligned likewise; else SV_ERR_ALIGN.
 *
 * specvocab_quantize_rows: the rows of x [rows x d] (SV_F32 or SV_BF16, d a multiple of 16) in 8 bits -- the output embedding
 * once, hidden rows per step.  A block's scale is the smallest 2^e, e >= -126, with max|x| <= 448 * 2^e (1 for a block of zeros); a
 * code is x / 2^e, which is exact, rounded to nearest even.  A block with an infinity or a NaN in it has scale 255 and
 * NaN codes.  rows is limited by int32 only.  The outputs must not overlap x. */
int specvocab_quantize_rows(const void* x, int64_t rows, int64_t d, int64_t ldx, int dt,
                            uint8_t* q_out, int64_t ldq, uint8_t* scales_out, int64_t lds, void* stream);

/* The root-mean-square norm in front of a head, with the residual's addition:
 *     t[r] = x[r] + residual[r]                       (x[r] where residual is NULL), rounded to `dt`
 *     y[r] = t[r] / sqrt(mean_i t[r, i]^2 + eps) * (weight + weight_offset), rounded to `dt`
 * sum_out (needs residual), y_out, and q_out with scales_out (y in 8 bits) receive t, y and the 8 bits of y as it is stored: the same
 * bits as an addition, a norm and specvocab_quantize_rows called one after the other.  Each may be NULL, but not both y_out and
 * q_out.  The selector reads y (specvocab_select), the 8-bit head q.  weight: [d] in `dt`; weight_offset: 0, or 1 for models that store
 * the weight's distance from 1.  Sums are float32.  sum_out and y_out may be x or residual themselves (same base and stride), not
 * otherwise overlap them or each other.  d a multiple of 16; eps >= 0 and finite.  No workspace.  A row with an infinity or a NaN
 * in t gets NaN throughout; finite rows whose squares are too large or too small for float32 are scaled on the way and get their norm. */
int specvocab_rms_norm(const void* x, int64_t rows, int64_t d, int64_t ldx, const void* residual, int64_t ldr,
                       const void* weight, float weight_offset, float eps, int dt,
                       void* sum_out, int64_t ld_sum, void* y_out, int64_t ldy,
                       uint8_t* q_out, int64_t ldq, uint8_t* scales_out, int64_t lds, void* stream);

/* specvocab_dense_logits and specvocab_subset_logits with the embedding in 8 bits:
 *     logits_out[r, j] = < U[row(j), :], h[r, :] >     over the values that codes and scales stand for, accumulated in float32
 * h: rows in 8 bits (h_scales not NULL; ldh in codes, ldhs in scale bytes), or bfloat16 rows (h_scales NULL; ldh in elements,
 * ldhs ignored).  d a multiple of 16.  idx, k, idx_mode as in specvocab_subset_logits (SV_IDX_SORTED makes no difference).  A
 * NaN code or scale makes the logits that use it NaN.  The values are widened to bfloat16, which is exact, and multiplied as such: values of
 * h or U below 2^-126 may count as 0, and |h| beyond 2^100 may overflow (some forms apply U's scale to sums of 16 products). */
int specvocab_quantized_dense_logits(const void* h, const uint8_t* h_scales, int64_t rows, int64_t d, int64_t ldh, int64_t ldhs,
                                     const uint8_t* U, const uint8_t* U_scales, int64_t V, int64_t ldu, int64_t ldus,
                                     float* logits_out, void* ws, size_t ws_bytes, void* stream);
int specvocab_quantized_subset_logits(const void* h, const uint8_t* h_scales, int64_t rows, int64_t d, int64_t ldh, int64_t ldhs,
                                      const uint8_t* U, const uint8_t* U_scales, int64_t V, int64_t ldu, int64_t ldus,
                                      const int32_t* idx, int64_t k, int idx_mode,
                                      float* logits_out, void* ws, size_t ws_bytes, void* stream);

/* One token per row, drawn with a given random number u[r] in [0, 1) (smaller ones count as 0, larger ones and 1 as the
 * largest float below 1).  logits: device [rows x n] float32, row stride ld (any alignment).  With T = temperature[r] and the
 * row's places ordered by descending logit, equal logits by place (for ascending lists: by token id), w = exp((logit - largest) / T):
 *   1. top_k[r] > 0:  the first top_k[r] places stay;
 *   2. top_p[r] < 1:  of those, the ones stay that have less than top_p[r] of their mass in front of them (always the first);
 *   3. min_p[r] > 0:  of those, the ones with w >= min_p[r] stay (above 1 counts as 1);
 *   4. the first place of those at which the running sum of w exceeds u[r] times the sum over all of them is drawn.
 * T <= 0 or NaN: the first place, with probability 1.  NaN in top_p or min_p: no such step.  temperature, top_k, top_p,
 * min_p: device [rows], or NULL for 1, 0, 1, 0.  Places with a logit of -inf or NaN are masked: they are in none of the steps.
 * Places with w below 2^-64 (or, in some rows, 2^-88) have no mass and count as masked too.  A +inf logit takes all of a row's
 * mass.
 * tok_out: device [rows] int32, the place, or idx(r, place) where idx (as in specvocab_subset_logits, padding slots having a logit of
 * -inf) is not NULL; -1 for a row that is masked throughout.  prob_out: device [rows] float32, w over the sum in 4 (0 for such
 * a row), or NULL.
 * Sums are kept to 2^-44 of each term (n up to 2^18; a bit less for each doubling of n), and do not depend on the run.  How they are
 * rounded below that depends on the form that serves the row, which goes by rows and n.
 * One launch; four (and workspace) for up to 64 rows of 49152 logits or more.  A row in which more than 1024 places crowd into one of
 * the 4096 steps (1024 for short rows) that its range, or 64 octaves of w, is cut into, at a border or where the token is drawn --
 * thousands of equal logits, clusters far apart --, costs some tens of passes over the row. */
int specvocab_sample(const float* logits, int64_t ld, int64_t rows, int64_t n, const int32_t* idx, int idx_mode,
                     const float* temperature, const int32_t* top_k, const float* top_p, const float* min_p, const float* u,
                     int32_t* tok_out, float* prob_out, void* ws, size_t ws_bytes, void* stream);

/* The step from hidden rows to tokens: specvocab_quantized_subset_logits (idx NULL: specvocab_quantized_dense_logits, k ignored)
 * followed by specvocab_sample on its logits, enqueued back to back.  logits_out: device [rows x k] (or V) float32, required. */
int specvocab_quantized_sample_step(const void* h, const uint8_t* h_scales, int64_t rows, int64_t d, int64_t ldh, int64_t ldhs,
                                    const uint8_t* U, const uint8_t* U_scales, int64_t V, int64_t ldu, int64_t ldus,
                                    const int32_t* idx, int64_t k, int idx_mode,
                                    const float* temperature, const int32_t* top_k, const float* top_p, const float* min_p,
                                    const float* u, float* logits_out, int32_t* tok_out, float* prob_out,
                                    void* ws, size_t ws_bytes, void* stream);

/* ---- Over finished rows of logits: what a token's probability is, and what a draft model learns from a teacher -------------------
 *
 * logits: device [rows x n] in `dt` (SV_F32: what the products of this library leave; SV_BF16: a training program's), row stride ld in
 * elements, aligned to an element.  -inf masks a place: it has probability 0 and no gradient.  Any other value is a logit, the type's
 * lowest too.  A row with a NaN or +inf has NaN throughout, and no alternatives (-1).  A row that is masked throughout has log probabilities of -inf, entropy
 * 0 and no gradient.  grad_out: device [rows x n] in `grad_dt` (SV_F32 or SV_BF16, rounded to nearest even), row stride ld_grad, every
 * place written; it may be the logits themselves (same base, stride and type; another type is SV_ERR_DTYPE, another stride SV_ERR_SHAPE) and must not
 * overlap them otherwise.
 * Results do not depend on the run.  Sums are float32, relative to a logit near the largest; probabilities below 2^-126 count as 0.
 * Tokens that name no place are allowed for.  The debug mode lets -1 pass and names the others (SV_ERR_INDEX): the tokens given to
 * specvocab_token_logprobs without a list and to its gradient, and a teacher's.
 * `state` is what a gradient needs of the forward call: device [rows x 4] float32, 16-byte aligned. */

/* Log probabilities of given tokens, the entropy and the largest alternatives of every row, natural logarithms at temperature T =
 * temperature[r] (device [rows] float32, or NULL for 1; kept within 2^-20 .. 2^20; T <= 0 and NaN count as 1):
 *     logprob_out[r, j] = z[t_j] / T - log sum_v exp(z[v] / T),  t_j = tokens[r, j]     device [rows x given] float32
 *     entropy_out[r]    = - sum_v p_v log p_v                                           device [rows] float32, or NULL
 *     top_tok_out, top_logprob_out: the `top` largest places and their log probabilities, by descending logit, equal logits by
 *                          place, -1 with -inf where the row has no more              device [rows x top] int32, float32
 *     state_out[r]      = (m, sum_v exp((z[v] - m) / T), entropy, 0), m a logit near the row's largest, or NULL
 * tokens: device [rows x given] int32, 0 <= given <= SPECVOCAB_MAX_GIVEN (0: none, tokens and logprob_out NULL); a token that names no place
 * (-1, a place past the row, an id that is not in the list) has -inf.  0 <= top <= min(n, SPECVOCAB_MAX_TOP); top > 0 with n above
 * 8388608 is SV_ERR_UNSUPPORTED.
 * idx, idx_mode: the token ids of the places, as in specvocab_sample (any order), or NULL: a token is its place.  Of equal ids
 * the first place counts.
 * One launch; two, and workspace, where there are few rows for their length, or rows of more than 262137 places.  Rows in which more than 1024 places may be among the
 * largest (equal logits in their hundreds) take some ten passes over the row. */
int specvocab_token_logprobs(const void* logits, int64_t ld, int64_t rows, int64_t n, int dt,
                             const int32_t* idx, int idx_mode, const float* temperature,
                             const int32_t* tokens, int64_t given, int64_t top,
                             float* logprob_out, float* entropy_out, int32_t* top_tok_out, float* top_logprob_out, float* state_out,
                             void* ws, size_t ws_bytes, void* stream);

/* The logits' gradient of specvocab_token_logprobs without a list (cross entropy, policy gradients, entropy bonuses):
 *     grad_out[r, v] = (sum_j grad_logprob[r, j] ([v = t_j] - p_v) - grad_entropy[r] p_v (log p_v + entropy[r])) / T
 * grad_logprob: device [rows x given] float32, or NULL (then tokens may be NULL); grad_entropy: device [rows] float32, or NULL; not both NULL.
 * state: what the forward call at the same temperature wrote.  A token that is given several times gets the sum; one that names no place, nothing.  No workspace. */
int specvocab_token_logprobs_grad(const void* logits, int64_t ld, int64_t rows, int64_t n, int dt, const float* temperature,
                                  const int32_t* tokens, int64_t given, const float* state,
                                  const float* grad_logprob, const float* grad_entropy,
                                  void* grad_out, int64_t ld_grad, int grad_dt, void* stream);

/* Distillation (Section 3.4's losses, for a teacher of whose rows the largest logits were kept): the divergence of q = softmax(z / T) from
 * the teacher's probabilities p_j of the tokens t_j = tok[r, j] that it lists, times weight[r],
 *     loss_out[r] = weight[r] (sum_j p_j (log p_j - log q[t_j])  [+ p' (log p' - log q')])         device [rows] float32
 *     grad_out[r, v] = weight[r] / T (m q[v] - sum_{j: t_j = v} p_j  [- p' q[v] / q', v not listed])
 * with m the mass that counts, sum_j p_j [+ p'].  In brackets: SV_TEACHER_REST only; p' = 1 - sum_j p_j (at least 0) and q' the mass
 * of all places that are not listed (left out where there is no such place).  tok, teacher: device [rows x known] int32 and float32, 1 <= known <=
 * SPECVOCAB_MAX_TEACHER, in any order; an entry whose token lies outside [0, n) (-1: padding) is not there, one of -inf has no mass, and a
 * token that is listed twice has both masses.  specvocab_token_logprobs writes such lists (top_tok_out, top_logprob_out).  A listed token with mass at a
 * masked place makes the loss +inf.  temperature: T, finite, within 2^-20 .. 2^20; weight: device [rows] float32, or NULL for 1; a row of weight 0
 * is not read: loss 0, gradient 0.  A mean over tokens or a factor T^2 goes into the weight.
 * state_out[r] = (m, sum_v exp((z[v] - m) / T), the same two over the places that are not listed (SV_TEACHER_REST only, else 0)), m a number
 * near the largest of those logits, or NULL.
 * grad_out may be NULL: the loss alone (or its gradient later, when the factors are known, by specvocab_distill_grad with the same arguments and
 * the state; weight[r] is then whatever factor the row's divergence has -- but a row that had weight 0 in the forward call was not read, has a state
 * of zeros and gets a gradient of 0 whatever its weight then is).  Both at once keep a part of each row
 * on the chip and read the others a second time.
 * One launch; two, three with the gradient (every row is read twice then), and workspace where there are few rows for their length, or rows of more than
 * 262137 places. */
int specvocab_distill(const void* logits, int64_t ld, int64_t rows, int64_t n, int dt,
                      const int32_t* tok, const float* teacher, int64_t known, int kind, float temperature, const float* weight,
                      float* loss_out, float* state_out, void* grad_out, int64_t ld_grad, int grad_dt,
                      void* ws, size_t ws_bytes, void* stream);
int specvocab_distill_grad(const void* logits, int64_t ld, int64_t rows, int64_t n, int dt,
                           const int32_t* tok, const float* teacher, int64_t known, int kind, float temperature, const float* weight,
                           const float* state, void* grad_out, int64_t ld_grad, int grad_dt, void* stream);

#ifdef __cplusplus
}
#endif
#endif /* SPECVOCAB_H */
