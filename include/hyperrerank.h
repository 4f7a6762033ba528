/*
 * hyperrerank - C ABI of the MI355X reranker scoring library.
 *
 * The method (HyperRAG, Section 3.3 Property 1 and Section 4.2): a decoder-only
 * reranker scores a (document, query) pair on the sequence [document ; query].
 * Because attention is lower-triangular and the document always starts the
 * sequence, every layer's K/V of the document can be computed once, stored, and
 * reused for any query; scoring then runs only the short query suffix through
 * the layers while attending to the stored document K/V ("static document
 * prefix | query suffix" KV layout).  This library keeps the stored K/V in a
 * paged pool in HBM and implements that scoring pass for a batch of pairs.
 *
 * Conventions
 *   - "host" pointers are ordinary CPU memory, read during the call only.
 *   - "device" pointers are HBM addresses on the current HIP device.  The
 *     library never allocates or frees device memory: pools, packed weights,
 *     workspaces and outputs are all caller-owned.
 *   - `stream` is a hipStream_t passed as void* (NULL = the default stream).
 *     Calls that take a stream enqueue work and return without waiting.
 *   - A model handle carries per-call host state (a pinned staging buffer, an event, a second stream): calls on
 *     one handle must not overlap in host time; different handles, and pools, are independent.  The library
 *     allocates no device memory, but it owns that small pinned host buffer (1 MiB from hr_weights_load on, grown
 *     when a call's metadata needs more) and, once a scoring call has been cut in two halves, one stream and three
 *     events per model handle (released by hr_model_destroy).
 *   - Calls that upload per-call metadata (scoring, prefill) wait on the host for the previous upload of the same
 *     handle and copy from its staging buffer: they are not meant to be recorded into a HIP graph.  hr_rerank_plan_run
 *     is the form that is.
 *   - Every call returns HR_OK (0) or a negative hr_status.  Every argument check happens before anything is enqueued
 *     or any library state changes; only HR_ERR_DEVICE (a HIP call failed mid-way) can leave part of a call's work on the
 *     stream, and the outputs of that call are then undefined.  Nothing throws or aborts.
 *   - All matrices are row-major [out][in]; activations use the model dtype
 *     (HR_F32 or HR_BF16); norm gains and scores are fp32.
 *   - A page holds 16 consecutive tokens of one document for one (layer,
 *     kv head): K as [16][head_dim] and V transposed; the in-pool arrangement
 *     is private to the library (use hr_doc_kv_write to fill it).
 */
#ifndef HYPERRERANK_H
#define HYPERRERANK_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

#define HR_PAGE_TOKENS 16

typedef enum hr_status {
    HR_OK = 0,
    HR_ERR_INVALID_ARG = -1,       /* null pointer, non-positive count, bad enum                    */
    HR_ERR_POOL_TOO_SMALL = -2,    /* device buffer smaller than hr_kv_pool_bytes                    */
    HR_ERR_PAGE_RANGE = -3,        /* page id < 0 or >= num_pages                                     */
    HR_ERR_PAGE_IN_USE = -4,       /* writing a page that already holds a document                    */
    HR_ERR_PAGE_DUP = -5,          /* the same page id twice in one document                          */
    HR_ERR_LEN_RANGE = -6,         /* document / query length <= 0 or above the supported maximum    */
    HR_ERR_TABLE_SHORT = -7,       /* page-table row too short, or -1 / unwritten page inside it     */
    HR_ERR_TOKEN_RANGE = -8,       /* token id < 0 or >= vocab                                        */
    HR_ERR_WORKSPACE_SMALL = -9,   /* workspace smaller than hr_rerank_workspace_bytes                */
    HR_ERR_UNSUPPORTED_SHAPE = -10,/* model / pool shape the kernels do not cover                     */
    HR_ERR_DEVICE = -11,           /* a HIP runtime call failed (no device, launch error)            */
    HR_ERR_POOL_FULL = -12,        /* hr_kv_pool_alloc_pages: not enough free pages                   */
    HR_ERR_MISMATCH = -13          /* pool and model disagree (layers, kv heads, head_dim, dtype)    */
} hr_status;

typedef enum hr_dtype { HR_F32 = 0, HR_BF16 = 1, HR_FP8_E4M3 = 2 } hr_dtype;

/* Paged document-KV pool.  kv_dtype: HR_F32, HR_BF16, or HR_FP8_E4M3 (OCP E4M3, one fp32 scale
 * per (layer, page, kv head) for K and one for V; value = decode(code) * scale).  The 8-bit form
 * follows Section 4.1 "KV-cache Quantization" / Appendix B (KV8, expanded after loading). */
typedef struct hr_pool_cfg {
    int32_t n_layers;
    int32_t n_kv_heads;
    int32_t head_dim;      /* multiple of 16, at most 256 */
    int32_t page_tokens;   /* must be HR_PAGE_TOKENS */
    int32_t num_pages;
    int32_t kv_dtype;      /* hr_dtype */
} hr_pool_cfg;

/* Reranker: pre-norm decoder blocks with RMSNorm, rotate-half RoPE, grouped-query attention,
 * SwiGLU, no biases; score = logit[yes_id] - logit[no_id] at the last query token with the
 * embedding matrix as the (tied) head, after the final RMSNorm. */
typedef struct hr_model_cfg {
    int32_t n_layers;
    int32_t hidden;
    int32_t n_q_heads;
    int32_t n_kv_heads;    /* divides n_q_heads */
    int32_t head_dim;
    int32_t ffn;
    int32_t vocab;
    int32_t yes_id;
    int32_t no_id;
    int32_t dtype;         /* HR_F32 or HR_BF16: weights and activations */
    float rope_base;
    float rms_eps;
} hr_model_cfg;

/* Device pointers to the caller's weights.  The per-layer members are HOST arrays of n_layers
 * DEVICE pointers.  Matrices are in the model dtype; norm gains are fp32. */
typedef struct hr_weight_ptrs {
    const void* embedding;        /* device [vocab][hidden] */
    const float* final_norm;      /* device [hidden] */
    const void* const* wq;        /* [n_q_heads*head_dim][hidden] */
    const void* const* wk;        /* [n_kv_heads*head_dim][hidden] */
    const void* const* wv;        /* [n_kv_heads*head_dim][hidden] */
    const void* const* wo;        /* [hidden][n_q_heads*head_dim] */
    const void* const* wg;        /* [ffn][hidden] */
    const void* const* wu;        /* [ffn][hidden] */
    const void* const* wd;        /* [hidden][ffn] */
    const float* const* norm1;    /* [hidden] pre-attention gain */
    const float* const* norm2;    /* [hidden] pre-MLP gain */
} hr_weight_ptrs;

typedef struct hr_pool hr_pool;     /* host-side handle: layout + page bookkeeping */
typedef struct hr_model hr_model;   /* host-side handle: config + packed-weight pointers */

const char* hr_status_str(int status);

/* Text of the HIP error behind the calling thread's most recent HR_ERR_DEVICE ("" if none). */
const char* hr_last_error(void);

/* ---- document-KV pool (the stored per-document KV of Section 3.3 / 4.2, kept resident in HBM) ---- */

/* Bytes of device memory a pool of this shape needs; 0 if cfg is invalid. */
size_t hr_kv_pool_bytes(const hr_pool_cfg* cfg);

/* Bind a pool to caller-owned device memory `dev_mem` (>= hr_kv_pool_bytes, 256-byte aligned).
 * Pure host work: nothing is enqueued; all pages start free.  *out is freed by hr_kv_pool_destroy
 * (which does not touch dev_mem). */
int hr_kv_pool_create(const hr_pool_cfg* cfg, void* dev_mem, size_t bytes, hr_pool** out);
void hr_kv_pool_destroy(hr_pool* pool);

/* Number of free pages, or a negative status. */
int64_t hr_kv_pool_free_pages(const hr_pool* pool);

/* Reserve the n lowest-numbered free pages and return their ids in page_ids_out (host).  Reserved
 * pages can be written once with hr_doc_kv_write and are released with hr_doc_kv_free. */
int hr_kv_pool_alloc_pages(hr_pool* pool, int32_t n, int32_t* page_ids_out);

/* Store one document's K/V (stage one of the two-stage inference) into the pages the caller names.
 *   page_ids      host, ceil(doc_len/16) distinct ids, each free or reserved
 *   k_dev, v_dev  device, logical layout [n_layers][doc_len][n_kv_heads][head_dim] in kv_dtype
 *                 (fp8: E4M3 codes, one byte each); K is post-RoPE at positions 0..doc_len-1
 *   k_scales_dev, v_scales_dev   fp8 only: device fp32 [n_layers][n_pages][n_kv_heads]; else NULL
 * One HBM->HBM scatter kernel is enqueued on `stream`; the tail of a short last page is zeroed.
 * The source buffers must stay valid until that kernel has run. */
int hr_doc_kv_write(hr_pool* pool, int32_t doc_len, const int32_t* page_ids,
                    const void* k_dev, const void* v_dev,
                    const float* k_scales_dev, const float* v_scales_dev, void* stream);

/* Read one document's K/V back from its pages (the inverse of hr_doc_kv_write): what a storage tier would take
 * from the pool (Section 4.1 keeps the cached KV outside GPU memory), and what makes the pages a prefill wrote
 * checkable value by value.
 *   page_ids      host, ceil(doc_len/16) ids of pages that hold a document (written or prefilled)
 *   k_dev, v_dev  device, logical layout [n_layers][doc_len][n_kv_heads][head_dim] in the pool's own element type:
 *                 fp32 for HR_F32 pools, IEEE half for HR_BF16 pools (the pool keeps the caller's bf16 values as
 *                 halves: exactly for magnitudes in [2^-14, 65504], see hr_kv_pool_range_report for the rest; prefilled
 *                 pages are halves in the first place), E4M3 codes for fp8 pools
 *   k_scales_dev, v_scales_dev   fp8 only: device fp32 [n_layers][n_pages][n_kv_heads]; else NULL
 * One gather kernel is enqueued on `stream`.  HR_ERR_PAGE_RANGE for an id out of range, HR_ERR_TABLE_SHORT for a page
 * that holds nothing, HR_ERR_LEN_RANGE for doc_len <= 0. */
int hr_doc_kv_read(const hr_pool* pool, int32_t doc_len, const int32_t* page_ids,
                   void* k_dev, void* v_dev, float* k_scales_dev, float* v_scales_dev, void* stream);

/* Mark pages free again (contents are left as they are). */
int hr_doc_kv_free(hr_pool* pool, const int32_t* page_ids, int32_t n);

/* ---- host tier (Sections 4.1 and 4.3: the documents' KV lives in a storage backend behind the GPU and is loaded for
 * the retrieved candidates; here the backend is the caller's memory, normally pinned host memory, and a page moves
 * as one record) ---- */

/* Bytes of one page record: the page's K and V blocks of every layer and kv head in the pool's own arrangement
 * ([n_layers][n_kv_heads][K block | V block]), followed for fp8 pools by its scales ([n_layers][n_kv_heads][K, V] fp32).
 * A multiple of 16; 0 if pool is NULL.  Records are opaque: only a pool of the same configuration reads them. */
size_t hr_kv_page_record_bytes(const hr_pool* pool);

/* Copy n_pages pages out of the pool: record i at dst + i * hr_kv_page_record_bytes is page page_ids[i].
 *   page_ids  host, ids of pages that hold a document (HR_ERR_PAGE_RANGE / HR_ERR_TABLE_SHORT otherwise)
 *   dst       n_pages records of memory the GPU can address: device memory, or host memory pinned by the HIP runtime
 *             (hipHostMalloc); 16-byte aligned.  Pageable host memory is refused with HR_ERR_INVALID_ARG.
 * Copy kernels are enqueued on `stream` (they write pinned host memory over the bus directly: no staging buffer);
 * dst is complete when the stream has drained.  The pool is unchanged. */
int hr_kv_pages_out(const hr_pool* pool, int32_t n_pages, const int32_t* page_ids, void* dst, void* stream);

/* The inverse: page page_ids[i] <- record i of src (same kinds of memory as dst above).  The pages must be distinct
 * and free or reserved (HR_ERR_PAGE_DUP / HR_ERR_PAGE_IN_USE) and are marked used on success; they may be scored as
 * soon as work enqueued after this call on the same stream runs, or after an event recorded behind it.  Issued on
 * a second stream it overlaps with hr_rerank_score calls that read other pages of the same pool. */
int hr_kv_pages_in(hr_pool* pool, int32_t n_pages, const int32_t* page_ids, const void* src, void* stream);

/* The same with 4-bit records (Section 4.1 names a 4-bit KV cache, KV4W16A16, and Appendix B expands quantised KV
 * to 16 bits after it is loaded; the paper gives no format, this is the library's): the pool stays 16-bit, a page
 * is quantised as it leaves and expanded as it arrives.  16-bit pools only (HR_ERR_UNSUPPORTED_SHAPE otherwise).
 * Per token and per 32 consecutive channels of one (layer, kv head), separately for K and V: scale = amax / 7 in
 * fp32 (1 if all zero), code = x / scale rounded to the nearest integer (ties to even) in [-7, 7]; a loaded page
 * holds code * scale rounded to half.  Record of one page, for every (layer, kv head) in that order:
 *   K codes [16 tokens][head_dim / 2] bytes (channel 2i in the low nibble, 2i + 1 in the high one, two's complement),
 *   V codes likewise, K scales [16][head_dim / 32] fp32, V scales [16][head_dim / 32] fp32
 * = 20 * head_dim bytes per (layer, kv head), 3.2 times smaller than the 16-bit record.  Arguments, memory kinds,
 * page states and errors as for hr_kv_pages_out / hr_kv_pages_in. */
size_t hr_kv_page_record4_bytes(const hr_pool* pool);
int hr_kv_pages_out4(const hr_pool* pool, int32_t n_pages, const int32_t* page_ids, void* dst, void* stream);
int hr_kv_pages_in4(hr_pool* pool, int32_t n_pages, const int32_t* page_ids, const void* src, void* stream);

/* ---- what the 16-bit operand format met ----
 * A 16-bit model computes on IEEE halves: the caller's bf16 weights and bf16 document K/V are converted once, when the
 * weights are packed and when a document is written.  bf16 has the range of fp32, half does not: a magnitude of 65520 or
 * more becomes infinity, and below 2^-14 half is subnormal (a bf16 value below 2^-17 loses bits, below 2^-25 it becomes
 * zero).  The conversions count what they meet, and for fp8 pools the write also counts what the format cannot express:
 *   overflow          values that became infinity (scores that depend on them come out non-finite)
 *   underflow         values that half does not hold exactly (absolute error below 2^-25; random-initialised weights
 *                     always have a few per ten thousand of these)
 *   nonfinite_inputs  NaN or infinity in the caller's data
 *   fp8_nan_codes     E4M3 codes 0x7f / 0xff (NaN; the kernels read them as +-480)
 *   fp8_bad_scales    K or V scales that are not positive and finite, and V scales outside [2^-22, 2^8) (the power of
 *                     two of a V scale is applied while the codes are expanded to half, which covers that range)
 * Activations are not counted: one that exceeds the half range becomes infinity and makes the pair's score non-finite.
 * The report calls copy 64 bytes from the device and wait for the work enqueued so far (not for use in a hot loop).
 * Pages that arrive through hr_kv_pages_in / hr_doc_prefill are not counted (they were halves or codes already). */
typedef struct hr_range_report {
    int64_t overflow, underflow, nonfinite_inputs, fp8_nan_codes, fp8_bad_scales;
    int64_t reserved[3];
} hr_range_report;
int hr_model_range_report(const hr_model* model, hr_range_report* out);      /* since hr_weights_load */
int hr_kv_pool_range_report(const hr_pool* pool, hr_range_report* out);      /* over every hr_doc_kv_write so far */

/* ---- weights ---- */

/* Bytes of device memory for the library's packed copy of the layer weights
 * (fused QKV rows, interleaved gate/up rows); 0 if cfg is invalid. */
size_t hr_weights_pack_bytes(const hr_model_cfg* cfg);

/* Build the packed copy inside caller-owned `pack_dev` (copy kernels on `stream`) and return a
 * handle.  The embedding and the norm gains are borrowed (must outlive the handle); the per-layer
 * matrices may be released once `stream` has drained. */
int hr_weights_load(const hr_model_cfg* cfg, const hr_weight_ptrs* weights,
                    void* pack_dev, size_t pack_bytes, void* stream, hr_model** out);
void hr_model_destroy(hr_model* model);

/* ---- scoring (stage two: only the query suffix is computed) ---- */

/* Workspace bytes for one hr_rerank_score call of this size; 0 on invalid arguments. */
size_t hr_rerank_workspace_bytes(const hr_model* model, int32_t n_pairs, int64_t total_q_tokens,
                                 int32_t pt_stride);

/* scores[p] for p < n_pairs.  For pair p the query tokens sit at positions doc_lens[p] + 0,1,..,
 * attend to all doc_lens[p] cached document keys (found through page_table row p) and causally to
 * the query keys before them; the score is read at the last query token.
 *   page_table    host int32 [n_pairs][pt_stride]; row p lists ceil(doc_lens[p]/16) written pages,
 *                 the rest of the row is ignored (-1 by convention)
 *   doc_lens      host int32 [n_pairs], each >= 0 (0: no cached document, plain causal pass)
 *   query_tokens  host int32, the pairs' query token ids back to back (sum of query_lens entries)
 *   query_lens    host int32 [n_pairs], each >= 1
 *   workspace_dev device scratch, >= hr_rerank_workspace_bytes, 256-byte aligned, private to this
 *                 call until `stream` has drained
 *   scores_dev    device fp32 [n_pairs]
 * The pool is only read.  Host arrays may be reused as soon as the call returns.
 * Pairs of one call whose doc_lens and page-table rows are identical (the same cached document: Section 3.3,
 * pairwise independence makes a document's KV reusable for every query) share one pass over its pages in the
 * attention kernels; the scores are bit for bit those of the pairs scored alone.
 * Pairs of one call with identical query token strings (the same query against several candidates) share the first
 * layer's normalised rows and pre-RoPE q / k / v projections, which are equal for equal strings; each pair's rotation for
 * its own positions doc_lens[p] + i is applied afterwards.  Same bits again.
 * A call with at least 8192 query tokens on the MFMA path whose O / down projection tiles would leave more than 20 % of
 * the device's workgroup slots empty in the rounds they take runs as two halves of the pairs, the first on `stream`,
 * the second on a stream of the library's own that starts behind the work already enqueued on `stream` and that
 * `stream` waits for before anything enqueued after the call (see hr_rerank_set_streams); to the caller the call
 * is ordered on `stream` as if it were one piece of work. */
int hr_rerank_score(hr_model* model, const hr_pool* pool, int32_t n_pairs,
                    const int32_t* page_table, int32_t pt_stride, const int32_t* doc_lens,
                    const int32_t* query_tokens, const int32_t* query_lens,
                    void* workspace_dev, size_t workspace_bytes, float* scores_dev, void* stream);

/* ---- fixed-shape plans: a scoring call whose launches can be recorded once and replayed (Section 4.2: the static
 * [document prefix | query suffix] layout exists so that the reranker's execution can be captured ahead of time) ----
 * A plan fixes the shape of a call: the number of pairs and every pair's document and query length.  Which pages and
 * which query tokens it scores can change between runs.  hr_rerank_plan_run enqueues the kernels, the
 * first of which reads a pinned block that the plan owns over the bus (plans of more than 1024 query tokens or 64 KiB of
 * metadata: behind a host-to-device copy of that block); it never waits on the host, allocates nothing and uses `stream` only,
 * so it may be recorded into a HIP graph (stream capture) and replayed.  The work of a plan depends on the lengths
 * alone: pairs are not regrouped by shared documents or shared query strings as hr_rerank_score does, which changes no
 * score bit.
 *   hr_rerank_plan_create      host: checks the lengths, carves `workspace_dev` (>= hr_rerank_workspace_bytes for these
 *                              sizes, private to the plan while it lives) and allocates the pinned metadata block (the one
 *                              allocation of a plan's life).  Uses the model's split-operand setting at this moment.
 *   hr_rerank_plan_set_inputs  host: validates page_table [n_pairs][pt_stride] and query_tokens (flat, pair after pair)
 *                              like hr_rerank_score and writes them into the pinned block.  A run or replay reads
 *                              that block when it executes: do not call this while a run or replay that has not
 *                              finished could still read the block.
 *   hr_rerank_plan_run         stream work only (see above); scores_dev fp32 [n_pairs].  HR_ERR_INVALID_ARG before the
 *                              first set_inputs.  Run it once outside capture first: the first launch of a kernel sets
 *                              its function attributes.
 * Plans of one model share its kernels but no state; a plan must not outlive its model, pool or workspace. */
typedef struct hr_plan hr_plan;
int hr_rerank_plan_create(hr_model* model, const hr_pool* pool, int32_t n_pairs, const int32_t* doc_lens,
                          const int32_t* query_lens, int32_t pt_stride, void* workspace_dev, size_t workspace_bytes,
                          hr_plan** out);
int hr_rerank_plan_set_inputs(hr_plan* plan, const int32_t* page_table, const int32_t* query_tokens);
int hr_rerank_plan_run(hr_plan* plan, float* scores_dev, void* stream);
void hr_rerank_plan_destroy(hr_plan* plan);

/* hr_rerank_score for callers that cannot allocate or hand over a workspace: code under HIP graph capture, tight
 * serving loops, harnesses that forbid hipMalloc.  Same arguments, validation, kernels and scores (bit for bit) as
 * hr_rerank_score, except that the workspace is a file-scope device array inside the library
 * (hr_rerank_static_scratch_bytes() = 128 MiB; every GPU the library runs on holds its own copy until the process ends)
 * and the per-call metadata goes through the pinned staging buffer the model handle got at hr_weights_load (1 MiB).
 * The call allocates nothing: no device or pinned memory, no streams, no events; it always runs in one piece on `stream`,
 * and per-kernel timing (hr_profile_enable) is off for its duration.
 *   HR_ERR_WORKSPACE_SMALL  the call would need more scratch than the array holds, or more metadata than the staging
 *                           buffer holds (hr_last_error says which and how much); nothing is enqueued.  One query with
 *                           20 candidates of 32 query tokens needs about 13 MiB at the 0.5B shape and 85 MiB at the 8B shape.
 * The array is shared by every static call on that GPU, whatever the model handle, and keeps the last call's contents
 * (what must start at zero is cleared by the call itself): static calls that overlap in time on one GPU race with each
 * other, also when issued on different streams.  Order them on one stream or with events. */
size_t hr_rerank_static_scratch_bytes(void);
int hr_rerank_score_static(hr_model* model, const hr_pool* pool, int32_t n_pairs,
                           const int32_t* page_table, int32_t pt_stride, const int32_t* doc_lens,
                           const int32_t* query_tokens, const int32_t* query_lens,
                           float* scores_dev, void* stream);

/* Precision of the scoring pass on the MFMA kernels (16-bit models).  Operands of the matrix instructions are IEEE halves
 * (11 significant bits): weights and cached document K/V are exact as halves, but every activation that feeds an MFMA is
 * rounded once per layer, and a deep, wide network amplifies the first layers' roundings most (Section 3.3 calls the
 * cached pass lossless; the arithmetic's own rounding is what is left).  The first `n_layers` layers of hr_rerank_score
 * therefore can run with split operands: each such activation is carried as a pair of halves hi + lo (22 bits) and every
 * product with a lo term is one more MFMA chain into the same fp32 accumulator, about twice the work of those layers.
 *   n_layers   0 .. model layers, or -1 for the default: 2 when layers x hidden >= 65536 (the 8B shape), else 0
 * Changes hr_rerank_workspace_bytes (ask again after setting it).  hr_rerank_score_full and hr_doc_prefill always run
 * with plain 16-bit operands.  HR_ERR_UNSUPPORTED_SHAPE if n_layers > 0 on a model that runs the generic kernels
 * (those compute in fp32 throughout). */
int hr_model_set_precise_layers(hr_model* model, int n_layers);
int hr_model_precise_layers(const hr_model* model);

/* 1: scoring calls use the caller's stream only; 2 (the default): large calls are cut in two halves that run on
 * two streams, so that one half's kernels fill the compute units that the last, partly filled round of the other
 * half's GEMM tiles leaves idle (pairs are independent, Section 3.3: the scores do not change by a bit).
 * HR_ERR_INVALID_ARG for other values. */
int hr_rerank_set_streams(hr_model* model, int n_streams);

/* In how many parts (1 or 2) a scoring call with this many query tokens runs on the current device, given at least two
 * pairs and a model / pool combination on the MFMA kernels; a negative status on invalid arguments.  For reporting. */
int hr_rerank_parts(const hr_model* model, int64_t total_q_tokens);

/* The host-side checks hr_rerank_score performs before it enqueues anything, on their own: no
 * device work, no model handle needed.  Returns HR_OK or the status hr_rerank_score would return
 * for these arguments (lengths, page-table rows, page states, token ids, pool/model agreement). */
int hr_rerank_validate(const hr_model_cfg* cfg, const hr_pool* pool, int32_t n_pairs,
                       const int32_t* page_table, int32_t pt_stride, const int32_t* doc_lens,
                       const int32_t* query_tokens, const int32_t* query_lens);

/* ---- same-GPU reference without reuse: full prefill of [document ; query] per pair ---- */
/* (Section 3.3 "Potential 1": what the scoring pass is compared with.) */
size_t hr_rerank_full_workspace_bytes(const hr_model* model, int32_t n_pairs, int64_t total_tokens);

/* scores[p] from one causal pass over the concatenation of doc_tokens and query_tokens of pair p;
 * no pool is involved.  doc_tokens / query_tokens are flat host int32 arrays, pair after pair.
 * A sequence may hold up to 32768 tokens on the MFMA kernels (15000 on the generic ones): HR_ERR_LEN_RANGE beyond. */
int hr_rerank_score_full(hr_model* model, int32_t n_pairs,
                         const int32_t* doc_tokens, const int32_t* doc_lens,
                         const int32_t* query_tokens, const int32_t* query_lens,
                         void* workspace_dev, size_t workspace_bytes, float* scores_dev, void* stream);

/* ---- document prefill (stage one of the two-stage inference, Section 3.3 Property 1) ---- */

/* Workspace bytes for hr_doc_prefill; 0 if the model / shape is not covered (see hr_doc_prefill). */
size_t hr_doc_prefill_workspace_bytes(const hr_model* model, int32_t n_docs, int64_t total_tokens);

/* Run n_docs documents alone through the layers (positions 0..len-1, causal) and store every layer's post-RoPE
 * K and V in the pool pages the caller names, ready for hr_rerank_score.  Same kernels as the scoring pass: a
 * document is processed as chunks of 64 tokens whose prefix is the document's own earlier pages.
 *   doc_tokens  host int32, the documents' token ids back to back
 *   doc_lens    host int32 [n_docs], each 1 .. 32768
 *   page_table  host int32 [n_docs][pt_stride]; row d names ceil(doc_lens[d]/16) distinct free (or reserved) pages
 * 16-bit and fp8 pools, MFMA-covered models only (HR_ERR_UNSUPPORTED_SHAPE otherwise).  For an fp8 pool every page
 * is quantised as it is stored: per (layer, page, kv head) and separately for K and V, scale = amax / 448 over the page
 * (1 if amax = 0) in fp32, code = the E4M3 value nearest to x / scale (ties to the even code).  Pages are marked used on
 * success.  Work is enqueued on `stream`. */
int hr_doc_prefill(hr_model* model, hr_pool* pool, int32_t n_docs, const int32_t* doc_tokens, const int32_t* doc_lens,
                   const int32_t* page_table, int32_t pt_stride, void* workspace_dev, size_t workspace_bytes, void* stream);

/* ---- per-query selection (what the pipeline does with the scores: Section 3.1, "select top-k"; Table 1 reranks
 * 5 / 10 / 20 candidates down to the best one) ---- */

/* For each query the k best of its candidates, best first: score descending, candidate index ascending among equal
 * scores (-0 equals +0; NaN ranks below every number).
 *   scores_dev   device fp32, the scores of all pairs (what hr_rerank_score wrote)
 *   seg_dev      device int32 [n_queries + 1], ascending: query i owns pairs seg[i] .. seg[i+1]-1
 *   max_cands    host int, an upper bound of seg[i+1] - seg[i] (1 .. 4096); a longer segment is cut to its first
 *                max_cands candidates
 *   k            1 .. max_cands
 *   topk_idx_dev device int32 [n_queries][k]: candidate index inside the query's segment, -1 where the query has
 *                fewer than k candidates
 *   topk_scores_dev  optional (may be NULL) device fp32 [n_queries][k], 0 where the index is -1
 * Nothing is allocated; work is enqueued on `stream`; n_queries = 0 is a no-op.  HR_ERR_INVALID_ARG on null
 * pointers or sizes out of range. */
int hr_rerank_topk(const float* scores_dev, const int32_t* seg_dev, int32_t n_queries, int32_t max_cands, int32_t k,
                   int32_t* topk_idx_dev, float* topk_scores_dev, void* stream);
/* The same with the offsets in host memory: they travel as kernel arguments, so there is no copy to wait for and the array
 * may be reused as soon as the call returns. */
int hr_rerank_topk_host(const float* scores_dev, const int32_t* seg_offsets, int32_t n_queries, int32_t max_cands, int32_t k,
                        int32_t* topk_idx_dev, float* topk_scores_dev, void* stream);

/* ---- operators of a layer, for models whose layers the caller runs ----
 * hr_rerank_score runs the layers of one kind of decoder.  A model with other positions, masks or score functions can still
 * keep its documents in a pool and run its own projections: these calls give it rotary positions (a pool's K is post-RoPE), the
 * tables of a batch of pairs, built on the device, and the attention of the pairs' query tokens over their documents' pages.
 * None of them allocates, waits on the host or keeps anything between calls; all may be recorded into a HIP graph.  None has a backward pass. */

/* Rotary positions.  The leading rotary_dim channels of every head are turned in rotary_dim / 2 pairs: pair i of a token at
 * position p by the angle p * freqs[i]:  a' = a cos - b sin, b' = b cos + a sin; the other channels stay as they are.
 *   HR_ROPE_HALF         pair i is channels i and i + rotary_dim / 2 (what hr_rerank_score and hr_doc_prefill apply)
 *   HR_ROPE_INTERLEAVED  pair i is channels 2 i and 2 i + 1
 * Frequencies f_i = base^(-2 i / rotary_dim), for contexts longer than the original_len a model was trained on:
 *   HR_ROPE_SCALE_NONE    f_i
 *   HR_ROPE_SCALE_LINEAR  f_i / factor
 *   HR_ROPE_SCALE_BASE    with base * factor^(rotary_dim / (rotary_dim - 2)) in place of base (rotary_dim > 2)
 *   HR_ROPE_SCALE_BANDS   by the pair's full turns over the original context, n_i = original_len f_i / 2 pi: f_i / factor up to
 *                         `low` turns, f_i from `high` turns on, between them in proportion to n_i
 *   HR_ROPE_SCALE_RAMP    in proportion to the index i instead, between the indices (rounded outwards, within the head) at
 *                         which n_i passes `high` and `low` */
typedef enum hr_rope_layout { HR_ROPE_HALF = 0, HR_ROPE_INTERLEAVED = 1 } hr_rope_layout;
typedef enum hr_rope_scale {
    HR_ROPE_SCALE_NONE = 0, HR_ROPE_SCALE_LINEAR = 1, HR_ROPE_SCALE_BASE = 2, HR_ROPE_SCALE_BANDS = 3, HR_ROPE_SCALE_RAMP = 4
} hr_rope_scale;
typedef struct hr_rope_cfg {
    int32_t head_dim;      /* 2 .. 1024 */
    int32_t rotary_dim;    /* even, 2 .. min(head_dim, 256) */
    int32_t layout;        /* hr_rope_layout */
    int32_t scaling;       /* hr_rope_scale */
    float amplitude;       /* factor on the rotated channels, positive and finite; 1 unless the scaling wants another */
    float base;            /* > 1 */
    float factor;          /* >= 1; read by every scaling but NONE */
    float original_len;    /* BANDS, RAMP: positive */
    float low, high;       /* BANDS, RAMP: 0 < low < high */
} hr_rope_cfg;
/* The frequencies of cfg in radians per position, freqs_out[rotary_dim / 2] (host).  A caller may pass others of its own to
 * hr_rope_apply. */
int hr_rope_frequencies(const hr_rope_cfg* cfg, double* freqs_out);

/* One tensor [n_tokens][n_heads][head_dim]: the channels of a head follow each other, strides are in elements.  out may be
 * `in` itself (then with the same strides) and must not overlap it otherwise. */
typedef struct hr_rope_tensor {
    const void* in;        /* device */
    void* out;             /* device */
    int32_t n_heads;
    int64_t in_token_stride, in_head_stride, out_token_stride, out_head_stride;
} hr_rope_tensor;
/* Rotates up to two tensors (q and k) of n_tokens tokens in one launch.
 *   freqs          host, [rotary_dim / 2], each in [0, 2 pi)
 *   dtype          HR_F32 or HR_BF16; angles are reduced in 64 bits, products are fp32, rounded once
 *   positions_dev  device int32 [n_tokens]; a token with a negative position is left out: its rows of `out` are not written.
 *                  NULL: token t is at first_position + t % period (period 0: first_position + t), which may not pass 2^31 - 1
 *   inverse        not 0: by the negative angles (takes the rotation back; amplitude multiplies again)
 * HR_ERR_INVALID_ARG on null pointers, bad configurations, frequencies or strides, and if one tensor's `out` is the other's `in` or
 * `out`; HR_ERR_LEN_RANGE beyond 2^30 tokens or what a launch can hold (2^24 workgroups of four wavefronts, each with the tokens whose
 * heads fill its lanes); n_tokens = 0 is a no-op. */
int hr_rope_apply(const hr_rope_cfg* cfg, const double* freqs, int dtype, int64_t n_tokens, const int32_t* positions_dev,
                  int32_t first_position, int32_t period, const hr_rope_tensor* tensors, int32_t n_tensors, int inverse, void* stream);

/* The documents a batch may ask for, in device memory: document i has doc_lens[i] tokens in the pages
 * pages[page_cu[i]], pages[page_cu[i] + 1], .. */
typedef struct hr_doc_list {
    int32_t n_docs;
    int32_t n_pages;             /* entries of pages */
    const int32_t* doc_lens;     /* [n_docs] */
    const int32_t* page_cu;      /* [n_docs + 1], ascending */
    const int32_t* pages;        /* [n_pages] */
} hr_doc_list;

/* What a batch of pairs needs on the device; all arrays are the caller's device memory.  max_tokens: room for the pairs'
 * query tokens (rows behind the last one belong to nobody). */
typedef struct hr_pair_tables {
    int32_t n_pairs, max_tokens, pt_stride;
    int32_t n_q_heads;      /* of the model, a multiple of the pool's n_kv_heads */
    int32_t* q_cu;          /* [n_pairs + 1]: pair p has the tokens q_cu[p] .. q_cu[p + 1] - 1 */
    int32_t* doc_lens;      /* [n_pairs] */
    int32_t* page_table;    /* [n_pairs][pt_stride]: -1 behind the document's last page */
    int32_t* tok_pos;       /* [max_tokens]: position doc_lens[p] + i of token i of pair p; -1 behind the last token */
    int32_t* tok_pair;      /* [max_tokens]: its pair; -1 likewise */
    int32_t* order;         /* [n_pairs]: the pairs by document (those without one first), in their order among equals */
    int32_t* report;        /* [4]: tokens, distinct documents (all pairs without one count as one), HR_TABLES_* bits, 0 */
    void* sched;            /* hr_pair_tables_sched_bytes, 16-byte aligned: the attention's work list (private) */
    size_t sched_bytes;
} hr_pair_tables;
#define HR_TABLES_BAD_DOC 1      /* a document id below -1 or >= n_docs: the pair has no document */
#define HR_TABLES_BAD_LENGTH 2   /* a negative query length, counted as 0, or one cut because max_tokens was reached */
#define HR_TABLES_CUT 4          /* a document longer than its entries of the page list or than pt_stride pages: cut to them */
#define HR_TABLES_BAD_PAGE 8     /* a page id outside the pool: -1 in page_table; such a pair's attention is undefined */

/* Bytes of hr_pair_tables.sched; 0 on invalid arguments. */
size_t hr_pair_tables_sched_bytes(const hr_pool* pool, int32_t n_pairs, int32_t max_tokens, int32_t n_q_heads);
/* Fills the tables from pair_doc_dev (device int32 [n_pairs]: a document, -1 for none) and query_lens_dev (device int32
 * [n_pairs], 0 and more).  Nothing comes back to the host: what is wrong with the contents is mended as the bits above say and
 * noted in report, and no table leads outside the pool, the page list or max_tokens.  Whether pages hold a document (hr_doc_kv_write)
 * is not checked.  HR_ERR_INVALID_ARG on null pointers and bad sizes, HR_ERR_LEN_RANGE for more than 2^30 pairs or rows of a kv head (max_tokens
 * times the heads of one) or 2^26 pages a document, HR_ERR_WORKSPACE_SMALL for sched_bytes;
 * n_pairs = 0 is a no-op. */
int hr_pair_tables_build(const hr_pool* pool, const hr_doc_list* docs, const int32_t* pair_doc_dev, const int32_t* query_lens_dev,
                         const hr_pair_tables* out, void* stream);

/* Attention of a batch of pairs at one layer.  A query token i of a pair (position D + i behind its document of D tokens) and
 * query head a have, for every key they see,
 *   s = scale q . k;  cap > 0: s = cap tanh(s / cap);  slopes: s -= slopes[a] |distance of the positions|
 * and out = sum softmax(s) v.  Keys are the document's, from the pool, and, with k and v, the pair's own: token j at position
 * D + j is seen by token i if j <= i (causal) or j < prefix_lens[p] (the first tokens of a query, seen by all of it).  window
 * w > 0: only keys less than w positions behind the query token.  A row that sees nothing is 0 (and its lse -infinity).  What is
 * not seen does not count, whatever it holds.
 * Pairs that share a document share one pass over its pages, whatever their order in the batch.
 *   dtype         of q, k, v and out: HR_BF16 with 16-bit and fp8 pools, HR_F32 with fp32 pools (HR_ERR_MISMATCH otherwise).
 *                 bf16 values are multiplied as halves (exact for magnitudes in [2^-14, 65504], as hr_doc_kv_write keeps them; smaller
 *                 ones lose digits, larger ones are infinite), and the weights of V are rounded to half (by 2^-11 of a weight, or
 *                 2^-25 of the row's largest); in fp32 where the head size is none of 64, 96 and 128.  Maxima, sums and the joins are fp32
 *   q, out        device [max_tokens][n_q_heads][head_dim]; k, v: [max_tokens][n_kv_heads][head_dim], both or neither; strides in
 *                 elements, channels of a head follow each other.  Rows behind the last token are neither read nor written.  out and
 *                 lse overlap none of the inputs (HR_ERR_INVALID_ARG where they begin where one of those does)
 *   lse           NULL or device fp32 [max_tokens][n_q_heads]: natural logarithm of the row's sum of exp(s)
 *   slopes        NULL or device fp32 [n_q_heads];  prefix_lens: NULL or device int32 [n_pairs] (cut to the query's length)
 * tables come from hr_pair_tables_build with the same pool, ahead of the call on its stream; n_q_heads is theirs.  HR_ERR_LEN_RANGE
 * if the work list has room for more than some 2^24 blocks of 32 rows (max_tokens x heads of a kv head / 32, and a block for every pair, times the kv heads). */
typedef struct hr_attention_args {
    int32_t dtype, layer;
    float scale;            /* finite; 0: 1 / sqrt(head_dim) */
    float cap;              /* 0 (none) or 1e-18 .. 1e18 */
    int32_t window;         /* 0 (none) or the number of positions */
    const void *q, *k, *v;
    void* out;
    float* lse;
    const float* slopes;
    const int32_t* prefix_lens;
    int64_t q_token_stride, q_head_stride, k_token_stride, k_head_stride, v_token_stride, v_head_stride, out_token_stride, out_head_stride;
} hr_attention_args;
/* Workspace of one call; may be 0.  It is private to the call until `stream` has drained.  It goes by the tables' room (n_pairs, max_tokens,
 * pt_stride), and so does the number of pieces that a long document's keys can be cut into where there are few rows: room for many tokens leaves few. */
size_t hr_pair_attention_workspace_bytes(const hr_pool* pool, const hr_pair_tables* tables);
int hr_pair_attention(const hr_pool* pool, const hr_pair_tables* tables, const hr_attention_args* args, void* workspace_dev,
                      size_t workspace_bytes, void* stream);

/* ---- a layer's projections in 8 bits, for models whose layers the caller runs ----
 * The norm in front of a projection, with the residual's addition, and the projection itself on 8-bit operands, with what follows it:
 *   hr_rms_norm (codes of x)  ->  hr_block_matmul (gate; codes)  ->  hr_block_matmul (adds onto the stream)  ->  hr_rms_norm ..
 * None of these calls allocates, waits on the host or keeps anything between calls; all may be recorded into a HIP graph.  None has a backward pass. */

/* A matrix in 8 bits: E4M3 codes and fp32 scales, value = decode(code) * scale.  One scale for 128 consecutive columns (the last block has what
 * is left) of block_rows rows: 1 for activations, 128 for weights.
 * Codes made here: scale = amax / 448 over the block's finite values, at least 2^-126 (1 if amax = 0); code = the E4M3 value nearest to
 * x * (1 / scale), ties to the even code (x / scale gives its neighbour now and then, where that lies within 2^-23 of a tie); a value that is not finite becomes
 * a code NaN (0x7f or 0xff). */
#define HR_BLOCK_COLS 128
typedef struct hr_block8 {
    void* codes;            /* device, 16-byte aligned */
    float* scales;          /* device, [ceil(rows / block_rows)][ceil(cols / 128)] */
    int64_t rows;           /* 0 .. 2^30 */
    int32_t cols;           /* 1 .. 2^22 */
    int32_t block_rows;     /* 1 or 128 */
    int64_t row_stride;     /* bytes from row to row, a multiple of 16, at least cols, at most 2^22.  What lies between a row's last code and the next
                             * multiple of 16 may be read (and does not count, whatever it holds) and is not written */
    int64_t scale_stride;   /* floats from one row of scales to the next, at least ceil(cols / 128), at most 2^20 */
} hr_block8;

/* Root-mean-square norm of every head of every token, after an addition:
 *   s = x + add;   y = s / sqrt(mean(s^2) + eps) * (gain + gain_offset)
 * over the head's channels.  total receives s (the residual stream), out receives y, block8 receives y as codes; all from the fp32 values, which
 * are rounded once.  Sums are fp32: a head whose squares pass 3.4e38 comes out as 0.  Heads of any small size down to fp32's least value are summed to the same
 * digits (their squares scaled where they would be below fp32's range).  A head of zeros is 0 with eps = 0 too.
 * Any of total, out and block8 may be left out, not all.  total and out may be x or add (then with the same strides) and share no memory
 * otherwise (HR_ERR_INVALID_ARG where outputs begin at the same place, or one begins where an input with other strides, gain or codes do). */
typedef struct hr_norm_args {
    int32_t dtype;            /* of x, add, total and out: HR_F32 or HR_BF16 */
    int32_t heads;            /* 1 .. 65536; 1 with block8 */
    int32_t channels;         /* 1 .. 65536; adjacent */
    float eps;                /* finite, 0 or more */
    float gain_offset;        /* finite: 0, or 1 where gains are kept as their distance from 1 */
    int64_t tokens;           /* 0 .. 2^30 */
    const void *x, *add;      /* device [tokens][heads][channels]; add: NULL or the same */
    void *total, *out;        /* device or NULL */
    const float* gain;        /* device [channels], or NULL: 1 - gain_offset */
    const hr_block8* block8;  /* NULL, or block_rows 1, rows = tokens, cols = channels (host struct, read during the call) */
    int64_t x_token_stride, x_head_stride, add_token_stride, add_head_stride;              /* in elements */
    int64_t total_token_stride, total_head_stride, out_token_stride, out_head_stride;
} hr_norm_args;
/* HR_ERR_INVALID_ARG on null pointers, bad sizes, strides and overlaps as above, HR_ERR_MISMATCH if block8 has another shape, HR_ERR_LEN_RANGE beyond
 * 2^30 tokens; tokens = 0 is a no-op. */
int hr_rms_norm(const hr_norm_args* args, void* stream);

/* Codes and scales of x, device [rows][cols] of dtype (HR_F32 or HR_BF16), rows x_stride elements apart: rows of activations (out->block_rows 1)
 * or weights (128).  HR_ERR_INVALID_ARG on null pointers and bad matrices, HR_ERR_LEN_RANGE beyond 2^24 - 512 tiles of 128 x 128; rows = 0 is a no-op. */
int hr_block_quantize(int dtype, const void* x, int64_t x_stride, const hr_block8* out, void* stream);

/* c[m][n] = sum over the blocks b of 128 columns of  a.scale[m][b] w.scale[n / 128][b] (sum over k in b of a[m][k] w[n][k])  + bias[n], then
 *   HR_GATE_NONE   y = c
 *   HR_GATE_SILU   y[m][f] = silu(c[m][f]) c[m][F + f] with F = w->rows / 2 (a multiple of 128): the weights' first half is the gate
 *   HR_GATE_GELU   the same with gelu(z) = z / 2 (1 + tanh(sqrt(2 / pi) (z + 0.044715 z^3)))
 * and out = y + add, rounded once; or block8 = codes and scales of y.
 * a: activations (block_rows 1), w: weights (block_rows 128) with as many columns.  Sums over k and over blocks are fp32, and so is a.scale w.scale, which is
 * formed first: scales whose product passes 3.4e38 give infinities and NaN.  Codes are multiplied as halves, exactly, so that nothing but fp32 additions
 * rounds a sum, whatever the result's type.
 * fast: products may be summed by the 8-bit instruction, at up to 1.8 times the speed, where the tile that M, N and K lead to has it (most have; those
 * for a few rows may not, so that a row alone and the same row in a batch can differ by what it rounds).  It adds the products of columns 8 i .. 8 i + 7 of a block at
 * once, each cut off at 2^-13 of the power of two of the largest of them: 7 * 2^-13 of that product at most for every eight columns.  Over normal deviates that is
 * 1.4e-5 of a row's rms; where large terms cancel it can be more than what is left, in bf16 too.
 * out may be add (then with the same stride).  HR_ERR_INVALID_ARG on null pointers, bad matrices, strides and overlaps (out, add, the codes and
 * scales of block8 and those of a and w begin at places of their own); HR_ERR_MISMATCH if a and w differ in columns, block8 from y's shape or a gate's half is no multiple
 * of 128; HR_ERR_LEN_RANGE beyond 2^22 - 512 tiles (the smallest, for a few rows, have 16 x 16 values); no rows of a or of w: a no-op. */
typedef enum hr_gate { HR_GATE_NONE = 0, HR_GATE_SILU = 1, HR_GATE_GELU = 2 } hr_gate;
typedef struct hr_matmul_args {
    int32_t dtype;            /* of out and add: HR_F32 or HR_BF16 */
    int32_t gate;             /* hr_gate */
    int32_t fast;             /* 0: fp32 sums; not 0: sums by the 8-bit instruction (see above) */
    const float* bias;        /* NULL or device [w->rows] */
    const void* add;          /* NULL or device [a->rows][columns of y]; not with block8 */
    void* out;                /* device, likewise; NULL with block8 */
    int64_t add_stride, out_stride;     /* elements from row to row */
    const hr_block8* block8;  /* NULL, or block_rows 1 and y's shape (host struct, read during the call) */
} hr_matmul_args;
int hr_block_matmul(const hr_block8* a, const hr_block8* w, const hr_matmul_args* args, void* stream);

/* ---- introspection for benchmarks ---- */

/* Per-kernel timing for benchmarks.  While enabled, every kernel launch of a scoring call is
 * bracketed by two HIP events on the call's stream, tagged with a kernel class (hr_profile_name:
 * "gemm_gate_up", "attention", ...; hr_profile_count classes).  hr_profile_read waits for the
 * recorded events, returns per class the summed duration in ms and the number of launches
 * (arrays of hr_profile_count entries, host) and clears the record. */
int hr_profile_enable(hr_model* model, int enable);
/* Restrict the timing to the classes whose bit (1 << class index) is set; the default is all classes.  Two
 * event records cost a few microseconds of stream time per launch, which adds up over ~170 launches per call,
 * so a benchmark times only the classes it reports while it measures the whole call. */
int hr_profile_select(hr_model* model, uint32_t class_mask);
int hr_profile_count(void);
const char* hr_profile_name(int idx);
int hr_profile_read(hr_model* model, double* ms_out, int64_t* launches_out);

/* A yardstick for the roofline of the KV-streaming attention (which is bound by reading HBM): one read-only pass over
 * `bytes` (whole KiB are read) of device memory at src_dev (16-byte aligned) with a kernel of the library's own, enqueued
 * on `stream`; time it from outside.  to_lds = 0: 16-byte loads into registers; 1: the direct-to-LDS loads the attention
 * kernel streams pages with.  sink_dev: >= 4 bytes of device memory that receive a fold of what was read (so that no load
 * can be dropped).  HR_ERR_INVALID_ARG on null or misaligned pointers or bytes < 1024. */
int hr_probe_read_bandwidth(const void* src_dev, size_t bytes, void* sink_dev, size_t sink_bytes, int to_lds, void* stream);

/* Name of the kernel family a model / pool combination runs; never NULL:
 *   "mfma"     16-bit models on the half matrix instructions
 *   "f32"      fp32 models with heads of 16, 32 or 64 channels: the fused pass on the fp32 matrix instruction
 *   "generic"  everything else, step by step (projections on the fp32 matrix instruction, the rest on the vector units)
 *   "none"     a null handle
 * The MFMA attention is only chosen together with the MFMA projections.  hr_attention_path answers for short
 * queries.  One attention work item holds 512 rows (query tokens x query heads per kv head) at 64-wide heads and 256 at
 * 128-wide heads; a scoring call spreads a longer query's rows over up to eight work items (each streams the document),
 * and beyond that (or with HR_NO_DOC_GROUPS=1, which switches the plan off that does the spreading) runs its attention on
 * the generic kernel next to the MFMA projections: same results within the tolerance of the model's dtype, and a
 * document plus query of at most 15000 tokens. */
const char* hr_attention_path(const hr_model* model, const hr_pool* pool);
const char* hr_gemm_path(const hr_model* model);

/* Environment switches, read once per model handle at hr_weights_load.  They exist for A/B runs of the tests and
 * benchmarks (each pair of settings must give the same score bits) and change no result:
 *   HR_NO_LAST_SHORTCUT=1   the last layer runs on every token instead of each pair's last one
 *   HR_NO_DOC_GROUPS=1      pairs that share a document are not batched into one attention work item
 *   HR_NO_QUERY_SHARING=1   the first layer's projections are computed for every pair instead of once per distinct query
 *   HR_STREAMS=1            the initial value of hr_rerank_set_streams is 1
 * and two that do change results (within the tolerance):
 *   HR_FORCE_GENERIC=1      every step on the step-by-step kernels (fp32 arithmetic)
 *   HR_PRECISE_LAYERS=n     the initial value of hr_model_set_precise_layers */

#ifdef __cplusplus
}
#endif
#endif /* HYPERRERANK_H */
