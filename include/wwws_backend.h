/*
 * wwws backend: the operators of a provider that answers the requests the network dispatched to it.
 *
 * The network of wwws.h treats a provider as a rate (cap_true_tok_s) and a hidden quality; the paper's node hands
 * the request to a Model Manager (Section "Request Routing and Node Design").  These calls are the
 * parts of such a backend that touch every generated token and are not plain matrix products:
 *   wwws_cache_append / wwws_cache_read   keys and values of new tokens into a paged cache (as given, int8 or e4m3),
 *                                         and whole sequences back out of it (to hand a request to another peer)
 *   wwws_attend                           attention of new tokens over the paged cache: one token per sequence,
 *                                         a few drafted ones, a chunk of a prompt, whole prompts; optional sliding
 *                                         window with a few first tokens that stay visible
 *   wwws_shape_logits                     repetition, presence and frequency penalties, biases and grammar masks on
 *                                         logits, and the token that a temperature of zero picks;
 *                                         a judge's verdict is a row whose mask leaves the verdict tokens
 *
 * Conventions are those of wwws.h: every call returns a wwws_status and never aborts; all device work is enqueued on
 * the stream given at creation and is asynchronous (wwws_backend_sync and wwws_destroy_backend synchronise it); the
 * library allocates no device memory (one workspace from the caller); "HOST" / "DEVICE" say where a pointer points;
 * a handle is not thread-safe and lives on the GPU that holds its workspace.  Arrays handed to a call must stay valid
 * until the stream has passed it, and must have been written by work that the stream waits for.
 * Ids read from device memory (pages, tokens, masks, offsets) are range-checked by the kernels: a bad one is skipped
 * (a page outside the pool reads as hidden keys and is not written) and reported by the next wwws_backend_sync.
 */
#ifndef WWWS_BACKEND_H
#define WWWS_BACKEND_H

#include "wwws.h"

#ifdef __cplusplus
extern "C" {
#endif

typedef struct wwws_backend wwws_backend; /* opaque */

typedef enum { WWWS_BF16 = 0, WWWS_F16 = 1, WWWS_F32 = 2 } wwws_dtype;
typedef enum {
    WWWS_CACHE_16 = 0,  /* elements of the backend's dtype */
    WWWS_CACHE_INT8 = 1,/* int8 codes, one fp32 scale per (token, kv head): value = code * scale */
    WWWS_CACHE_E4M3 = 2 /* 8-bit floats with 4 exponent bits (finite range 448), scales as above */
} wwws_cache_kind;

/* Plain data, copied at creation.  n_heads = 0: a backend for wwws_shape_logits alone (the cache fields are not read). */
typedef struct {
    uint32_t n_heads;    /* query heads, a multiple of n_kv_heads; query head h reads kv head h / (n_heads / n_kv_heads) */
    uint32_t n_kv_heads; /* n_heads / n_kv_heads <= 16 */
    uint32_t head_dim;   /* 64 or 128 */
    uint32_t page_tokens;/* tokens of a page: 16, 32, 64 or 128 */
    uint32_t n_pages;    /* pages of the pool; n_pages * n_kv_heads * page_tokens < 2^31 */
    uint32_t max_seqs;   /* sequences of one call, 1 .. 2048 */
    uint32_t max_tokens; /* new tokens of one call, < 2^27 */
    uint32_t max_pages;  /* columns of a page table, max_pages * page_tokens < 2^30 */
    uint32_t max_rows;   /* logits rows of one call, 0 .. 65535 */
    uint32_t dtype;      /* WWWS_BF16 or WWWS_F16: queries, keys, values, outputs */
    uint32_t cache;      /* wwws_cache_kind */
} wwws_backend_config;

/* DEVICE page pool, caller-owned, 16-byte aligned: k and v [n_pages][n_kv_heads][page_tokens][head_dim] of the cache's
 * element, scales [n_pages][n_kv_heads][page_tokens] (NULL with WWWS_CACHE_16).  One pool per layer of a model. */
typedef struct { void* k; void* v; float* k_scale; float* v_scale; } wwws_kv_pages;

/* One step's sequences.  The arrays are DEVICE and caller-owned; the counts are HOST bounds that size the launches: a
 * sequence that exceeds them is skipped and reported.  New token t of sequence i is row q_start[i] + t of the call's
 * arrays and token kv_len[i] - q_len + t of the sequence (q_len = q_start[i + 1] - q_start[i]); a token whose place
 * would be negative is not written and sees nothing. */
typedef struct {
    const int32_t* q_start;    /* [n_seqs + 1], q_start[0] = 0, nondecreasing, q_start[n_seqs] = n_tokens */
    const int32_t* kv_len;     /* [n_seqs] tokens of the sequence, the new ones included, <= max_kv_len */
    const int32_t* page_table; /* [n_seqs][max_pages of the configuration] page of each page_tokens tokens */
    uint32_t n_seqs, n_tokens, max_q_len, max_kv_len;
} wwws_batch;

/* Bytes of device workspace a backend with this configuration needs. */
wwws_status wwws_backend_workspace_bytes(const wwws_backend_config* cfg, uint64_t* bytes_out);

/* Build a backend in `workspace` (DEVICE, 256-byte aligned); `cuda_stream` is a cudaStream_t (NULL = default stream).
 * The library keeps the workspace until wwws_destroy_backend; the caller frees it afterwards. */
wwws_status wwws_create_backend(const wwws_backend_config* cfg, void* workspace, uint64_t workspace_bytes,
                                void* cuda_stream, wwws_backend** out);
wwws_status wwws_destroy_backend(wwws_backend* b);

/* Write the batch's new keys and values to their pages.  k and v: [n_tokens][n_kv_heads][head_dim] of the backend's
 * dtype, 16-byte aligned, `stride` elements from one token to the next (a multiple of 8: slices of a joint projection
 * are fine).  Quantised kinds, per (token, kv head) and in fp32: amax = max |x|, scale = amax * fp32(1 / top) with top
 * 127 or 448, code = x * (1 / scale) rounded to nearest even and clamped to +-top.  amax < 2^-100: scale 0, codes 0.
 * A row that holds a NaN or an infinity: scale NaN, codes 0, so it reads back as NaN wherever it is visible. */
wwws_status wwws_cache_append(wwws_backend* b, const wwws_batch* batch, const wwws_kv_pages* pages, const void* k,
                              uint64_t k_stride, const void* v, uint64_t v_stride);

/* Read whole sequences back: token t of sequence i to row row_start[i] + t of k_out and v_out ([n_rows][n_kv_heads]
 * [head_dim] of the backend's dtype, 16-byte aligned).  row_start is DEVICE [n_seqs + 1], nondecreasing, n_rows =
 * row_start[n_seqs]; row_start[i + 1] - row_start[i] <= kv_len[i] is how many tokens are read.  The batch's q_start is
 * not read. */
wwws_status wwws_cache_read(wwws_backend* b, const wwws_batch* batch, const wwws_kv_pages* pages,
                            const int32_t* row_start, uint64_t n_rows, void* k_out, void* v_out);

/* Attention of the batch's new tokens (whose own keys and values have been appended): the row of a token at place p
 * sees key j <= p; with window > 0 only j > p - window or j < sinks.
 *   out = sum_j softmax_j(scale * q . k_j) v_j,   0 where nothing is seen.
 * q and out: [n_tokens][n_heads][head_dim] of the backend's dtype, 16-byte aligned, strides in elements (multiples of
 * 8).  Scores, softmax and sums are fp32; the softmax weights are rounded to 16 bits for the second product (f16 or bf16 as
 * the backend; f16 for few rows over a quantised cache, whatever the backend), weights in f16 with a factor that keeps them
 * out of its subnormals.  A hidden key never reaches a row's result, whatever its key and value hold (e4m3 codes that are
 * no numbers, which wwws_cache_append never writes, excepted); a visible one that is infinite or not a number does (a
 * value: in its own column).  Results do not depend on what else is in the batch's pages, and repeat bit for bit.
 * Where a sequence may have more than 32 new rows per kv head (48 over a quantised cache; a row is a new token and one of
 * its query heads), the call is launched 32 sequences at a time. */
wwws_status wwws_attend(wwws_backend* b, const wwws_batch* batch, const wwws_kv_pages* pages, const void* q,
                        uint64_t q_stride, void* out, uint64_t out_stride, float scale, uint32_t window, uint32_t sinks);

/* What is done to the logits of each row, all arrays DEVICE and caller-owned; a NULL array leaves its part out.  Per row
 * r, in fp32 and in this order, x being the logit of token v:
 *   v in the row's history          x = x > 0 ? x / repetition[r] : x * repetition[r]
 *   c times in its output           x = x - frequency[r] * c;  if c > 0: x = x - presence[r]
 *   v in its bias list              x = x + bias_value (the last entry of a repeated id holds; at most 2,047 entries a row)
 *   bit v of its mask is 0          x = -infinity
 * The history of row r, at most 2^20 - 1 tokens, is history[history_start[r] .. history_start[r + 1]): prompt_len[r]
 * prompt tokens (none if NULL; all of it if prompt_len[r] is more), then its output.  Masks are [n_masks][mask_stride]
 * words of 32 tokens, lowest bit first; mask_index[r] < 0: no mask for the row; mask_index NULL: row r has mask r. */
typedef struct {
    const int32_t* history; const int32_t* history_start; const int32_t* prompt_len; /* [..], [n_rows + 1], [n_rows] */
    const float* repetition; const float* presence; const float* frequency;           /* [n_rows] */
    const int32_t* bias_id; const float* bias_value; const int32_t* bias_start;       /* [..], [..], [n_rows + 1] */
    const uint32_t* mask; const int32_t* mask_index;                                   /* see above, [n_rows] */
    uint64_t n_history, n_bias;  /* entries of history and of the bias lists (offsets beyond them are errors) */
    uint32_t n_masks, mask_stride;
} wwws_shaping;

/* Shape n_rows rows of `vocab` logits (dtype WWWS_BF16, WWWS_F16 or WWWS_F32; strides in elements) into `out` (same
 * dtype; may be `logits` itself with the same stride), rounded once.  token (may be NULL): the lowest index of the
 * row's largest rounded value, -1 if none is above -infinity; a NaN is never chosen. */
wwws_status wwws_shape_logits(wwws_backend* b, const wwws_shaping* shaping, uint32_t n_rows, uint32_t vocab,
                              uint32_t dtype, const void* logits, uint64_t stride, void* out, uint64_t out_stride,
                              int32_t* token);

/* Wait for the stream and report what the kernels found wrong since the last call: WWWS_ERR_INDEX (a page, token or
 * mask id out of range), WWWS_ERR_ARG (offsets or lengths outside the batch's bounds), WWWS_ERR_TIMEOUT (a wait inside
 * wwws_attend ran out after about two seconds: its outputs are not to be trusted; the next call starts clean). */
wwws_status wwws_backend_sync(wwws_backend* b);

const char* wwws_backend_last_error(const wwws_backend* b);

#ifdef __cplusplus
}
#endif
#endif /* WWWS_BACKEND_H */
