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
 * and, where a request is answered with several drafted tokens or several hypotheses at a time:
 *   wwws_rotate / wwws_rotate_append      norms of queries and keys for each head and their rotation by position, in one
 *                                         pass, which may write keys and values to the cache as well
 *   wwws_attend_tree                      attention of a tree of drafted tokens over the paged cache
 *   wwws_cache_compact                    the accepted tokens of a tree moved together
 *   wwws_select_beams                     the best continuations over a request's beams and the vocabulary
 *   wwws_pages_fork / wwws_cache_copy     sequences continued, dropped, cut back and given room: their pages counted,
 *                                         shared, taken and given back, and the pages copied that two would write
 *
 * Conventions are those of wwws.h: every call returns a wwws_status and never aborts; all device work is enqueued on
 * the stream given at creation and is asynchronous (wwws_backend_sync and wwws_destroy_backend synchronise it); the
 * library allocates no device memory (one workspace from the caller); "HOST" / "DEVICE" say where a pointer points;
 * a handle is not thread-safe and lives on the GPU that holds its workspace.  Arrays handed to a call must stay valid
 * until the stream has passed it, and must have been written by work that the stream waits for.  Calls captured into graphs use the
 * handle's workspace when they are replayed: no two of them, nor one beside a call, at the same time.
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
 * Over a quantised cache weights in f16 are kept relative to the value scales of a sequence's kv head, so what each key adds to a row,
 * relative to its largest weight, may be off by 2^-35 of the largest value that any new token of the sequence sees there: a value 2^20 times the
 * others takes precision from the rows that do not see it as well.  (bf16 backends: wwws_attend_tree, and few rows.)
 * Where a sequence may have more than 32 new rows per kv head (48 over a quantised cache; a row is a new token and one of
 * its query heads), a kernel for many rows takes all of the call's sequences, 32 a launch: single tokens are answered sooner in a call of their own
 * than beside prompts. */
wwws_status wwws_attend(wwws_backend* b, const wwws_batch* batch, const wwws_kv_pages* pages, const void* q,
                        uint64_t q_stride, void* out, uint64_t out_stride, float scale, uint32_t window, uint32_t sinks);

/* The same for new tokens that are a tree of drafts behind the context, the kv_len[i] - q_len tokens before them: parents
 * come before their children, and a new token sees the context and, of the new tokens j up to itself, those whose bit is set in
 * its row of `tree` (DEVICE [n_tokens][tree_words], 32 places a word, lowest bit first; tree_words * 32 >= max_q_len):
 * its ancestors and itself, as a rule.  It stands d places behind the context, d being one less than the new tokens that it sees
 * (0 if it sees none); the window is counted from there and hides context alone: what `tree` shows stays visible however far above, so
 * that a chain deeper than the window sees more than wwws_attend shows its tokens.  Where the longest sequence has more than 32 rows
 * per kv head (48 over a quantised cache) the call is launched up to 256 sequences at a time. */
wwws_status wwws_attend_tree(wwws_backend* b, const wwws_batch* batch, const wwws_kv_pages* pages, const void* q,
                             uint64_t q_stride, void* out, uint64_t out_stride, float scale, uint32_t window,
                             uint32_t sinks, const uint32_t* tree, uint32_t tree_words);

/* How queries and keys are turned.  Of the first `dim` elements of a head (a multiple of 16, 16 .. head_dim), pair i < dim / 2
 * is (i, dim / 2 + i), or (2 i, 2 i + 1) where interleaved is 1; the elements behind them stay where they are.  At position p
 * pair (a, b) becomes (a cos t - b sin t, b cos t + a sin t), t = 2 pi p turns[i] / 2^64; the product wraps around exactly, so
 * that no position is too far.  A weight makes x into x * weight / sqrt(mean(x^2) + eps) over the whole head before that.
 * In fp32, rounded once; cosines and sines are within 2^-21 of theirs. */
typedef struct {
    const uint64_t* turns;  /* DEVICE [dim / 2] turns of pair i per position, times 2^64: f / (2 pi) * 2^64 of f radians */
    const uint8_t* axis;    /* DEVICE [dim / 2] by which of a token's positions pair i turns, < n_axes; NULL: the first */
    const float* q_weight;  /* DEVICE [head_dim], 16-byte aligned; NULL: queries are not normed */
    const float* k_weight;  /* the same for keys */
    float eps;              /* >= 0 */
    uint32_t dim, n_axes, interleaved; /* n_axes 1 .. 8 */
} wwws_rotation;

/* Norm and turn queries and keys of n_tokens tokens (< 2^31): q and q_out [n_tokens][n_heads][head_dim], k and k_out
 * [n_tokens][n_kv_heads][head_dim] of the backend's dtype, 16-byte aligned, strides in elements (multiples of 8); an output
 * may be its input with the same stride, and overlaps nothing otherwise.  positions: DEVICE [n_tokens][n_axes]. */
wwws_status wwws_rotate(wwws_backend* b, const wwws_rotation* rotation, uint32_t n_tokens, const int32_t* positions,
                        const void* q, uint64_t q_stride, const void* k, uint64_t k_stride, void* q_out,
                        uint64_t q_out_stride, void* k_out, uint64_t k_out_stride);

/* The same for a batch's new tokens, turned keys and the values v written to their pages as wwws_cache_append does (a quantised
 * cache takes its codes from the turned keys in fp32).  positions NULL: each token's place in its sequence, on every axis. */
wwws_status wwws_rotate_append(wwws_backend* b, const wwws_batch* batch, const wwws_kv_pages* pages,
                               const wwws_rotation* rotation, const int32_t* positions, const void* q, uint64_t q_stride,
                               const void* k, uint64_t k_stride, const void* v, uint64_t v_stride, void* q_out,
                               uint64_t q_out_stride);

/* Sequences continued.  All arrays DEVICE; tables are [sequences][max_pages of the configuration].  refs counts how often each
 * page of the pool is held: by the sequences of `table`, a page in held[j] (<= max_pages) first entries of row j, and by whatever
 * else the caller counts; a page of 0 is free.  New sequence i takes the first keep[i] tokens of old sequence source[i] (keep[i] <=
 * held[source[i]] * page_tokens; source[i] < 0: it starts empty, keep[i] is not read) and gets pages for room[i] tokens, or
 * keep[i] if that is more.  Old sequences end: what no new one continues is let go.
 *   - Pages wholly within keep[i] tokens are shared.
 *   - The page that keep[i] ends inside will be written further: it stays with the first new sequence that ends inside it if nobody
 *     holds it otherwise; every other one gets a page of its own and a row of `moves`: from, to, tokens (else -1, -1, 0).
 *   - Fresh pages are the free ones of lowest number, in the order of (sequence, place).  Where the pool runs out a place gets
 *     -1, a page outside the pool, and the next wwws_backend_sync says WWWS_ERR_ALLOC.  Such places may be let go, not continued.
 * A bad new sequence is reported and left empty; entries behind a row's pages are 0.  refs_out may be refs; nothing else may overlap. */
typedef struct {
    const int32_t* refs; int32_t* refs_out;                                          /* [n_pages] */
    const int32_t* table; const int32_t* held;                                       /* [n_old][max_pages], [n_old] */
    const int32_t* source; const int32_t* keep; const int32_t* room;                 /* [n_new] */
    int32_t* table_out; int32_t* held_out; int32_t* moves;                           /* [n_new][max_pages], [n_new], [n_new][3] */
    uint32_t n_old, n_new;                                                           /* <= max_seqs */
} wwws_fork;
wwws_status wwws_pages_fork(wwws_backend* b, const wwws_fork* fork);

/* Copy the first moves[i][2] tokens of page moves[i][0] to page moves[i][1] in each of n_layers pools (HOST array of records); a
 * negative target is no copy.  No page is the target of two moves, nor the target of one and the source of another. */
wwws_status wwws_cache_copy(wwws_backend* b, const wwws_kv_pages* layers, uint32_t n_layers, const int32_t* moves,
                            uint32_t n_moves);

/* Move new token path[i][m] of sequence i to place m of its new tokens, for m < path_len[i], in each of n_layers pools: path
 * ([n_seqs][path_stride] DEVICE, path_stride <= 2048) ascends, so that a place is written after it is read.  The sequence's last page of
 * new tokens is its own.  A bad path moves nothing and is reported. */
wwws_status wwws_cache_compact(wwws_backend* b, const wwws_batch* batch, const wwws_kv_pages* layers, uint32_t n_layers,
                               const int32_t* path, const int32_t* path_len, uint32_t path_stride);

/* The best `keep` (1 .. 128) continuations of each request: row r of logits (dtype as for wwws_shape_logits, stride in elements) is
 * beam r % beams of request r / beams, beams 1 .. 256; n_rows is a multiple of beams and <= max_rows; vocab <= 2^24.
 *   score(r, v) = total[r] + logits[r][v] - log sum_w exp(logits[r][w])
 * with the sum's terms in fp32 and the rest in 64 bits; largest first, ties to the lowest (row, token).
 * score [requests][keep] is rounded to fp32, parent (the row) and token are int32; where a request has fewer continuations above
 * -infinity: -infinity, -1, -1.  A row whose total is -infinity, infinite or NaN, or that holds a NaN or +infinity, has none.
 * scratch: DEVICE, 16-byte aligned, of wwws_beams_scratch_bytes, free again when the stream has passed the call. */
wwws_status wwws_beams_scratch_bytes(uint32_t n_rows, uint32_t vocab, uint32_t dtype, uint32_t keep, uint64_t* bytes_out);
wwws_status wwws_select_beams(wwws_backend* b, uint32_t n_rows, uint32_t beams, uint32_t vocab, uint32_t dtype,
                              const void* logits, uint64_t stride, const float* total, uint32_t keep, void* scratch,
                              uint64_t scratch_bytes, float* score, int32_t* parent, int32_t* token);

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
 * wwws_attend or wwws_attend_tree ran out after about two seconds: its outputs are not to be trusted; the next call starts clean),
 * WWWS_ERR_ALLOC (the page pool ran out in wwws_pages_fork). */
wwws_status wwws_backend_sync(wwws_backend* b);

const char* wwws_backend_last_error(const wwws_backend* b);

#ifdef __cplusplus
}
#endif
#endif /* WWWS_BACKEND_H */
