/*
 * symb_block.h -- what a client runs between two shared projections, for the whole flattened batch: the norm before them (with its
 * backward pass), and attention over the clients' key/value caches.
 *
 * Every call works on the flattened token batch of symb.h: S segments, segment i owns rows off[i] .. off[i+1]-1.  Types, ownership,
 * ordering and errors are symb.h's: bf16 activations, DEVICE tensors owned by the caller, 16-byte aligned, HOST descriptors copied during the
 * call, everything enqueued on `stream`, all checks before the first launch.  A batch without rows is legal and enqueues nothing, except
 * that symb_norm_bwd writes the zeros of SYMB_GRAD_OVERWRITE.
 *
 * A call's descriptors fill one slot of 2 MiB (symb.h): 36 bytes a segment for symb_norm_fwd; 32 a segment, 24 a gradient and 16 a chunk of rows (768 more than segments at most) for symb_norm_bwd; 16 for
 * every page that a segment's new tokens go to (131072 of them); 32 for every work item of symb_kv_attention, of which a key head's rows (tokens times the query heads that share it) make at least one
 * in 128.  More is SYMB_ERR_UNSUPPORTED, from the workspace queries too: one prompt of 170000 tokens with 48 query heads on a key head is about the longest; a longer one is given in several calls.
 */
#ifndef SYMB_BLOCK_H
#define SYMB_BLOCK_H

#include "symb.h"

#ifdef __cplusplus
extern "C" {
#endif

/* ---- norms --------------------------------------------------------------------------------------------------------------------
 * For a row x of segment i, w = weight_base + weight_i (weight_i = NULL: w = 1, b = bias_i or 0):
 *   LAYER: mu = mean(x), r = 1 / sqrt(mean((x - mu)^2) + eps), z = (x - mu) r;   RMS: z = x r, r = 1 / sqrt(mean(x^2) + eps)
 *   forward:  y = z w + b
 *   backward: g = dy w;  dx = r (g - z mean(g z) - [LAYER] mean(g));   dweight_i = sum_t dy z,  dbias_i = sum_t dy  over its rows
 * Statistics and sums are fp32, y and dx are rounded once.  Nothing is kept from forward: backward takes x and forms the statistics again.
 */
typedef enum { SYMB_NORM_LAYER = 0, SYMB_NORM_RMS = 1 } symb_norm_kind;

typedef struct {
    const void* weight;            /* DEVICE bf16 [width] or NULL (ones, whatever weight_base is) */
    const void* bias;              /* DEVICE bf16 [width] or NULL */
    void* dweight;                 /* DEVICE fp32 [width] or NULL = no gradient wanted */
    void* dbias;                   /* DEVICE fp32 [width] or NULL = no gradient wanted */
} symb_norm;

typedef struct {
    int32_t width;                 /* a multiple of 8, at most SYMB_NORM_MAX_WIDTH */
    int32_t num_segments;
    const int32_t* seg_offsets;    /* HOST, as in symb_batch */
    const symb_norm* norms;        /* HOST, num_segments entries.  Segments may share weight and bias; segments that name the same dweight
                                      and the same dbias add up there (one of the two alone shared: SYMB_ERR_INVALID_ARG) */
    int32_t kind;                  /* symb_norm_kind */
    float eps;                     /* >= 0, finite; a row with eps + variance = 0 gives what the formulas do (NaN) */
    float weight_base;             /* added to every weight: 1 for models that store the weight less one, else 0 */
} symb_norm_batch;

enum { SYMB_NORM_MAX_WIDTH = 16384 };

/* Bytes of workspace symb_norm_bwd needs (partial sums of the weight gradients; may be 0).  Host-only. */
symb_status symb_norm_workspace_bytes(const symb_norm_batch* b, size_t* out);

/* X, Y [T][width] bf16, dense rows.  Y may be X. */
symb_status symb_norm_fwd(symb_handle h, const symb_norm_batch* b, const void* X, void* Y, void* stream);

/* X, dY, dX [T][width] bf16, dense rows.  dX may be dY or X.  flags: SYMB_GRAD_OVERWRITE or SYMB_GRAD_ACCUMULATE for dweight and dbias; an
 * empty segment writes zeros or leaves them.  Deterministic: sums are formed in a fixed order (in chunks of rows that the batch as a whole decides on; dX hangs on its own row alone). */
symb_status symb_norm_bwd(symb_handle h, const symb_norm_batch* b, const void* X, const void* dY, void* dX, uint32_t flags, void* ws,
                          size_t ws_bytes, void* stream);

/* ---- the key/value cache ------------------------------------------------------------------------------------------------------
 * A pool of pages of `page_tokens` tokens.  Keys and values are held in 8 bits, E4M3 (four significant bits, largest 448, no infinity, 0x7f/0xff NaN),
 * with one scale for each page and head, a power of two held as E8M0 (2^(byte - 127)):
 *     k       [num_pages][kv_heads][page_tokens][head_dim]
 *     v       [num_pages][kv_heads][head_dim][page_tokens]      (a value channel's tokens side by side, as the products over tokens read them)
 *     k_scale, v_scale [num_pages][kv_heads]
 * Because the scale is a power of two, a page whose scale grows is held again without a second rounding, except of values that
 * become subnormal (below 2^-6 of the new scale).
 */
typedef struct {
    void* k;                       /* DEVICE */
    void* v;                       /* DEVICE */
    void* k_scale;                 /* DEVICE */
    void* v_scale;                 /* DEVICE */
    int32_t num_pages;
    int32_t kv_heads;
    int32_t head_dim;              /* 64 or 128 (others: SYMB_ERR_UNSUPPORTED) */
    int32_t page_tokens;           /* 32, 64 or 128 (others: SYMB_ERR_UNSUPPORTED) */
} symb_kv_cache;

/* The flattened batch as the cache calls see it: segment i's rows are the tokens past[i] .. past[i] + n_i - 1 of its sequence, in
 * order.  Token s of segment i lies in page page_table[i][s / page_tokens], slot s % page_tokens. */
typedef struct {
    int32_t num_segments;
    const int32_t* seg_offsets;    /* HOST, as in symb_batch */
    const int32_t* past;           /* HOST, num_segments entries: tokens in the cache before this call's (>= 0) */
    const int32_t* page_table;     /* DEVICE int32 [num_segments][table_stride].  Entries of pages that a call does not touch are not read.
                                      A page number outside 0 .. num_pages-1 is never followed: its tokens are not stored, and the rows
                                      that see them, and no others, come out NaN */
    int32_t table_stride;          /* entries per segment: (past[i] + n_i) / page_tokens rounded up at least, for every segment with rows */
} symb_kv_batch;

/* Turning by position: pairs (a, b) of a head's first `dim` elements become (a cos - b sin, b cos + a sin) with the cosines
 * table[s][0 .. dim/2-1] and sines table[s][dim/2 .. dim-1] of the token's position s; the elements behind stay. */
typedef enum { SYMB_ROTATE_HALVES = 0,      /* pair j is elements j and j + dim/2 */
               SYMB_ROTATE_ADJACENT = 1     /* pair j is elements 2j and 2j + 1 */
             } symb_rotation_pairs;
typedef struct {
    const void* table;             /* DEVICE fp32 [positions][dim] */
    int32_t positions;             /* more than the last token's position */
    int32_t dim;                   /* a multiple of 16, at most head_dim */
    int32_t pairs;                 /* symb_rotation_pairs */
} symb_rotation;

/* Appends the batch's keys and values to the cache, keys turned, and turns its queries.
 *   k, v [T][kv_heads][head_dim] bf16, rows `k_stride` / `v_stride` elements apart (multiples of 8: columns of one product may be passed as they lie);
 *   q [T][q_heads][head_dim] -> q_out, likewise with strides (q_out may be q); q NULL with q_heads 0: keys and values only.
 *   rotation NULL: nothing is turned.
 * For each touched page and head: the smallest power of two that brings the largest finite new value to 448 at most, and no smaller than the
 * page's scale if it holds earlier tokens of the segment (slots before the first new one; these are held again where the scale
 * grows).  Values are turned in fp32 and rounded once, to nearest even; infinities and NaN become NaN and leave the scale alone.  Slots behind the last
 * new token keep their bytes.  A page that is given zeros alone gets the smallest scale, 2^-126.  Segments of one call must not share a page that one of them writes. */
symb_status symb_kv_append(symb_handle h, const symb_kv_batch* b, const symb_kv_cache* cache, const symb_rotation* rotation, const void* q,
                           int64_t q_stride, int32_t q_heads, void* q_out, int64_t q_out_stride, const void* k, int64_t k_stride, const void* v,
                           int64_t v_stride, void* stream);

/* Bytes of workspace symb_kv_attention needs for this batch (may be 0).  Host-only; cache's pointers are not looked at. */
symb_status symb_kv_workspace_bytes(const symb_kv_batch* b, const symb_kv_cache* cache, int32_t q_heads, int32_t window, size_t* out);

/* Causal attention of the batch's rows over their own segment's tokens in the cache, the batch's own among them (symb_kv_append comes first):
 *     x_s = scale q . k_s  (cap > 0: cap tanh(x_s / cap)),   out = sum_s exp(x_s - max) v_s / sum_s exp(x_s - max)
 * over the tokens s of the row's segment with  position - window < s <= position  (window 0: all up to its position).  Query head j reads
 * key head j / (q_heads / kv_heads); q_heads is a multiple of kv_heads.
 *   q, out [T][q_heads][head_dim] bf16 with row strides in elements (multiples of 8); out must not overlap q.
 *   scale > 0; cap >= 0, of any size (capping is good to 2^-19 of a score); window >= 0.
 * What lies in hidden tokens, NaN and scales of any byte included, never reaches a row.  A value of 2^128 or more (a scale byte of 247 at least) is infinite or NaN to the rows that see it, all
 * of a page whose scale byte is 0xff NaN.
 * What is rounded: a row's query enters the scores as two E4M3 terms, exact for elements from 2^-13 of its largest on, off by 2^-21 of the largest (taken as 2^-93 at least) at most below; of a score's products those some
 * 2^-15 below the largest are dropped; the weights exp(x - max) enter the second product as bf16, 2^-9 of each at most (their sum takes them as they were).  Scores, maxima, sums and outputs are
 * otherwise fp32, outputs rounded once.
 * The same batch gives the same bits.  The same segment in another batch may not: its rows' kernel and the split of its tokens are chosen for the batch as a whole.
 * Under capture, `past` and the work lists made of it become part of the graph: a replay attends from the same positions (and symb_kv_append appends at them). */
symb_status symb_kv_attention(symb_handle h, const symb_kv_batch* b, const symb_kv_cache* cache, const void* q, int64_t q_stride, int32_t q_heads,
                              void* out, int64_t out_stride, float scale, int32_t window, float cap, void* ws, size_t ws_bytes, void* stream);

#ifdef __cplusplus
}
#endif
#endif /* SYMB_BLOCK_H */
