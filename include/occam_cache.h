/*
 * occam_cache.h -- the serving side of the register-anchored evidence test: rotary
 * positions, a paged 8-bit key/value cache, attention over it, and the page operations
 * that drop what the test pruned.
 *
 * The paper's pipeline keeps the K/V rows of the surviving tokens (Algorithm 1, the pruned
 * sequence [S2; T]; Appendix Eq. kv_memory_appendix).  How many survive is known on the
 * device only (occam_prune writes kept_count there), and differs from question to question
 * on the same image.  The calls here therefore keep the whole state of the cache -- page
 * tables, lengths, free pages -- in device memory and never synchronise with the host:
 *
 *   occam_rotate          rotary positions with several axes on query and key rows
 *   occam_pages_reset     empty every sequence
 *   occam_pages_reserve   make room for new tokens (once per step, for every layer)
 *   occam_cache_append    quantise a layer's new K/V rows into the reserved room
 *   occam_cache_attend    a layer's attention of the sequences' last rows; its
 *                         normalisers are the row_lse of occam_score / occam_prune
 *   occam_cache_read      a layer's K/V rows as values (the keys Stage II scores)
 *   occam_pages_fork      another sequence over the same pages (another question)
 *   occam_pages_keep      drop the tokens that occam_select did not list
 *   occam_cache_move      move a layer's survivors into the pages occam_pages_keep chose
 *   occam_pages_free      give a sequence up
 *
 * Conventions are those of occam.h: device pointers owned by the caller, host structs read
 * during the call only, host validation before anything is enqueued, no allocation, no
 * synchronisation, no memset nodes, one stream per call.  Calls that share an occam_pages
 * must be ordered (one stream, or events); calls that only read it (occam_cache_append of
 * different layers, occam_cache_attend, occam_cache_read, occam_cache_move of different
 * layers) may overlap each other.  Inputs must be finite.
 *
 * What the host cannot check is checked on the device: a slot outside the cache or listed
 * twice, a sequence that would outgrow its table, a pool without enough free pages, row
 * offsets that descend or pass the stated bound.  The call then changes nothing at all, its
 * plan is empty (the calls that read the plan do nothing), and a bit of *status is set, which
 * stays until the caller clears it.  occam_cache_read and occam_cache_attend set the bits for
 * slots and row offsets too, and serve the other sequences of the batch: rows of a slot that
 * there is not are left alone by the one and get zeros and -infinity from the other, rows of a
 * sequence whose offsets are wrong are left alone by both.
 *
 * 8-bit values.  A page holds page_tokens tokens of one sequence.  For every page and key
 * head, keys and values have one scale each: the smallest power of two that brings the
 * largest magnitude written to at most 448 (the largest e4m3 number), its exponent within
 * [-100, 120].  A value is an e4m3 number (OCP: 4 exponent bits, 3 of mantissa, no
 * infinities) times that scale, rounded to nearest, ties to even (within float32's range: the
 * largest exponent goes with numbers up to 240).  Tokens appended to a page
 * that holds some already may raise its scale; the values there are then rounded once more,
 * which changes only what falls below the smallest normal number, 2^-6 times the new scale.
 * Power-of-two scales make every value exact in bfloat16 (8 bits of mantissa hold 4).
 */
#ifndef OCCAM_CACHE_H
#define OCCAM_CACHE_H

#include "occam.h"

#ifdef __cplusplus
extern "C" {
#endif

#define OCCAM_MAX_PAIRS 128
#define OCCAM_MAX_SLOTS 65536   /* sequences of one occam_pages                        */
#define OCCAM_MAX_BATCH 8192    /* sequences of one call                               */

/* Bits of occam_pages.status. */
typedef enum {
    OCCAM_PAGES_FULL = 1,     /* not enough free pages                                 */
    OCCAM_PAGES_BAD_SEQ = 2,  /* a slot out of range, listed twice, or (fork) not empty */
    OCCAM_PAGES_TOO_LONG = 4, /* a sequence would need more than max_pages pages       */
    OCCAM_PAGES_BAD_SPAN = 8, /* keep: a span outside its sequence, or more survivors  */
    OCCAM_PAGES_BAD_ROWS = 16 /* row_offsets that descend, or pass max_rows            */
} occam_pages_status;

/* The pages of a cache, shared by all its layers.  Device arrays of the caller,
 * initialised by occam_pages_reset; between calls they may be read (length, table), but
 * only the calls below change them.  Free pages are taken lowest number first. */
typedef struct {
    int32_t num_pages;    /* pages of every layer's storage, 1 .. 2^24                  */
    int32_t page_tokens;  /* 16, 32, 64, 128 or 256                                     */
    int32_t num_seqs;     /* slots for sequences, 1 .. OCCAM_MAX_SLOTS                  */
    int32_t max_pages;    /* pages one sequence can have, >= 1                          */
    int32_t *table;       /* [num_seqs][max_pages] page numbers                         */
    int32_t *length;      /* [num_seqs] tokens held                                     */
    int32_t *refs;        /* [num_pages] sequences that hold the page                   */
    uint32_t *taken;      /* [(num_pages + 31) / 32] bit p % 32 of word p / 32          */
    int32_t *status;      /* [1] occam_pages_status bits, sticky                        */
} occam_pages;

/* One layer's storage.  A row of d elements takes dp = 64, 128 or 256 bytes (the next that
 * holds d).  The order of a page's bytes is the library's: per key head, keys by token
 * ([page_tokens][dp]), values by groups of four tokens ([page_tokens / 4][dp][4]). */
typedef struct {
    int32_t num_kv_heads; /* Hkv >= 1                                                   */
    int32_t head_dim;     /* d: a multiple of 8, 8 .. 256                               */
    uint8_t *k, *v;       /* [num_pages][Hkv][page_tokens * dp], 16-byte aligned        */
    float *k_scale, *v_scale; /* [num_pages][Hkv]                                       */
} occam_cache;

/* The sequences of a call and their packed rows: sequence i is slot seq[i] (slot i when seq
 * is NULL) and owns rows ro_i .. ro_{i+1}, ro_i = row_offsets[i] (or i * rows).  Slots of a
 * call are distinct.  A sequence may own no rows when row_offsets is given. */
typedef struct {
    int32_t n;                  /* 1 .. OCCAM_MAX_BATCH                                 */
    const int32_t *seq;         /* device [n], or NULL                                  */
    int32_t rows;               /* rows per sequence when row_offsets == NULL, >= 1     */
    const int32_t *row_offsets; /* device [n+1], non-decreasing, or NULL                */
    int32_t max_rows;           /* upper bound of a sequence's rows with row_offsets,
                                   >= 1 (also where no sequence owns a row)             */
} occam_batch;

/* --------------------------------------------------------------- rotary positions */
typedef enum { OCCAM_PAIRS_HALVES = 0, OCCAM_PAIRS_ADJACENT = 1 } occam_pairs;

/* Filled by occam_rotary_init; plain data, no device memory. */
typedef struct {
    int32_t head_dim, pairs, axes, layout;
    uint64_t turn[OCCAM_MAX_PAIRS]; /* a position's fraction of a turn, in 2^-64        */
    uint8_t axis[OCCAM_MAX_PAIRS];
} occam_rotary;

/* One tensor of rows to rotate: [rows][heads][head_dim], heads packed, rows stride apart
 * (in elements, >= heads * head_dim).  dst may be src (in place); otherwise they must not
 * overlap, and no tensor's dst may overlap another one's src or dst (rows that interleave, as
 * slices of one projection do, must be equally far apart). */
typedef struct {
    const void *src;
    void *dst;
    int32_t heads;
    int64_t src_row_stride, dst_row_stride;
} occam_heads;

/* Pair p of a head is (e_p, e_{p + pairs}) with HALVES, (e_2p, e_{2p+1}) with ADJACENT;
 * elements from 2 * pairs on are copied.  It turns with axis axis[p] (NULL: axis 0) by
 * inv_freq[p] radians per position.  head_dim in [2, 256], 1 <= pairs <= head_dim / 2,
 * axes in [1, 4], axis[p] < axes, inv_freq finite. */
occam_status occam_rotary_init(occam_rotary *rotary, int32_t head_dim, int32_t pairs,
                               int32_t axes, int32_t layout, const double *inv_freq,
                               const uint8_t *axis);

/* (x, y) -> (x cos a - y sin a, x sin a + y cos a), a = positions[row][axis[p]] *
 * inv_freq[p], for every head of the n <= OCCAM_MAX_ROW_TENSORS tensors; inverse != 0 turns
 * by -a (the transpose: the gradient of the forward call).  positions: device int32
 * [rows][axes], any value (the angle is reduced to one turn exactly, in 64-bit integers).
 * dtype: occam_dtype of all tensors; the arithmetic is float32, rounded once. */
occam_status occam_rotate(const occam_rotary *rotary, int32_t rows, const int32_t *positions,
                          int32_t inverse, int32_t dtype, int32_t n, const occam_heads *tensors,
                          hipStream_t stream);

/* --------------------------------------------------------------- pages */
/* Bytes of the plan that occam_pages_reserve, _fork and _keep write and the calls after
 * them read, for calls of up to n sequences (0 for invalid arguments). */
size_t occam_pages_plan_size(const occam_pages *pages, int32_t n);

/* Bytes of each of occam_cache.k and .v (0 for invalid arguments). */
size_t occam_cache_storage_size(const occam_pages *pages, int32_t num_kv_heads,
                                int32_t head_dim);

/* Every sequence empty, every page free, status 0. */
occam_status occam_pages_reset(const occam_pages *pages, hipStream_t stream);

/* Room for the batch's rows behind what its sequences hold: takes pages, raises the
 * lengths, and writes the plan that every layer's occam_cache_append of the step reads.  A
 * partly filled last page that other sequences share is replaced by a page of its own,
 * which the append fills with its tokens.  All rows of the batch or none.  Every layer's
 * append has to be enqueued before any later call that takes pages (the shared page may
 * have become free). */
occam_status occam_pages_reserve(const occam_pages *pages, const occam_batch *batch,
                                 void *plan, size_t plan_bytes, hipStream_t stream);

/* Sequence dst[i] (empty, distinct) becomes a copy of src[i] over the same pages. */
occam_status occam_pages_fork(const occam_pages *pages, int32_t n, const int32_t *src,
                              const int32_t *dst, void *plan, size_t plan_bytes,
                              hipStream_t stream);

/* Empties n sequences; pages that no other sequence holds become free.  A slot listed
 * twice is freed once, a slot out of range is skipped. */
occam_status occam_pages_free(const occam_pages *pages, int32_t n, const int32_t *seq,
                              hipStream_t stream);

/* Drops tokens: of the span_len[i] tokens of seq[i] from token span_start[i] on, those
 * stay whose index within the span is listed in kept_idx[kept_offsets[i] ..
 * kept_offsets[i + 1]), ascending -- the lists of occam_select / occam_prune (what a list
 * that is not ascending leaves is undefined, but comes from the same sequence).  Tokens
 * outside the span stay.  kept_idx is not NULL, also where every list is empty.  The pages from the first dropped token's on are replaced by fresh
 * ones, so pages shared with other sequences are not touched; the fresh pages must be free
 * while the old ones are still held.  Every layer's occam_cache_move has to be enqueued
 * with the same plan, kept_idx and kept_offsets before any later call that takes pages. */
occam_status occam_pages_keep(const occam_pages *pages, int32_t n, const int32_t *seq,
                              const int32_t *span_start, const int32_t *span_len,
                              const int32_t *kept_idx, const int32_t *kept_offsets, void *plan,
                              size_t plan_bytes, hipStream_t stream);

/* --------------------------------------------------------------- a layer's rows */
/* The batch's new rows, k and v [rows][Hkv][d] of dtype (F32 or BF16), rows k_row_stride /
 * v_row_stride elements apart (multiples of 16 bytes, 16-byte aligned), into the room that
 * occam_pages_reserve made with the same batch and plan. */
occam_status occam_cache_append(const occam_pages *pages, const occam_cache *cache,
                                const occam_batch *batch, const void *plan, size_t plan_bytes,
                                int32_t dtype, const void *k, int64_t k_row_stride,
                                const void *v, int64_t v_row_stride, hipStream_t stream);

/* Tokens start[i] .. of every sequence (start NULL: from token 0), as many as the batch
 * gives it rows, as values of dtype (exact in both): k and v (either may be NULL) in the
 * layout of occam_cache_append.  Rows of tokens that the sequence does not hold are left as
 * they were. */
occam_status occam_cache_read(const occam_pages *pages, const occam_cache *cache,
                              const occam_batch *batch, const int32_t *start, int32_t dtype,
                              void *k, int64_t k_row_stride, void *v, int64_t v_row_stride,
                              hipStream_t stream);

/* The survivors of occam_pages_keep (n, plan, kept_idx, kept_offsets as there) into their
 * fresh pages, whose scales follow from the values they hold. */
occam_status occam_cache_move(const occam_pages *pages, const occam_cache *cache, int32_t n,
                              const void *plan, size_t plan_bytes, const int32_t *kept_idx,
                              const int32_t *kept_offsets, hipStream_t stream);

/* --------------------------------------------------------------- attention */
typedef struct {
    int32_t num_heads;    /* H, a multiple of Hkv; head h reads key head h / (H / Hkv)   */
    int32_t causal;       /* 1: row t of T sees keys 0 .. len - T + t; 0: all len keys   */
    float softmax_scale;  /* 0 => 1/sqrt(d)                                              */
    int32_t max_tokens;   /* upper bound of the sequences' lengths (0: max_pages * page_tokens);
                             the nearer, the better the form that the call takes         */
} occam_attention;

/* Bytes of device workspace that occam_cache_attend with the same arguments may use (0 for
 * invalid ones).  It needs no initialisation and holds nothing between calls; calls that may
 * overlap (streams, graphs) need a workspace each. */
size_t occam_cache_workspace_size(const occam_pages *pages, const occam_cache *cache,
                                  const occam_batch *batch, const occam_attention *attention);

/* out[row, h] = sum_j softmax_j(scale <q[row, h], k_j>) v_j over the keys j the row sees,
 * where the batch's rows of sequence i are its last T_i tokens (already appended).  q and
 * out: bfloat16 [rows][H][d], rows q_row_stride / out_row_stride elements apart (multiples
 * of 8, 16-byte aligned).  row_lse (nullable): float32 [rows][H], the natural-log softmax
 * normaliser over those keys, in the layout of occam_score's row_lse.  A row that sees no
 * key gets zeros and -infinity.  Probabilities are rounded to float16 (2^-11 of them), sums are
 * float32; a key whose weight (its probability times its block's scale) is far below the row's
 * largest one adds its share to within 2^-26 of that weight.  q and out must not overlap.
 * max_tokens sizes the launch and the workspace and chooses between forms for few and for many
 * codes (without a near bound, short sequences in long tables can take a quarter longer); a
 * longer sequence is still attended to in full. */
occam_status occam_cache_attend(const occam_pages *pages, const occam_cache *cache,
                                const occam_batch *batch, const occam_attention *attention,
                                const void *q, int64_t q_row_stride, void *out,
                                int64_t out_row_stride, float *row_lse, void *workspace,
                                size_t ws_bytes, hipStream_t stream);

#ifdef __cplusplus
}
#endif

#endif /* OCCAM_CACHE_H */
