/*
 * libpreserve_mi355x -- operators around the decode step: what a program that serves with preserve.h has to run before a
 * step (rotary positions, places in the cache, a prompt's keys and values into it) and after it (log probabilities).
 *
 * Same conventions as preserve.h: every call returns a psv_status, nothing throws, aborts or prints, "dev" pointers are HIP
 * device pointers, the caller owns every buffer and stream.  Further:
 *  - The argument structs are host memory, read before the call returns.  No call here needs a context (psv_set_rope apart),
 *    allocates, synchronises, or keeps anything; every one can be captured into a HIP graph.
 *  - Calls are asynchronous on `stream` (hipStream_t), which belongs to the current device, as every pointer does.  Calls
 *    on different streams are independent as long as what one writes is not read or written by another.
 *  - Outputs must not overlap inputs or other outputs unless said otherwise.
 *  - What is checked on the host (null pointers, sizes, alignment, strides) is refused with PSV_ERR_INVALID_ARG or
 *    PSV_ERR_UNSUPPORTED before anything is launched.  What lies on the device is never trusted with an address: a slot or block
 *    id out of range is skipped as each call says.
 *  - 0 rows are valid everywhere and launch nothing.
 */
#ifndef PRESERVE_OPS_H
#define PRESERVE_OPS_H

#include "preserve.h"

#ifdef __cplusplus
extern "C" {
#endif

/* element types of rows */
enum { PSV_F32 = 0u, PSV_BF16 = 1u, PSV_F16 = 2u };

/* ---- rotary positions ------------------------------------------------------------------------ */

/* Which channels of a head are rotated, in which pairs, at which frequencies.  Channel pair i of `dims` / 2 at position p is
 * turned by the angle p * f_i and scaled by `magnitude`; channels from `dims` on pass through unchanged.
 * Frequencies: f_i = theta^(-2i / dims), scaled for contexts longer than the model was trained on by one of
 *   PSV_ROPE_PLAIN      f_i
 *   PSV_ROPE_LINEAR     f_i / factor: every position is divided by the factor
 *   PSV_ROPE_BY_TURNS   w f_i + (1 - w) f_i / factor, w = (n_i - low_turns) / (high_turns - low_turns) clamped to [0, 1], where
 *                       n_i = trained_context * f_i / 2 pi is how often pair i turns within the trained context
 *   PSV_ROPE_BY_CHANNEL the same with w linear in i instead of n_i: w = 1 up to the pair that makes high_turns (rounded down),
 *                       0 from the pair that makes low_turns (rounded up), both kept within [0, dims - 1]. */
enum { PSV_ROPE_HALF = 0u /* (i, i + dims/2) */, PSV_ROPE_INTERLEAVED = 1u /* (2i, 2i + 1) */ };
enum { PSV_ROPE_PLAIN = 0u, PSV_ROPE_LINEAR = 1u, PSV_ROPE_BY_TURNS = 2u, PSV_ROPE_BY_CHANNEL = 3u };
#define PSV_ROPE_MAX_DIMS 256u

typedef struct {
    uint32_t dims;            /* even, 2 .. PSV_ROPE_MAX_DIMS */
    uint32_t pairing;
    uint32_t scaling;
    uint32_t reserved;
    double   magnitude;       /* of the rotated channels; 0 means 1 */
    double   theta;           /* > 1 */
    double   factor;          /* >= 1; read by the three scaled forms */
    double   low_turns, high_turns;   /* 0 < low < high; read by the last two forms */
    double   trained_context; /* tokens, >= 1; read by the last two forms */
} psv_rope_desc;

/* The frequencies of a description, made once and handed to the calls below: plain data, to be copied freely. */
typedef struct {
    uint32_t dims, pairing;
    double   magnitude;
    double   freq[PSV_ROPE_MAX_DIMS / 2];   /* radians per position; 0 from dims / 2 on */
} psv_rope;

/* Pure host function. */
psv_status psv_rope_plan(const psv_rope_desc *desc, psv_rope *out);

/* The decode steps of this context (psv_decode_step) that run after this on stream_main rotate with these frequencies and this magnitude
 * instead of the descriptor's rope_theta (rope = NULL: with the descriptor's again).  psv_decode_step_static has no context and goes by its
 * descriptor.  A step rotates whole heads in halves: dims = 128 and PSV_ROPE_HALF, else PSV_ERR_UNSUPPORTED (a model of other pairs is served by
 * permuting the rows of its query and key projections: the product of a query and a key does not depend on the order of the channels; unrotated
 * channels are pairs of frequency 0, which a magnitude other than 1 would scale as well).  Both travel as a kernel argument on stream_main into
 * the context's workspace, where a step reads them: ordered with the steps, nothing is awaited.  A captured call takes effect when its graph
 * runs, and a step that a graph holds rotates with what was set last when it runs. */
psv_status psv_set_rope(psv_ctx *ctx, const psv_rope *rope);

/* Rotates rows: y = x with the first rope->dims channels of every head rotated to the row's position, computed in 32 bits (angles
 * in 64) and rounded once.  transpose = 1 turns by the negative angle, with the same magnitude: the gradient with respect
 * to x, and for magnitude 1 the inverse. */
typedef struct {
    const void *x;                /* dev */
    void *y;                      /* dev; y == x with equal strides rotates in place */
    const int32_t *positions;     /* dev [rows], any value */
    uint32_t rows;                /* <= 2^24 */
    uint32_t heads;               /* 1 .. 65535 */
    uint32_t head_dim;            /* rope->dims .. 1024 */
    uint32_t dtype;               /* of x and y */
    uint32_t transpose;
    uint32_t reserved;
    int64_t x_row, x_head;        /* strides in elements, >= 0 (0: the row or head is broadcast); channels are adjacent */
    int64_t y_row, y_head;        /* rows or heads outermost, and no two elements of y in one place */
} psv_rotate_args;
psv_status psv_rotate(const psv_rotate_args *a, const psv_rope *rope, void *stream);

/* ---- places in the cache ----------------------------------------------------------------------- */

/* Block tables and slot maps of a step, from the lengths of its requests.  Request b has lens[b] tokens in the cache and brings
 * new_lens[b] more (>= 0; 1 in a decode step, a prompt or a part of one otherwise); their rows follow one another, request by request,
 * in the step's row arrays.  Blocks that a request needs beyond those that hold its lens[b] tokens are taken from the free list, in
 * request order, and entered into its row of the block table.
 * A request is refused -- it keeps its length, takes no block, and its rows get slot -1, which append and gather skip -- when a length is negative, lens + new_lens
 * exceeds max_blocks * 16, its rows do not fit `rows`, or it needs blocks and the free list does not hold those of all requests up to it
 * (refused ones of the other kinds need none).  A negative new length stands for no rows.
 * Slot of the token at position p of request b: block_table[b][p / 16] * 16 + p % 16 -- what psv_cache_append and psv_cache_gather take --
 * or -1 where the block's id is not in [0, num_pool_blocks).
 * A decode step knows lengths alone: one over a refused request's kept length would write the new token over the last cached one.  Its seq_lens are
 * 0 there (an empty sequence, whose cache a step leaves alone); with one row a request, seq_lens[b] where slots[b] >= 0 and 0 elsewhere.
 * Nothing read is written (block_table apart, whose entries of held blocks are read and whose new ones are written), so a repeated call
 * gives the same answers; a program alternates between two sets of lens / seq_lens and free_range / free_range_out. */
typedef struct {
    const int32_t *lens;          /* dev [batch] tokens in the cache */
    const int32_t *new_lens;      /* dev [batch] */
    int32_t *block_table;         /* dev [batch][max_blocks], or NULL for a contiguous cache (block b * max_blocks + i) */
    const int32_t *free_blocks;   /* dev [free_capacity] block ids; ignored without a block table */
    const int32_t *free_range;    /* dev [2]: free_blocks[range[0]] .. free_blocks[range[1] - 1] are free; ignored without a block table */
    uint32_t free_capacity;
    uint32_t batch;               /* 1 .. PSV_SLOTS_MAX_BATCH */
    uint32_t max_blocks;
    uint32_t num_pool_blocks;
    uint32_t rows;                /* entries of the row arrays */
    uint32_t reserved;
    int32_t *seq_lens;            /* dev [batch] out: lens + new_lens, or lens where refused; psv_kv_desc's seq_lens of a decode step in which none was */
    int32_t *row_starts;          /* dev [batch + 1] out: first row of each request and the end of the last, at most `rows` */
    int64_t *slots;               /* dev [rows] out; -1 for rows of refused requests and behind the last */
    int32_t *positions;           /* dev [rows] out: lens + place within the request, refused ones included; 0 behind the last row */
    int32_t *requests;            /* dev [rows] out: the row's request; -1 behind the last row */
    int32_t *free_range_out;      /* dev [2] out; NULL without a block table */
    int32_t *refused;             /* dev [1] out: how many requests were refused */
} psv_slots_args;
#define PSV_SLOTS_MAX_BATCH 4096u
psv_status psv_cache_slots(const psv_slots_args *a, void *stream);

/* ---- rows into and out of the cache ------------------------------------------------------------- */

/* One layer's pools (preserve.h, KV-cache).  Of a call, rows * n_kv_heads <= 2^28 (else PSV_ERR_UNSUPPORTED). */
typedef struct {
    void *k_pool, *v_pool;        /* dev, 16-byte aligned */
    uint32_t n_kv_heads;          /* 1 .. 128 */
    uint32_t kv_format;           /* PSV_FMT_* */
    uint32_t kv_layout;           /* PSV_KV_* */
    uint32_t num_pool_blocks;
} psv_cache;

/* The rows of a prompt, or of one step of a program with its own attention: queries and keys are rotated (rope != NULL), keys and
 * values go into the cache, as the decode step does with its one token a sequence: computed in 32 bits, then rounded to bf16, or
 * quantised to int8 by the rule in preserve.h.  (A quotient that is not a number has the code -127 in both: a NaN's, and that of an infinity in its
 * own row, whose scale is infinite and whose finite elements have code 0.)  Rows are [heads][128] elements, rows of 16-byte aligned starts.
 * A slot outside [0, num_pool_blocks * 16) skips the row's key and value (its query is still rotated).  Slots must differ: which of
 * the rows that share one it ends up with, channel by channel, is not defined.
 * rope->dims must be a multiple of 16 and at most 128 (PSV_ERR_UNSUPPORTED). */
typedef struct {
    const void *q;                /* dev; NULL (n_q_heads = 0): no queries */
    const void *k, *v;            /* dev */
    void *q_out;                  /* dev; may be q, with equal strides */
    const int32_t *positions;     /* dev [rows]; may be NULL without rope */
    const int64_t *slots;         /* dev [rows] */
    uint32_t rows;                /* <= 2^24 */
    uint32_t n_q_heads;           /* <= 128 */
    uint32_t dtype;               /* of q, k, v and q_out */
    uint32_t reserved;
    int64_t q_row, k_row, v_row, q_out_row;   /* strides in elements */
} psv_append_args;
psv_status psv_cache_append(const psv_append_args *a, const psv_cache *cache, const psv_rope *rope, void *stream);

/* Rows of the cache as values: k[r], v[r] = the key and value at slots[r] ([kv heads][128], int8 codes times their scale, rounded once
 * to dtype).  A row whose slot is out of range is left as it was.  A slot may be named more than once. */
typedef struct {
    const int64_t *slots;         /* dev [rows] */
    void *k, *v;                  /* dev out */
    uint32_t rows;                /* <= 2^24 */
    uint32_t dtype;
    int64_t k_row, v_row;         /* strides in elements */
} psv_gather_args;
psv_status psv_cache_gather(const psv_gather_args *a, const psv_cache *cache, void *stream);

/* ---- answers ------------------------------------------------------------------------------------- */

/* Log probabilities, entropy and most likely tokens of rows of logits.  With x the logits of a row over the whole vocabulary, M their
 * largest, s the scale (1 / temperature), d_i = s (x_i - M) and S the sum of exp d_i:
 *   log p_i = d_i - ln S        entropy = ln S - (sum of d_i exp d_i) / S
 * computed in 32 bits.  Alternatives: the `top` tokens of the largest logits, largest first, equal ones by lowest id.
 * A masked logit (-infinity) has log probability -infinity, no part in the entropy, and is no alternative; where fewer than `top` remain
 * the rest are id -1 and -infinity.  A row whose mask leaves nothing has log probabilities -infinity and entropy 0.  A row that holds a
 * NaN or +infinity has NaN for all values and -1 for all ids.  A given token below 0 (padding) has log probability 0, one beyond the
 * vocabulary NaN.
 *
 * Tensor parallel: a shard has `columns` of the vocabulary, from `first_token` on.  psv_logprobs_part reduces them to `records` records
 * a row; the records of all shards, gathered behind one another, go to psv_logprobs_join, which gives every rank the answer.  psv_logprobs is
 * both, for one shard that has the whole vocabulary (columns = vocab, first_token = 0).  All shards take the same records, rows, given,
 * top and scale. */
#define PSV_LOGPROBS_MAX_TOP 32u
#define PSV_LOGPROBS_MAX_GIVEN 32u
#define PSV_LOGPROBS_MAX_RECORDS 256u      /* of all shards together, a row */
typedef struct {
    const void *logits;           /* dev [rows][columns] */
    const int32_t *tokens;        /* dev [rows][given]; NULL with given = 0 */
    uint32_t rows;                /* <= 2^20, and rows * records <= 2^23 (else PSV_ERR_UNSUPPORTED) */
    uint32_t columns;             /* 1 .. 2^21 */
    uint32_t first_token;
    uint32_t vocab;               /* first_token + columns .. 2^21 */
    uint32_t dtype;
    uint32_t given;               /* tokens a row, 0 .. PSV_LOGPROBS_MAX_GIVEN */
    uint32_t top;                 /* alternatives a row, 0 .. PSV_LOGPROBS_MAX_TOP */
    float    scale;               /* 2^-32 .. 2^32 */
    uint32_t records;             /* psv_logprobs_records of this shard or of one with more columns; 0: of this one */
    uint32_t reserved;
    int64_t  row;                 /* stride in elements, >= 0 (rows start at any element) */
} psv_logprobs_args;

typedef struct {
    float *logprobs;              /* dev [rows][given]; may be NULL */
    float *entropy;               /* dev [rows]; may be NULL */
    float *top_logprobs;          /* dev [rows][top]; NULL if top_ids is */
    int32_t *top_ids;             /* dev [rows][top]; may be NULL */
} psv_logprobs_out;

/* Records a row into which psv_logprobs_part divides `columns` (0 if an argument is out of range), and the bytes of the records of one
 * shard: 4 * rows * records * (4 + given + 2 top).  Pure host functions. */
uint32_t psv_logprobs_records(uint32_t rows, uint32_t columns);
size_t psv_logprobs_bytes(uint32_t rows, uint32_t records, uint32_t given, uint32_t top);
psv_status psv_logprobs_part(const psv_logprobs_args *a, void *records /* dev out, floats */, void *stream);
/* rows, given, top, vocab, scale, tokens and records of `a` are read (records: not 0). */
psv_status psv_logprobs_join(const psv_logprobs_args *a, const void *records /* dev [shards] of them */, uint32_t shards,
                             const psv_logprobs_out *out, void *stream);
psv_status psv_logprobs(const psv_logprobs_args *a, const psv_logprobs_out *out, void *workspace /* dev, psv_logprobs_bytes */,
                        size_t workspace_bytes, void *stream);

#ifdef __cplusplus
}
#endif
#endif
