/*
 * tm_paged - a quantised KV cache kept in pages, attention over it, and rotary positions; part of libtm_w4.
 *
 * The cache of tm_attn.h gives every sequence a slab of its own.  A server whose sequences come and go keeps pages instead: a pool of
 * equally large pages, and for every sequence a table of the pages that hold its tokens.  The codes, their rounding and their order inside a run of 32
 * tokens are those of tm_attn.h; new is where a run lies, that sequences bring different numbers of new tokens to one call, and that keys and queries
 * are rotated on the way in.
 *
 *     tm_rope_apply    rotary positions of packed tokens
 *     tm_paged_append  (rotates and) quantises new keys and values into their pages, rotates the queries along
 *     tm_paged_read    the cached keys and values back as fp16
 *     tm_paged_attn    causal attention of every sequence's new tokens over its pages
 *
 * Conventions as in tm_w4.h: plain C ABI, DEVICE pointers unless marked host, fp16 as uint16_t bit patterns, nothing synchronises or
 * allocates except the create calls, work is enqueued on the given stream, negative tm_status codes with tm_last_error().
 */
#ifndef TM_PAGED_H
#define TM_PAGED_H

#include "tm_attn.h"

#ifdef __cplusplus
extern "C" {
#endif

/* ------------------------------------------------------------------------------------------------ rotary positions
 *
 * The first rot_dim dimensions of a head form rot_dim / 2 pairs (x1, x2); at position p pair i becomes
 *     y1 = amplitude * (x1 cos(p f_i) - x2 sin(p f_i)),    y2 = amplitude * (x2 cos(p f_i) + x1 sin(p f_i)),
 * the other dimensions stay as they are.  Sines and cosines are right to 1e-11 at every int32 position and for every f_i that is accepted (up to 1e6), the result is rounded to
 * fp32 and then to fp16.
 */
typedef enum tm_rope_layout {
    TM_ROPE_HALF = 0,         /* pair i = dimensions (i, i + rot_dim / 2) */
    TM_ROPE_INTERLEAVED = 1   /* pair i = dimensions (2i, 2i + 1) */
} tm_rope_layout;

/* f_i for n = rot_dim and g_i = base^(-2i / n); the scaled forms stretch contexts of original_len tokens by `factor`. */
typedef enum tm_rope_scaling {
    TM_ROPE_PLAIN = 0,        /* g_i */
    TM_ROPE_LINEAR = 1,       /* g_i / factor */
    TM_ROPE_BASE = 2,         /* g_i of the base  base * factor^(n / (n - 2)) */
    TM_ROPE_WAVELENGTH = 3,   /* w g_i + (1 - w) g_i / factor,  w = (turns_i - low) / (high - low) limited to [0, 1], where
                                 turns_i = original_len * g_i / 2 pi is how often the pair turns over the original length */
    TM_ROPE_RAMP = 4          /* the same with w falling linearly in i between the pairs that turn `high` and `low` times:
                                 w = 1 - (i - a) / (b - a) limited to [0, 1], at(t) = n log(original_len / (2 pi t)) / (2 log base),
                                 a = max(floor(at(high)), 0), b = min(ceil(at(low)), n - 1) (b - a at least 0.001);
                                 its amplitude is 0.1 log(factor) + 1 */
} tm_rope_scaling;

typedef struct tm_rope_params {
    int rot_dim;                  /* a multiple of 16, 16 .. 256 */
    int layout;                   /* tm_rope_layout */
    int scaling;                  /* tm_rope_scaling */
    double base;                  /* above 1 */
    double factor;                /* >= 1; every scaling but TM_ROPE_PLAIN */
    double original_len;          /* > 0; TM_ROPE_WAVELENGTH and TM_ROPE_RAMP */
    double low, high;             /* 0 < low < high; the same two */
    double amplitude;             /* 0 = the scaling's own (1, or that of TM_ROPE_RAMP) */
    const double* frequencies;    /* host, rot_dim / 2 radians per position, -1e6 .. 1e6; if not NULL these are the f_i and the scaling counts for nothing but
                                     the amplitude */
} tm_rope_params;

typedef struct tm_rope tm_rope;   /* opaque; owns a table of rot_dim / 2 entries on the device */
TM_API tm_rope* tm_rope_create(const tm_rope_params* params);       /* synchronous copy; NULL on error */
TM_API void tm_rope_free(tm_rope* rope);
/* The f_i (host, rot_dim / 2) and the amplitude (host) that the handle works with; either may be NULL. */
TM_API int tm_rope_frequencies(const tm_rope* rope, double* frequencies, double* amplitude);

/*
 * X fp16 [tokens][heads][head_dim] -> Y of the same shape; token t at X + t * x_stride and Y + t * y_stride (strides in values, multiples of 8, at least
 * heads * head_dim; both pointers 16-byte aligned), so that parts of a fused projection's output are taken as they lie.  positions int32 [tokens], any value.  head_dim is a
 * multiple of 8 from rot_dim to 256.  Y may be X with the same stride; any other overlap is undefined.  tokens == 0 is a successful no-op.
 */
TM_API int tm_rope_apply(const uint16_t* X, int64_t x_stride, const int32_t* positions, const tm_rope* rope, uint16_t* Y, int64_t y_stride, int tokens,
                         int heads, int head_dim, tm_stream stream);

/* ------------------------------------------------------------------------------------------------ the paged cache
 *
 * The pool is the caller's memory (16-byte aligned), so that pages can be copied, shared and moved by whoever manages them:
 *     k, v    codes: run r of KV head h of page p at byte ((p * kv_heads + h) * (page_tokens / 32) + r) * 512 * bits; within a run
 *             of 32 tokens the order is that of a block of 32 tokens in tm_attn.h
 *     pairs   fp16 [pages][kv_heads][page_tokens][key, value][scale, zero-point]
 * page_tokens is 32, 64, ... 1024 (a power of two), bits 8 or 4.  What a page holds before tokens are stored in it may be anything.
 * `workspace` (256-byte aligned, tm_paged_workspace_bytes() bytes) must be zero-filled once before its first use; every call leaves it ready for the next
 * one.  Calls that share a workspace must be ordered on one stream; caches of layers that run after one another may share one.
 * The handle allocates nothing on the device; the memory stays the caller's and must outlive it.  NULL on error.
 */
typedef struct tm_paged_cache tm_paged_cache;
TM_API size_t tm_paged_workspace_bytes(void);
TM_API tm_paged_cache* tm_paged_create(uint8_t* k, uint8_t* v, uint16_t* pairs, int pages, int kv_heads, int page_tokens, int bits, void* workspace,
                                       size_t workspace_bytes);
TM_API void tm_paged_free(tm_paged_cache* cache);

/*
 * The sequences of a call.  New tokens are packed: rows offsets[b] .. offsets[b+1] - 1 of the token arrays belong to sequence b (offsets ascending, clamped to
 * [0, tokens]; rows outside them are not touched), row offsets[b] + i is the token at position positions[b] + i of its sequence.  Token t of sequence b lies in
 * page table[b][t / page_tokens]; an entry outside [0, pages) names no page, and what would lie there is not stored, not attended over and reads as zeros.
 * Everything marked device is read when the work runs, so a captured graph follows what the arrays hold at its replay.  A call that would take a launch of 2^32 threads or more is
 * refused: 256 for every 32 tokens and KV head that are stored or read, 512 for every 256 rows (or 128) of a KV head that attend, parts of a sequence counted whole.
 */
typedef struct tm_paged_batch {
    const int32_t* table;         /* device [batch][max_pages] */
    const int32_t* offsets;       /* device [batch + 1] */
    const int32_t* positions;     /* device [batch] */
    int batch;                    /* sequences, 1 .. 65535 */
    int max_pages;                /* entries of a table row; max_pages * page_tokens < 2^30 */
    int tokens;                   /* rows of the packed arrays */
    int max_count;                /* host hints, 0 = unknown: most new tokens of a sequence, and most tokens of one (cached and new).  They choose between */
    int max_len;                  /* kernels and launch shapes; results do not depend on them beyond rounding. */
} tm_paged_batch;

/*
 * Stores the new tokens: K, V fp16 [tokens][kv_heads][128], row r at K + r * k_stride and V + r * v_stride (strides in values, multiples of 8, at least
 * kv_heads * 128; pointers 16-byte aligned).  With a rope (rot_dim <= 128) keys are rotated for their positions and rounded to fp16 before they are quantised, as by
 * tm_rope_apply, and if Q is not NULL so are the queries, Q fp16 [tokens][q_heads][128] -> Q_out (strides as for tm_rope_apply; Q_out may be Q).  Without one Q must be NULL.
 * Tokens at positions outside [0, max_pages * page_tokens) are dropped (their queries are rotated all the same).  Codes are those of tm_kv_append, bit for bit.
 * A page that a call writes to belongs to one sequence of that call, at one place of its table; else its contents are undefined.
 * Appends to one pool must be ordered on one stream.
 */
TM_API int tm_paged_append(tm_paged_cache* cache, const tm_paged_batch* batch, const uint16_t* K, int64_t k_stride, const uint16_t* V, int64_t v_stride,
                           const tm_rope* rope, const uint16_t* Q, int64_t q_stride, uint16_t* Q_out, int64_t q_out_stride, int q_heads, tm_stream stream);

/*
 * Reads cached tokens back: row offsets[b] + i of K and V, fp16 [tokens][kv_heads][128] (16-byte aligned), becomes fp16((q - z) * s) of the token at
 * position positions[b] + i.  Rows whose position lies outside [0, max_pages * page_tokens) are left untouched.
 */
TM_API int tm_paged_read(const tm_paged_cache* cache, const tm_paged_batch* batch, uint16_t* K, uint16_t* V, tm_stream stream);

/*
 * Attention of the new tokens.  Q fp16 [tokens][q_heads][128] (row r at Q + r * q_stride, as for tm_rope_apply), O fp16 [tokens][q_heads][128] contiguous,
 * both 16-byte aligned, not overlapping: row offsets[b] + i, the query at position p = positions[b] + i of its sequence, attends over the cached tokens 0 .. p, its own
 * included, so its key and value have to be stored first (tm_paged_append, on the same stream):
 *     O = softmax(scale * K^ q) V^,   query head h with KV head h / (q_heads / kv_heads),   q_heads = 1 .. 128 times kv_heads.
 * Tokens on pages that the pool does not have are not attended over; a row that is left with none gets O = 0.  Rows whose position lies outside
 * [0, max_pages * page_tokens) are left untouched.  One token a sequence is a decoding step, a few are drafted tokens to be verified, hundreds a prompt; a call takes any mix.
 * As by tm_attn_decode and tm_attn_prefill, each probability (relative to about the largest) times its value's scale is rounded to fp16, by at most 2^-11 of it or 2^-25; everything else is
 * held in fp32 up to the result's own rounding.
 * Work is counted in 32 bits, so a call must have less than 2^30 rows (tokens * q_heads / kv_heads), and (rows / 8 + batch) * kv_heads times (max_pages * page_tokens / 128 + 1)
 * must stay below 2^31: 64 decoding sequences of 8 KV heads and 4 query heads each take tables of up to 2^28 tokens.  Others are refused, whatever the lengths.
 * Never allocates.  Partial results go through the cache's workspace.  Results are bit-identical from run to run (same arguments and hints).
 */
TM_API int tm_paged_attn(const uint16_t* Q, int64_t q_stride, const tm_paged_cache* cache, const tm_paged_batch* batch, uint16_t* O, int q_heads, float scale,
                         tm_stream stream);

/*
 * Query hook: how tm_paged_attn divides such a call (host out-pointers, any may be NULL).  Sequences with up to *column_rows (token, query head of a KV head) rows, *columns of
 * them at a time (8, 16 or 32; 0 = no such launch), the others in CTAs of *rows rows (128 or 256; 0 = no such launch), their contexts in up to *pieces.
 */
TM_API int tm_get_paged_plan(const tm_paged_cache* cache, const tm_paged_batch* batch, int q_heads, int* columns, int* column_rows, int* rows, int* pieces);
/*
 * Further: *launches of a call, *column_ctas, the CTAs that take the columns (0 = none do), and *alone, 1 if every wave of them works by itself.  Columns and rows of a call go in
 * one launch, the rows' pieces are put together in another.
 */
TM_API int tm_get_paged_form(const tm_paged_cache* cache, const tm_paged_batch* batch, int q_heads, int* launches, int* column_ctas, int* alone);

#ifdef __cplusplus
}
#endif
#endif /* TM_PAGED_H */
