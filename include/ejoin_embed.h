/*
 * ejoin_embed -- operators of libejoin.so around a table of vectors that is being learnt: products of rows held in
 * 8-bit floating point, rows looked up by token and the gradient of that, and the loss that fits scores to lists of ids
 * with logits (a teacher's top entries, or the neighbour lists that the joins of ejoin.h return).
 *
 * Conventions are those of ejoin.h: device pointers owned by the caller, calls that enqueue on `stream` and return,
 * EJOIN_OK or a negative code with nothing enqueued, no two calls at a time on one context.  What differs:
 *   - Matrices are row-major with a row stride in elements >= their width; rows need no alignment and no padding
 *     except where a call says so.
 *   - A call that needs device memory to work in takes it from the context, which grows it on demand (the growth
 *     waits for the device, as that of the joins' workspace does) or ahead of time (ejoin_embed_reserve).  Where a
 *     call is to be captured into a graph the memory has to be there before.  A graph works in the memory that it was captured
 *     with: the context keeps it until it is destroyed, also when it has grown since, and a replay is a call on the context like any other.
 *   - Sizes of zero rows are allowed where noted, and enqueue nothing.
 *   - Results are the same bits from call to call: no sum is taken in an order that depends on timing.
 */
#ifndef EJOIN_EMBED_H
#define EJOIN_EMBED_H

#include "ejoin.h"

#ifdef __cplusplus
extern "C" {
#endif

/* Types of elements and of tokens. */
#define EJOIN_F32 0
#define EJOIN_F16 1
#define EJOIN_BF16 2
#define EJOIN_I32 0
#define EJOIN_I64 1

/* Grow the memory that the calls below work in to `bytes`.  What each needs is stated with it. */
int ejoin_embed_reserve(ejoin_ctx* ctx, int64_t bytes);

/* ------------------------------------------------------------------ rows in 8-bit floating point
 * A row of d coordinates is cut into blocks of 128.  Block b holds x[k] as the nearest (ties to even) 8-bit value of
 * x[k] * 2^-e, 2^e the least power of two that brings the block's largest finite magnitude into the format's range (448 for
 * E4M3, 57344 for E5M2); e + 127 is the block's scale byte, cut off at 0 (and 127 for a block of zeros).  So no value
 * saturates, and multiplying by a scale never rounds; only magnitudes from 1.9375 * 2^127 on (from 1.875 * 2^127 in E5M2), FP32's and BF16's lowest value among
 * them, which would round up to 2^128, are held as the value below it, so that whatever is finite stays a finite FP32 value.
 * NaN stays NaN; an infinity becomes NaN in E4M3 and stays one in E5M2.
 *   values  n rows of roundup(d, 128) bytes, row stride ld (a multiple of 128, at most 2^23), 128-byte aligned; coordinates d and up are zero
 *   scales  n rows of roundup(ceil(d / 128), 4) bytes, row stride ld_scales (a multiple of 4, at most 2^24), 4-byte aligned;
 *           bytes past the last block hold 127 */
#define EJOIN_E4M3 0
#define EJOIN_E5M2 1
typedef struct {
  uint8_t* values;
  uint8_t* scales;
  int64_t ld;
  int64_t ld_scales;
  int64_t n; /* rows */
  int64_t d; /* coordinates */
  int32_t format;
} ejoin_f8_rows;

/* X (n x d, row stride ldx >= d) into 8-bit rows: `rows` takes X's own rows (rows->n = n, rows->d = d), `columns` those
 * of X transposed (columns->n = d, columns->d = n); either may be NULL.  Both are host structs whose format,
 * pointers and strides the caller fills in; with both, X is read once.  1 <= n, d < 2^23; rows alone may be up to 2^31 - 1. */
int ejoin_f8_quantize(ejoin_ctx* ctx, const void* X, int32_t type, int64_t n, int64_t d, int64_t ldx, const ejoin_f8_rows* rows,
                      const ejoin_f8_rows* columns, void* stream);

/* C[i][j] = scale * sum_k a_ik b_jk for the rows of A and of B (A->d = B->d), summed on the matrix cores block by block in
 * ascending order of k (in several pieces of that order, added up in it, where there are few tiles), rounded once to `type`.
 * FP32 results are sums in FP32 of the exact products (of values held; those below 2^-126 are taken to the nearest 2^-133).  So are 16-bit results before
 * they are rounded, where A has up to 64 rows of up to 1,024 coordinates (48 of 1,280, 32 of 2,048, 16 of 4,096) or where k is cut into pieces.  Other 16-bit
 * results come from the 8-bit matrix cores, whose sums of eight products keep no more than 13 bits below the largest of them: some 1.5e-5 of the result's norm,
 * up to 2^-10 of sum |a b| where sums cancel.  A row's bits may thus differ with the rows beside it; FP32 results are the call for sums that cancel.
 * C: A->n x B->n, row stride ldc; rows that are 16-byte aligned are written faster than others.
 * Formats may differ.  Works in at most EJOIN_F8_PRODUCT_BYTES of the context's memory. */
#define EJOIN_F8_PRODUCT_BYTES (128ll << 20)
int ejoin_f8_product(ejoin_ctx* ctx, const ejoin_f8_rows* A, const ejoin_f8_rows* B, float scale, void* C, int32_t type, int64_t ldc, void* stream);

/* The same for rows X (m x B->d, of type xtype, row stride ldx) that are quantised to E4M3 within the call: the scores
 * of m query rows against a table held in 8 bits.  Works in a further m * (roundup(d, 128) + roundup(ceil(d / 128), 4)) bytes, rounded up to 256. */
int ejoin_f8_scores(ejoin_ctx* ctx, const void* X, int32_t xtype, int64_t m, int64_t ldx, const ejoin_f8_rows* B, float scale, void* C, int32_t type,
                    int64_t ldc, void* stream);

/* ------------------------------------------------------------------ rows by token
 * Y[t][k] = round(scale * table[tokens[t]][k]) for k < d, zero for d <= k < roundup(d, 64): the layout that the
 * joins take, where ldy is a multiple of 64 and Y's type FP16.  table: v x d, row stride ldt; Y: t rows, row stride ldy >= roundup(d, 64).
 * A token of -1 stands for none: its row is zero.  So is that of any other token outside 0 .. v-1, which ejoin_embed_status reports.
 * t = 0 enqueues nothing. */
int ejoin_lookup(ejoin_ctx* ctx, const void* table, int32_t type, int64_t v, int32_t d, int64_t ldt, const void* tokens, int32_t token_type, int64_t t,
                 float scale, void* Y, int32_t ytype, int64_t ldy, void* stream);

/* The gradient of that with respect to the table, every row of it written:
 *   G[r][k] = round(scale * sum of dY[t][k] over the t with tokens[t] = r),  r < v, k < d,
 * summed in FP32 in ascending order of t (in pieces of that order, added up in it).  Tokens outside 0 .. v-1 are left
 * out (and reported, but for -1).  dY: t rows of d, row stride ldy; t < 2^31, v < 2^31; t = 0 gives zeros.  Works in at most
 * 17 * t + 8 * (d + 8) * (t / 32 + 1) + 4096 bytes of the context's memory, of up to 8,192 tokens in none. */
int ejoin_lookup_grad(ejoin_ctx* ctx, const void* dY, int32_t type, int64_t t, int32_t d, int64_t ldy, const void* tokens, int32_t token_type, int64_t v,
                      float scale, void* G, int32_t gtype, int64_t ldg, void* stream);

/* What the lookups, their gradients and the losses on this context saw since it was last asked: EJOIN_STATUS_OK, or
 * EJOIN_STATUS_TOKEN where a token or id was neither -1 nor inside its range.  Waits for the device; *status is a host pointer. */
#define EJOIN_STATUS_TOKEN 3
int ejoin_embed_status(ejoin_ctx* ctx, int* status);

/* ------------------------------------------------------------------ the loss against lists of ids with logits
 * Row t has scores (logits) Z[t][0 .. v-1] and a list of up to k ids with logits teacher[t][0 .. k-1].  An id of -1
 * stands for no entry; so does any other id outside 0 .. v-1 (reported by ejoin_embed_status), and an entry whose teacher
 * logit is -infinity.  With T the temperature,
 *   p = softmax of teacher / T over the entries of the row,   q = softmax of Z / T over the row,
 *   loss[t] = T^2 * sum_i p_i (log p_i - log q_id(i)),   lse[t] = log sum_j exp(Z[t][j] / T),
 * and, for a loss of sum_t weights[t] * loss[t],
 *   dZ[t][j] = weights[t] * T * (q_j * (sum_i p_i) - sum of the p_i with id(i) = j),
 * in FP32, rounded once.  sum_i p_i is 1, or 0 for a row without entries: its loss and gradient are zero, whatever its scores
 * hold.  An id may stand in a list more than once.  Scores of -infinity are left out (q = 0); one that an entry names
 * makes the loss infinite; a NaN or +infinity makes the row's loss, lse and gradient NaN.  Of a row that holds nothing but
 * -infinity all q are 0.  A NaN or +infinity among the entries' logits makes the row's loss NaN, and the gradient where its entries point.
 *   Z, dZ    t x v, row strides ldz, lddz, both of type ztype; dZ may be Z
 *   ids      t x k, row stride ldi;  teacher FP32, t x k, row stride ldi
 *   0 <= k <= EJOIN_DISTILL_MAX_ENTRIES;  1 <= v < 2^31;  t = 0 enqueues nothing;  temperature finite and at least 4.24e-39 (log2(e) / T is finite) */
#define EJOIN_DISTILL_MAX_ENTRIES 1024
/* Each call works in at most 16 KiB + 16 * t bytes of the context's memory, where rows are not cut into pieces (few or very long ones are) in none. */
int ejoin_distill(ejoin_ctx* ctx, const void* Z, int32_t ztype, int64_t t, int64_t v, int64_t ldz, const void* ids, int32_t id_type, const float* teacher,
                  int32_t k, int64_t ldi, float temperature, float* loss, float* lse, void* stream);
/* The gradient, from the lse of the forward call (what a differentiation engine keeps).  q is exp(Z / T - lse), so it carries the rounding of
 * an lse in FP32: a factor of exp(|lse| 2^-24), 1.00006 at an lse of 1,000, and anything between 0 and v where |lse| passes 2^24 (a row that holds
 * the type's lowest value throughout).  ejoin_distill_with_grad goes by (largest score, sum) and has no such limit. */
int ejoin_distill_grad(ejoin_ctx* ctx, const void* Z, int32_t ztype, int64_t t, int64_t v, int64_t ldz, const float* lse, const void* ids, int32_t id_type,
                       const float* teacher, int32_t k, int64_t ldi, const float* weights, float temperature, void* dZ, int64_t lddz, void* stream);
/* Loss and gradient in one call, Z read once but for few rows of more than 53,248 scores and rows that no workgroup's registers hold. */
int ejoin_distill_with_grad(ejoin_ctx* ctx, const void* Z, int32_t ztype, int64_t t, int64_t v, int64_t ldz, const void* ids, int32_t id_type,
                            const float* teacher, int32_t k, int64_t ldi, const float* weights, float temperature, float* loss, void* dZ, int64_t lddz,
                            void* stream);

#ifdef __cplusplus
}
#endif
#endif /* EJOIN_EMBED_H */
