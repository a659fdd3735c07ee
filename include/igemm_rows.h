/*
 * igemm_rows.h -- products whose rows choose their weights, on AMD Instinct
 * MI355X (gfx950): the routing of tokens to experts, the experts' int8 products,
 * the sum of a token's results, and a shared int8 projection beside which each
 * row has the low-rank adapter of its request (inference of language models
 * with int8 weights). Part of the library of igemm.h (from igemm_version 500 on),
 * whose status codes and igemm_strerror apply.
 *
 * Operands and results are DEVICE pointers owned by the caller. Checks,
 * asynchrony and errors are those of igemm.h: arguments are checked on the host
 * before any HIP call, kernels are enqueued on `stream`, the library allocates
 * nothing. What is read on the device (offsets, order, ids, ranks) is not checked
 * on the host: entries out of range choose nothing, and never lead a read or write
 * out of the arrays described here. As in igemm.h, elements between the rows of an
 * int8, down or up matrix, and bytes of the aligned 16 that hold its first or last
 * element, may be read; their values never matter. Values are the same from run to
 * run, bit for bit (but for rows of out that several positions name).
 */
#ifndef IGEMM_ROWS_H
#define IGEMM_ROWS_H

#include <stdint.h>

#include "igemm.h"

#ifdef __cplusplus
extern "C" {
#endif

typedef enum igemm_type {
    IGEMM_F32 = 0,
    IGEMM_BF16 = 1,
    IGEMM_F16 = 2
} igemm_type;

/*
 * Routing: for each token t (a row of `experts` logits l)
 *
 *   s[e]   = exp(l[e]) / sum exp(l)   (score IGEMM_SOFTMAX)
 *            1 / (1 + exp(-l[e]))     (score IGEMM_SIGMOID)
 *   key[e] = s[e] + bias[e]           (bias NULL: key = s)
 *
 * The experts form `groups` groups of consecutive indices; a group's key is the
 * sum of its group_best (1 or 2) largest keys, and only the experts of the
 * top_groups groups of largest key stay. Of these the top_k experts of largest
 * key are chosen, largest first; equal keys go to the lower index, in both
 * steps. A chosen expert's weight is scale * s[e], with renormalise
 * scale * s[e] / (the sum of the chosen s; weights 0 where that is 0).
 *
 * Keys are compared as in 64-bit floating point. Where the keys are in the order of
 * the logits (no bias, and one group or group_best 1) the logits are compared.
 * Logits of -infinity or NaN, and keys of -infinity or NaN, exclude their
 * expert: its score is 0 and it is not chosen (the best two of a group with
 * one expert left are that one; a group with none is not chosen). A logit of
 * +infinity counts as the largest finite float. Slots that find no expert have
 * id -1 and weight 0, so a padded token is a row of -infinity.
 *
 *   logits   tokens x experts of `type`, rows of unit stride, ld >= experts.
 *   bias     experts floats or NULL.
 *   ids      tokens x top_k int32, dense: the chosen expert, or -1. Slot t * top_k
 *            + j is choice j of token t.
 *   weights  tokens x top_k floats, dense.
 *   offsets, order   the plan of the experts' products, or both NULL: order
 *            (tokens * top_k int32) lists the slots by expert, those of one
 *            expert ascending; offsets (experts + 1 int32) where each
 *            expert's begin. Entries of order from offsets[experts] on are -1.
 *   workspace  device memory, 256-byte aligned, at least the bytes
 *            igemm_route_query reports (IGEMM_ENOMEM otherwise; 0: NULL is
 *            accepted); calls that share one must be ordered.
 *
 * Errors: IGEMM_EINVAL for a NULL descriptor or array, experts, top_k, groups,
 * top_groups or group_best out of their ranges (top_k <= experts, groups a
 * divisor of experts, 1 <= top_groups <= groups), ld < experts, or a scale
 * that is not finite; IGEMM_ENOTSUP for more than 1024 experts, top_k or groups
 * over 64, or tokens * top_k beyond 2^31 - 2^16. tokens = 0 writes offsets alone.
 */
#define IGEMM_SOFTMAX 0
#define IGEMM_SIGMOID 1
typedef struct igemm_route_desc {
    int64_t tokens;
    int experts, top_k;
    int groups, top_groups, group_best;
    int score;         /* IGEMM_SOFTMAX or IGEMM_SIGMOID */
    int renormalise;   /* 0 or 1 */
    float scale;
    int type;          /* igemm_type of the logits */
} igemm_route_desc;
int igemm_route_query(const igemm_route_desc *desc, int64_t *workspace_bytes);
int igemm_route(const igemm_route_desc *desc, const void *logits, int64_t ld, const float *bias,
                int32_t *ids, float *weights, int32_t *offsets, int32_t *order, void *workspace,
                int64_t workspace_bytes, void *stream);

/*
 * The experts' products. Positions 0 .. rows - 1 are sorted by group: group g
 * has the positions offsets[g] <= i < offsets[g + 1]. With the slot
 * s = order[i] (order NULL: s = i), the row a = i (slots 0) or s / slots of A
 * and the row o = i (scatter 0) or s of out,
 *
 *   out[o, j] = scale_a[a] * scale_b[g, j] * sum over p of A[a, p] * B[g, p, j]
 *
 * The sum is exact, converted to float, multiplied by scale_a, then scale_b
 * (NULL: 1), and rounded to `type` once. out is overwritten. Rows of out that no
 * position reaches, among them those of positions from offsets[groups] on, are
 * left as they were. If several positions name one row of out, each of its elements is
 * one of theirs, not always the same one from run to run.
 * A position whose row of A or out is outside a_rows or out_rows is skipped.
 *
 *   offsets  groups + 1 int32, ascending (or the values of out are not specified);
 *            values outside [0, rows] act as the nearest bound.
 *   order    rows int32, or NULL.
 *   A        a_rows x k int8, row-major, leading dimension lda >= k.
 *   scale_a  a_rows floats or NULL.
 *   B        groups matrices k x n int8, row-major with leading dimension ldb,
 *            group g at B + g * stride_b (elements; stride_b >= 0).
 *   scale_b  groups x n floats, dense, or NULL.
 *   out      out_rows x n of `type`, row-major, ldo >= n; it must not overlap
 *            the inputs.
 *   workspace  as for igemm_route, sized by igemm_i8_grouped_query (num_cu: the
 *            device's compute units).
 *
 * Errors: IGEMM_EINVAL as for igemm_i8, and for slots < 0, scatter not 0 or 1 or
 * an unknown type; IGEMM_ENOTSUP for k beyond 131071 (sums past 2^31), extents
 * beyond 2^31 - 1, more than 65536 groups, an A or a matrix of B within 256 bytes of
 * 2 GiB or over, 256 rows of out of 2 GiB or more, or a grid of 2^32 threads. rows = 0
 * or n = 0: IGEMM_OK, out unchanged. k = 0: zeros.
 */
typedef struct igemm_grouped_desc {
    int64_t rows, n, k, groups;
    int64_t a_rows, out_rows;
    int64_t slots;   /* 0: A's row is the position; else order[i] / slots */
    int scatter;     /* 0: out's row is the position; 1: order[i]         */
    int type;        /* igemm_type of out                                 */
} igemm_grouped_desc;
int igemm_i8_grouped_query(const igemm_grouped_desc *desc, int num_cu, int64_t *workspace_bytes);
int igemm_i8_grouped(const igemm_grouped_desc *desc, const int32_t *offsets,
                     const int32_t *order, const int8_t *A, int64_t lda, const float *scale_a,
                     const int8_t *B, int64_t ldb, int64_t stride_b, const float *scale_b,
                     void *out, int64_t ldo, void *workspace, int64_t workspace_bytes,
                     void *stream);

/*
 * The sum of each token's slots:
 *   out[t, :] = base[t, :] + sum over j of weights[t, j] * Z[t * top_k + j, :]
 * in float, in order of j, rounded to `type` once. Slots whose id is negative
 * are left out, whatever Z and the weight hold there.
 *   Z        tokens * top_k rows of n, ldz >= n, of `type` (as base and out).
 *   weights  tokens x top_k floats, dense.
 *   ids      tokens x top_k int32, dense, or NULL (every slot counts).
 *   base     tokens x n, ld_base >= n, or NULL (0). May be out itself.
 *   out      tokens x n, ldo >= n; overwritten; overlaps neither Z nor, unless
 *            it is the same, base.
 * Errors: IGEMM_EINVAL as for igemm_i16 (top_k >= 1); IGEMM_ENOTSUP for n, tokens
 * or top_k beyond 2^31 - 1 or a grid of 2^32 threads (64 GiB of out). tokens = 0 or
 * n = 0: IGEMM_OK.
 */
int igemm_combine(int64_t tokens, int64_t top_k, int64_t n, int type, const void *Z, int64_t ldz,
                  const float *weights, const int32_t *ids, const void *base, int64_t ld_base,
                  void *out, int64_t ldo, void *stream);

/*
 * A shared int8 projection and, beside it, the low-rank adapters of many requests
 * in one batch. With a = ids[i] (none if outside [0, adapters)), r < ranks[a]:
 *
 *   out[i, j] = scale_a[i] * scale_b[j] * sum over p of A[i, p] * B[p, j]
 *               + sum over r of u[i, r] * up[a, j, r]
 *   u[i, r]   = scaling[a] * scale_a[i] * sum over p of A[i, p] * down[a, r, p]
 *
 * The first sum is exact; the others are held in 32-bit floating point (u is
 * carried into the second in parts that add up to at least 22 bits of its row's
 * largest value, or to 2^-134), and the result is rounded to `type` once. Nothing of
 * an adapter, infinities and NaN included, reaches the rows of another; in its own
 * rows they give what the formula gives (but for an infinite `up` against a u below
 * 2^-100 that is not 0, which may give NaN).
 *
 *   A, scale_a, B, scale_b, out   as for igemm_i8_grouped with one group: m x k,
 *            k x n (ldb), m x n (ldo); scale_a m floats, scale_b n floats, or NULL.
 *   ids      m int32.
 *   down     adapters x rank x k of weight_type (IGEMM_BF16 or IGEMM_F16): row r of
 *            adapter a at down + a * stride_down + r * ld_down (elements), its
 *            k values consecutive: the adapter's first matrix as it is
 *            trained and saved, a row per output.
 *   up       adapters x n x rank: row j at up + a * stride_up + j * ld_up.
 *   ranks    adapters int32 or NULL (all `rank`): values outside [0, rank] act as
 *            the nearest bound; what lies beyond an adapter's rank is not read
 *            into the result.
 *   scaling  adapters floats or NULL (1).
 *   workspace  as for igemm_route, sized by igemm_i8_adapters_query.
 * adapters = 0 or rank = 0: the projection alone (ids, down and up may be NULL).
 *
 * Errors: as for igemm_i8_grouped; IGEMM_ENOTSUP for rank beyond 1024 or a matrix of
 * down or up of 2 GiB or more.
 */
typedef struct igemm_adapters_desc {
    int64_t m, n, k;
    int64_t adapters, rank;
    int type;          /* igemm_type of out */
    int weight_type;   /* igemm_type of down and up */
} igemm_adapters_desc;
int igemm_i8_adapters_query(const igemm_adapters_desc *desc, int num_cu,
                            int64_t *workspace_bytes);
int igemm_i8_adapters(const igemm_adapters_desc *desc, const int8_t *A, int64_t lda,
                      const float *scale_a, const int8_t *B, int64_t ldb, const float *scale_b,
                      const int32_t *ids, const void *down, int64_t ld_down,
                      int64_t stride_down, const void *up, int64_t ld_up, int64_t stride_up,
                      const int32_t *ranks, const float *scaling, void *out, int64_t ldo,
                      void *workspace, int64_t workspace_bytes, void *stream);

#ifdef __cplusplus
}
#endif

#endif /* IGEMM_ROWS_H */
