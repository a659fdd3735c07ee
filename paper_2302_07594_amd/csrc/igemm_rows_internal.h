// Internal declarations of the products whose rows choose their weights
// (igemm_rows.h): the kernels' arguments and launches.
#pragma once

#include <stdint.h>

#include "igemm_internal.h"
#include "igemm_rows.h"

namespace igemm {
namespace rows {

// One grouped product, as the kernels take it. groups = 1 with offsets null is
// the shared projection: every position belongs to the one group.
struct Product {
    const int8_t *A, *B;
    const float *scale_a, *scale_b;
    const int32_t *offsets, *order;
    void *out;
    int64_t lda, ldb, stride_b, ldo;
    int rows, n, k, groups, a_rows, out_rows, slots, scatter, type;
};

// The adapters beside a projection (adapters = 0: none).
struct Adapters {
    const int32_t *ids, *ranks;
    const void *down, *up;
    const float *scaling;
    int64_t ld_down, stride_down, ld_up, stride_up;
    int adapters, rank, type;
};

// Row tiles of bm rows at most: every group with rows may end inside one.
inline int64_t most_tiles(int64_t rows, int64_t groups, int64_t bm) {
    const int64_t used = groups < rows ? groups : rows;
    return (rows + used * (bm - 1)) / bm;
}

int launch_route(const igemm_route_desc &d, const void *logits, int64_t ld, const float *bias,
                 int32_t *ids, float *weights, int32_t *offsets, int32_t *order, void *workspace,
                 void *stream);
int64_t route_workspace(const igemm_route_desc &d, bool plan);

int launch_product(const Product &p, const Adapters &ad, int num_cu, void *workspace,
                   void *stream);
int64_t product_workspace(int64_t rows, int64_t n, int64_t k, int64_t groups, int64_t adapters,
                          int64_t rank, int num_cu);

int launch_combine(int64_t tokens, int64_t top_k, int64_t n, int type, const void *Z, int64_t ldz,
                   const float *weights, const int32_t *ids, const void *base, int64_t ld_base,
                   void *out, int64_t ldo, void *stream);

}  // namespace rows
}  // namespace igemm
