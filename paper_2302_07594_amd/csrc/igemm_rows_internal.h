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

inline int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }

// The ring of k-tiles: 128 k, one whole line of a row of A.
constexpr int kStepK = 128;
constexpr int kShrinkK = 1024;   // k a workgroup of a sliced product's shrink_row
constexpr int kShrinkRows = 32;  // rows a workgroup of shrink_tiles

// How a product is cut (igemm_rows_plan.cpp).
struct Choice {
    int bm, bn;       // tile
    int slices, kchunk;
    bool by_row;      // u: a workgroup a row (and k slice, where the product is
    int ks, rpad;     // sliced: ks of kShrinkK), else blocks of 32 rows and
    int shrink_ranks; // so many ranks
    int64_t u_bytes, part_bytes;
};
// By sizes alone, so that the workspace can be sized before the operands exist.
Choice choose(int64_t rows, int64_t n, int64_t k, int64_t groups, int64_t adapters, int64_t rank,
              int num_cu);
// The tile that these operands take, and whether through registers.
struct Tile {
    int bm, bn;
    bool reg;
};
Tile tile_of(const Choice &c, const Product &p, const Adapters &ad, int num_cu);

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
