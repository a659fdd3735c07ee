// The C entry points of igemm_rows.h: validation and dispatch. Every check
// runs on the host before any HIP call; the library allocates no device memory.
#include <hip/hip_runtime.h>
#include <math.h>
#include <stdint.h>

#include "igemm.h"
#include "igemm_internal.h"
#include "igemm_rows.h"
#include "igemm_rows_internal.h"

namespace igemm {
namespace rows {
namespace {

constexpr int64_t kMax = 0x7fffffff;
constexpr int64_t kMaxK = 131071;  // 2^14 a product: sums below 2^31

bool type_ok(int t) { return t == IGEMM_F32 || t == IGEMM_BF16 || t == IGEMM_F16; }
bool half_type(int t) { return t == IGEMM_BF16 || t == IGEMM_F16; }
int64_t size_of(int t) { return t == IGEMM_F32 ? 4 : 2; }
bool aligned(const void *p, int64_t to) { return (uintptr_t)p % (uintptr_t)to == 0; }

// Bytes of rows x cols elements of es bytes at leading dimension ld, or -1 where
// that does not fit 63 bits.
int64_t extent(int64_t rows, int64_t cols, int64_t ld, int64_t es) {
    if (rows <= 0 || cols <= 0) return 0;
    int64_t b = 0;
    if (__builtin_mul_overflow(rows - 1, ld, &b) || __builtin_add_overflow(b, cols, &b) ||
        __builtin_mul_overflow(b, es, &b))
        return -1;
    return b;
}

int check_workspace(const void *workspace, int64_t bytes, int64_t need) {
    if (workspace != nullptr && (!aligned(workspace, 256) || bytes < 0)) return IGEMM_EINVAL;
    if (need > 0 && (workspace == nullptr || bytes < need)) return IGEMM_ENOMEM;
    return IGEMM_OK;
}

int check_route(const igemm_route_desc *d) {
    if (d == nullptr || d->tokens < 0 || d->experts < 1 || d->top_k < 1 ||
        d->top_k > d->experts || d->groups < 1 || d->groups > d->experts ||
        d->experts % d->groups != 0 || d->top_groups < 1 || d->top_groups > d->groups ||
        (d->group_best != 1 && d->group_best != 2) ||
        (d->score != IGEMM_SOFTMAX && d->score != IGEMM_SIGMOID) ||
        (d->renormalise != 0 && d->renormalise != 1) || !isfinite(d->scale) || !type_ok(d->type))
        return IGEMM_EINVAL;
    if (d->experts > 1024 || d->top_k > 64 || d->groups > 64 || d->tokens > (kMax - 65535) / d->top_k)
        return IGEMM_ENOTSUP;
    return IGEMM_OK;
}

// m x k int8 A, k x n int8 B (groups of them) and an output of the given rows.
int check_product(int64_t a_rows, int64_t out_rows, int64_t n, int64_t k, int64_t groups, int type) {
    if (a_rows < 0 || out_rows < 0 || n < 0 || k < 0 || groups < 0 || !type_ok(type))
        return IGEMM_EINVAL;
    if (a_rows > kMax || out_rows > kMax || n > kMax || groups > 65536 || k > kMaxK)
        return IGEMM_ENOTSUP;
    return IGEMM_OK;
}
int check_operands(int64_t a_rows, int64_t n, int64_t k, const void *A, int64_t lda,
                   const void *B, int64_t ldb, const void *out, int64_t ldo, int type,
                   const float *scale_a, const float *scale_b) {
    if (out == nullptr || ldo < n || !aligned(out, size_of(type)) || !aligned(scale_a, 4) ||
        !aligned(scale_b, 4))
        return IGEMM_EINVAL;
    if (ldo > kMax || extent(256, n, ldo, size_of(type)) > kMax) return IGEMM_ENOTSUP;
    if (k == 0) return IGEMM_OK;
    if (A == nullptr || B == nullptr || lda < k || ldb < n) return IGEMM_EINVAL;
    if (lda > kMax || ldb > kMax) return IGEMM_ENOTSUP;
    const int64_t a = extent(a_rows, k, lda, 1), b = extent(k, n, ldb, 1);
    // (32-bit offsets, of a k-tile that may reach past the end)
    if (a < 0 || a > kMax - 256 || b < 0 || b > kMax - 256) return IGEMM_ENOTSUP;
    return IGEMM_OK;
}

int check_grouped(const igemm_grouped_desc *d) {
    if (d == nullptr || d->rows < 0 || d->slots < 0 || (d->scatter != 0 && d->scatter != 1))
        return IGEMM_EINVAL;
    const int st = check_product(d->a_rows, d->out_rows, d->n, d->k, d->groups, d->type);
    if (st != IGEMM_OK) return st;
    return d->rows > kMax || d->slots > kMax ? IGEMM_ENOTSUP : IGEMM_OK;
}

int check_adapters(const igemm_adapters_desc *d) {
    if (d == nullptr || d->adapters < 0 || d->rank < 0 || !half_type(d->weight_type))
        return IGEMM_EINVAL;
    const int st = check_product(d->m, d->m, d->n, d->k, 1, d->type);
    if (st != IGEMM_OK) return st;
    return d->adapters > kMax || d->rank > 1024 ? IGEMM_ENOTSUP : IGEMM_OK;
}

bool nothing(const igemm_grouped_desc &d) {
    return d.rows == 0 || d.n == 0 || d.groups == 0 || d.a_rows == 0 || d.out_rows == 0;
}

}  // namespace
}  // namespace rows
}  // namespace igemm

using namespace igemm::rows;

extern "C" {

int igemm_route_query(const igemm_route_desc *desc, int64_t *workspace_bytes) {
    if (workspace_bytes == nullptr) return IGEMM_EINVAL;
    *workspace_bytes = 0;
    const int st = check_route(desc);
    if (st != IGEMM_OK) return st;
    *workspace_bytes = route_workspace(*desc, true);
    return IGEMM_OK;
}

int igemm_route(const igemm_route_desc *desc, const void *logits, int64_t ld, const float *bias,
                int32_t *ids, float *weights, int32_t *offsets, int32_t *order, void *workspace,
                int64_t workspace_bytes, void *stream) {
    int st = check_route(desc);
    if (st != IGEMM_OK) return st;
    const igemm_route_desc &d = *desc;
    const bool plan = offsets != nullptr;
    if (plan != (order != nullptr) && !(plan && d.tokens == 0)) return IGEMM_EINVAL;
    if (d.tokens > 0) {
        if (logits == nullptr || ids == nullptr || weights == nullptr || ld < d.experts ||
            !aligned(logits, size_of(d.type)))
            return IGEMM_EINVAL;
        if (extent(d.tokens, d.experts, ld, size_of(d.type)) < 0) return IGEMM_ENOTSUP;
    }
    if (!aligned(bias, 4) || !aligned(ids, 4) || !aligned(weights, 4) || !aligned(offsets, 4) ||
        !aligned(order, 4))
        return IGEMM_EINVAL;
    st = check_workspace(workspace, workspace_bytes, route_workspace(d, plan));
    if (st != IGEMM_OK || (d.tokens == 0 && !plan)) return st;
    return launch_route(d, logits, ld, bias, ids, weights, offsets, order, workspace, stream);
}

int igemm_i8_grouped_query(const igemm_grouped_desc *desc, int num_cu, int64_t *workspace_bytes) {
    if (workspace_bytes == nullptr || num_cu < 0) return IGEMM_EINVAL;
    *workspace_bytes = 0;
    const int st = check_grouped(desc);
    if (st != IGEMM_OK || nothing(*desc)) return st;
    *workspace_bytes = product_workspace(desc->rows, desc->n, desc->k, desc->groups, 0, 0,
                                         num_cu > 0 ? num_cu : 256);
    return IGEMM_OK;
}

int igemm_i8_grouped(const igemm_grouped_desc *desc, const int32_t *offsets,
                     const int32_t *order, const int8_t *A, int64_t lda, const float *scale_a,
                     const int8_t *B, int64_t ldb, int64_t stride_b, const float *scale_b,
                     void *out, int64_t ldo, void *workspace, int64_t workspace_bytes,
                     void *stream) {
    int st = check_grouped(desc);
    if (st != IGEMM_OK) return st;
    const igemm_grouped_desc &d = *desc;
    if (workspace != nullptr && (!aligned(workspace, 256) || workspace_bytes < 0))
        return IGEMM_EINVAL;
    if (nothing(d)) return IGEMM_OK;
    if (offsets == nullptr || !aligned(offsets, 4) || !aligned(order, 4) || stride_b < 0)
        return IGEMM_EINVAL;
    st = check_operands(d.a_rows, d.n, d.k, A, lda, B, ldb, out, ldo, d.type, scale_a, scale_b);
    if (st != IGEMM_OK) return st;
    if (d.k > 0 && extent(d.groups, 1, stride_b, 1) < 0) return IGEMM_ENOTSUP;
    const int num_cu = igemm::num_cu_of_current_device();
    st = check_workspace(workspace, workspace_bytes,
                         product_workspace(d.rows, d.n, d.k, d.groups, 0, 0, num_cu));
    if (st != IGEMM_OK) return st;
    const Product p = {A, B, scale_a, scale_b, offsets, order, out, lda, ldb, stride_b, ldo,
                       (int)d.rows, (int)d.n, (int)d.k, (int)d.groups, (int)d.a_rows,
                       (int)d.out_rows, (int)d.slots, d.scatter, d.type};
    return launch_product(p, Adapters{}, num_cu, workspace, stream);
}

int igemm_combine(int64_t tokens, int64_t top_k, int64_t n, int type, const void *Z, int64_t ldz,
                  const float *weights, const int32_t *ids, const void *base, int64_t ld_base,
                  void *out, int64_t ldo, void *stream) {
    if (tokens < 0 || top_k < 1 || n < 0 || !type_ok(type)) return IGEMM_EINVAL;
    if (tokens > kMax || top_k > kMax || n > kMax) return IGEMM_ENOTSUP;
    if (tokens == 0 || n == 0) return IGEMM_OK;
    const int64_t es = size_of(type);
    if (Z == nullptr || weights == nullptr || out == nullptr || ldz < n || ldo < n ||
        (base != nullptr && ld_base < n) || !aligned(Z, es) || !aligned(base, es) ||
        !aligned(out, es) || !aligned(weights, 4) || !aligned(ids, 4))
        return IGEMM_EINVAL;
    if (extent(tokens * top_k, n, ldz, es) < 0 || extent(tokens, n, ldo, es) < 0 ||
        (base != nullptr && extent(tokens, n, ld_base, es) < 0))
        return IGEMM_ENOTSUP;
    return launch_combine(tokens, top_k, n, type, Z, ldz, weights, ids, base, ld_base, out, ldo,
                          stream);
}

int igemm_i8_adapters_query(const igemm_adapters_desc *desc, int num_cu,
                            int64_t *workspace_bytes) {
    if (workspace_bytes == nullptr || num_cu < 0) return IGEMM_EINVAL;
    *workspace_bytes = 0;
    const int st = check_adapters(desc);
    if (st != IGEMM_OK || desc->m == 0 || desc->n == 0) return st;
    *workspace_bytes = product_workspace(desc->m, desc->n, desc->k, 1, desc->adapters, desc->rank,
                                         num_cu > 0 ? num_cu : 256);
    return IGEMM_OK;
}

int igemm_i8_adapters(const igemm_adapters_desc *desc, const int8_t *A, int64_t lda,
                      const float *scale_a, const int8_t *B, int64_t ldb, const float *scale_b,
                      const int32_t *ids, const void *down, int64_t ld_down,
                      int64_t stride_down, const void *up, int64_t ld_up, int64_t stride_up,
                      const int32_t *ranks, const float *scaling, void *out, int64_t ldo,
                      void *workspace, int64_t workspace_bytes, void *stream) {
    int st = check_adapters(desc);
    if (st != IGEMM_OK) return st;
    const igemm_adapters_desc &d = *desc;
    if (workspace != nullptr && (!aligned(workspace, 256) || workspace_bytes < 0))
        return IGEMM_EINVAL;
    if (d.m == 0 || d.n == 0) return IGEMM_OK;
    st = check_operands(d.m, d.n, d.k, A, lda, B, ldb, out, ldo, d.type, scale_a, scale_b);
    if (st != IGEMM_OK) return st;
    Adapters ad = {};
    if (d.adapters > 0 && d.rank > 0 && d.k > 0) {
        if (ids == nullptr || down == nullptr || up == nullptr || ld_down < d.k ||
            ld_up < d.rank || stride_down < 0 || stride_up < 0 || !aligned(ids, 4) ||
            !aligned(down, 2) || !aligned(up, 2) || !aligned(ranks, 4) || !aligned(scaling, 4))
            return IGEMM_EINVAL;
        const int64_t dn = extent(d.rank, d.k, ld_down, 2), u = extent(d.n, d.rank, ld_up, 2);
        if (dn < 0 || dn > kMax || u < 0 || u > kMax ||
            extent(d.adapters, 1, stride_down, 2) < 0 || extent(d.adapters, 1, stride_up, 2) < 0)
            return IGEMM_ENOTSUP;
        ad = Adapters{ids, ranks, down, up, scaling, ld_down, stride_down, ld_up, stride_up,
                      (int)d.adapters, (int)d.rank, d.weight_type};
    }
    const int num_cu = igemm::num_cu_of_current_device();
    st = check_workspace(workspace, workspace_bytes,
                         product_workspace(d.m, d.n, d.k, 1, ad.adapters, ad.rank, num_cu));
    if (st != IGEMM_OK) return st;
    const Product p = {A, B, scale_a, scale_b, nullptr, nullptr, out, lda, ldb, 0, ldo,
                       (int)d.m, (int)d.n, (int)d.k, 1, (int)d.m, (int)d.m, 0, 0, d.type};
    return launch_product(p, ad, num_cu, workspace, stream);
}

}  // extern "C"
