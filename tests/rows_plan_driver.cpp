// Prints what igemm_rows_plan.cpp chooses for dense operands: one line for each line
// "rows n k groups adapters rank compute-units" read.
#include <cstdio>

#include "igemm_rows_internal.h"
using namespace igemm::rows;
int main() {
    long long rows, n, k, groups, adapters, rank;
    int cu;
    while (std::scanf("%lld %lld %lld %lld %lld %lld %d", &rows, &n, &k, &groups, &adapters, &rank,
                      &cu) == 7) {
        const Choice c = choose(rows, n, k, groups, adapters, rank, cu);
        Product p = {};
        p.rows = (int)rows, p.n = (int)n, p.k = (int)k, p.groups = (int)groups;
        p.lda = k, p.ldb = n, p.stride_b = groups > 1 ? k * n : 0;
        Adapters ad = {};
        ad.adapters = (int)adapters, ad.rank = (int)rank, ad.ld_up = rank;
        ad.stride_up = adapters > 1 ? n * rank : 0;
        const Tile t = tile_of(c, p, ad, cu);
        std::printf("%d %d %d %d %d %d %lld\n", t.bm, t.bn, t.reg, c.slices, c.by_row,
                    c.shrink_ranks, (long long)(c.part_bytes + c.u_bytes));
    }
    return 0;
}
