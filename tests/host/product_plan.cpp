// Prints the plan of every "m n k exact" read from standard input: tile, splits, blocks of k of a workgroup, and whether few rows take
// 64 columns a workgroup.
#include <cstdio>

#include "../../paper_1702_05911_amd/csrc/product_plan.hpp"

int main() {
    long long m, n, k;
    int exact;
    while (std::scanf("%lld %lld %lld %d", &m, &n, &k, &exact) == 4) {
        const pqt::Plan p = pqt::plan_of(m, n, (int)((k + 127) / 128), exact != 0);
        std::printf("%d %d %d %d\n", p.tile, p.splits, p.per_split, p.tile == 16 && n >= pqt::kManyColumns);
    }
    return 0;
}
